// Activations kept in 8 bits: compress, expand (with an activation applied) and the gradient through an activation whose
// argument was kept. Elementwise, bound by HBM: 3 bytes a value for bf16 tensors, 5 for the gradient.
#include "sc_act8.cuh"

namespace sc {
namespace {

template <typename T>
__device__ __forceinline__ float ld1(const T* p) { return (float)*p; }
template <typename T>
__device__ __forceinline__ T cvt(float v);
template <>
__device__ __forceinline__ float cvt<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 cvt<bf16>(float v) { return __float2bfloat16_rn(v); }

// one warp per block of 32 features
template <typename T>
__global__ void __launch_bounds__(256)
a8_compress_kernel(const T* __restrict__ X, int8_t* __restrict__ q, uint8_t* __restrict__ qe, int64_t wide,
                   int64_t tokens, int64_t features, int64_t ldx) {
  const int lane = threadIdx.x & 31;
  const int64_t per_row = wide / 32, total = tokens * per_row;
  for (int64_t b = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); b < total; b += (int64_t)gridDim.x * 8) {
    const int64_t t = b / per_row, c = (b - t * per_row) * 32 + lane;
    const float x = c < features ? ld1(X + t * ldx + c) : 0.f;
    const uint32_t e = a8_scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(x) & 0x7fffffffu));
    const float inv = a8_inverse(e);
    q[t * wide + c] = (int8_t)(inv == 0.f ? 0u : a8_round(x, inv) & 255u);
    if (lane == 0) qe[b] = (uint8_t)e;
  }
}

// Y = act(v), or with dA: Y = dA * act'(v)
template <typename T, int ACT, bool GRAD>
__global__ void __launch_bounds__(256)
a8_expand_kernel(const int8_t* __restrict__ q, const uint8_t* __restrict__ qe, int64_t wide, const T* dA, T* Y,
                 int64_t tokens, int64_t features, int64_t ldda, int64_t ldy) {
  const int lane = threadIdx.x & 31;
  const int64_t per_row = wide / 32, total = tokens * per_row;
  for (int64_t b = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); b < total; b += (int64_t)gridDim.x * 8) {
    const int64_t t = b / per_row, c = (b - t * per_row) * 32 + lane;
    if (c >= features) continue;
    const float v = (float)q[t * wide + c] * a8_step(qe[b]);
    Y[t * ldy + c] = cvt<T>(GRAD ? ld1(dA + t * ldda + c) * act_slope<ACT>(v) : act_value<ACT>(v));
  }
}

unsigned grid_for(int64_t blocks32) {
  const int64_t g = (blocks32 + 7) / 8;
  return (unsigned)(g < 148 * 32 ? g : 148 * 32);
}

sc_status check(const void* act8, int dtype, int64_t tokens, int64_t features) {
  if (dtype != SC_DTYPE_BF16 && dtype != SC_DTYPE_FP32) return SC_ERR_DTYPE;
  if (tokens < 0 || features <= 0) return SC_ERR_SHAPE;
  if (tokens > (1 << 30) || features > (1 << 30)) return SC_ERR_TOO_LARGE;
  if (tokens > 0 && !act8) return SC_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(act8) & 15) return SC_ERR_ALIGNMENT;
  return SC_OK;
}
bool off(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == SC_DTYPE_BF16 ? 1 : 3)) != 0; }

template <typename T, int ACT, bool GRAD>
void expand_one(const Act8View& v, const void* dA, void* Y, int64_t tokens, int64_t features, int64_t ldda, int64_t ldy,
                cudaStream_t s) {
  a8_expand_kernel<T, ACT, GRAD><<<grid_for(tokens * (v.wide / 32)), 256, 0, s>>>(
      v.q, v.e, v.wide, static_cast<const T*>(dA), static_cast<T*>(Y), tokens, features, ldda, ldy);
}
template <typename T, bool GRAD>
void expand_act(const Act8View& v, int act, const void* dA, void* Y, int64_t tokens, int64_t features, int64_t ldda,
                int64_t ldy, cudaStream_t s) {
  switch (act) {
    case SC_ACT_RELU: expand_one<T, SC_ACT_RELU, GRAD>(v, dA, Y, tokens, features, ldda, ldy, s); break;
    case SC_ACT_GELU: expand_one<T, SC_ACT_GELU, GRAD>(v, dA, Y, tokens, features, ldda, ldy, s); break;
    case SC_ACT_SILU: expand_one<T, SC_ACT_SILU, GRAD>(v, dA, Y, tokens, features, ldda, ldy, s); break;
    default: expand_one<T, SC_ACT_NONE, GRAD>(v, dA, Y, tokens, features, ldda, ldy, s);
  }
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" size_t sc_act8_bytes(int64_t tokens, int64_t features) {
  if (tokens < 0 || features <= 0 || tokens > (1 << 30) || features > (1 << 30)) return 0;
  const size_t wide = ((size_t)features + 31) / 32 * 32;
  const size_t head = ((size_t)tokens * wide + 255) / 256 * 256;
  return (head + (size_t)tokens * (wide / 32) + 15) / 16 * 16 + 16;      // never 0 on valid input
}

extern "C" sc_status sc_act8_compress(const void* X_dev, int dtype, void* act8_dev, int64_t tokens, int64_t features,
                                      int64_t ldx, void* stream) {
  const sc_status st = check(act8_dev, dtype, tokens, features);
  if (st != SC_OK) return st;
  if (ldx < features) return SC_ERR_SHAPE;
  if (tokens == 0) return SC_OK;
  if (!X_dev) return SC_ERR_INVALID_ARG;
  if (off(X_dev, dtype)) return SC_ERR_ALIGNMENT;
  const Act8View v = act8_view(act8_dev, tokens, features);
  const unsigned grid = grid_for(tokens * (v.wide / 32));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == SC_DTYPE_BF16)
    a8_compress_kernel<bf16><<<grid, 256, 0, s>>>(static_cast<const bf16*>(X_dev), v.q, v.e, v.wide, tokens, features, ldx);
  else
    a8_compress_kernel<float><<<grid, 256, 0, s>>>(static_cast<const float*>(X_dev), v.q, v.e, v.wide, tokens, features, ldx);
  ++g_kernel_launches;
  return cudaGetLastError() == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}

extern "C" sc_status sc_act8_expand(const void* act8_dev, int act, void* Y_dev, int dtype, int64_t tokens,
                                    int64_t features, int64_t ldy, void* stream) {
  const sc_status st = check(act8_dev, dtype, tokens, features);
  if (st != SC_OK) return st;
  if (act < SC_ACT_NONE || act > SC_ACT_SILU) return SC_ERR_INVALID_ARG;
  if (ldy < features) return SC_ERR_SHAPE;
  if (tokens == 0) return SC_OK;
  if (!Y_dev) return SC_ERR_INVALID_ARG;
  if (off(Y_dev, dtype)) return SC_ERR_ALIGNMENT;
  const Act8View v = act8_view(const_cast<void*>(act8_dev), tokens, features);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == SC_DTYPE_BF16) expand_act<bf16, false>(v, act, nullptr, Y_dev, tokens, features, 0, ldy, s);
  else expand_act<float, false>(v, act, nullptr, Y_dev, tokens, features, 0, ldy, s);
  ++g_kernel_launches;
  return cudaGetLastError() == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}

extern "C" sc_status sc_act8_backward(const void* dA_dev, const void* act8_dev, int act, void* dZ_dev, int dtype,
                                      int64_t tokens, int64_t features, int64_t ldda, int64_t lddz, void* stream) {
  const sc_status st = check(act8_dev, dtype, tokens, features);
  if (st != SC_OK) return st;
  if (act < SC_ACT_NONE || act > SC_ACT_SILU) return SC_ERR_INVALID_ARG;
  if (ldda < features || lddz < features) return SC_ERR_SHAPE;
  if (tokens == 0) return SC_OK;
  if (!dA_dev || !dZ_dev) return SC_ERR_INVALID_ARG;
  if (off(dA_dev, dtype) || off(dZ_dev, dtype)) return SC_ERR_ALIGNMENT;
  const Act8View v = act8_view(const_cast<void*>(act8_dev), tokens, features);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == SC_DTYPE_BF16) expand_act<bf16, true>(v, act, dA_dev, dZ_dev, tokens, features, ldda, lddz, s);
  else expand_act<float, true>(v, act, dA_dev, dZ_dev, tokens, features, ldda, lddz, s);
  ++g_kernel_launches;
  return cudaGetLastError() == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}
