// The linear layer around the step: forward with bias, activation, residual and an 8-bit checkpoint of the
// pre-activation in the epilogue; input gradient with the slope of a checkpointed activation in the epilogue; weight
// gradient from a checkpoint. One product D[m, n] = sum_k A(m, k) B(n, k) serves all three:
//   forward   A = X  (k fast)              B = W (k fast)              M = tokens, N = rows, K = cols
//   input     A = dY (k fast)              B = W (n fast)              M = tokens, N = cols, K = rows
//   weight    A = dY (m fast)              B = act(v) (n fast)         M = rows,   N = cols, K = tokens
#include "sc_linear.cuh"

namespace sc {
namespace {

constexpr int kSimtTile = 64, kSimtK = 16;

template <typename T>
__device__ __forceinline__ float lin_ld(const void* p, int64_t i) { return (float)static_cast<const T*>(p)[i]; }

__device__ __forceinline__ float epi_read(const void* p, int f32, int64_t i) {
  return f32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const bf16*>(p)[i]);
}
__device__ __forceinline__ void epi_write(void* p, int f32, int64_t i, float v) {
  if (f32) static_cast<float*>(p)[i] = v;
  else static_cast<bf16*>(p)[i] = __float2bfloat16_rn(v);
}

// CUDA-core product in fp32: 64 x 64 tiles, 4 x 4 sums per thread, any strides. Serves fp32 operands and layouts that
// TMA cannot describe.
template <int KIND, typename T, bool A_KFAST, bool B_KFAST>
__global__ void __launch_bounds__(256)
linear_simt_kernel(const LinProblem p) {
  __shared__ float As[kSimtK][kSimtTile + 4], Bs[kSimtK][kSimtTile + 4];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int64_t tiles_n = (p.N + kSimtTile - 1) / kSimtTile;
  const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * kSimtTile, n0 = (int64_t)(blockIdx.x % tiles_n) * kSimtTile;
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < p.K; k0 += kSimtK) {
#pragma unroll
    for (int i = tid; i < kSimtTile * kSimtK; i += 256) {
      const int ra = A_KFAST ? i / kSimtK : i % kSimtTile, ka = A_KFAST ? i % kSimtK : i / kSimtTile;
      const int rb = B_KFAST ? i / kSimtK : i % kSimtTile, kb = B_KFAST ? i % kSimtK : i / kSimtTile;
      As[ka][ra] = (m0 + ra < p.M && k0 + ka < p.K) ? lin_ld<T>(p.A.base, (m0 + ra) * p.A.s_row + (k0 + ka) * p.A.s_k) : 0.f;
      Bs[kb][rb] = (n0 + rb < p.N && k0 + kb < p.K) ? lin_ld<T>(p.B.base, (n0 + rb) * p.B.s_row + (k0 + kb) * p.B.s_k) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSimtK; ++k) {
      const float4 a = *reinterpret_cast<const float4*>(&As[k][ty * 4]), b = *reinterpret_cast<const float4*>(&Bs[k][tx * 4]);
      const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
    }
    __syncthreads();
  }
  const LinEpilogue& e = p.epi;
  const int64_t n = n0 + tx * 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t m = m0 + ty * 4 + i;
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = acc[i][j];
    if (KIND == kEpiForward) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (e.bias && n + j < p.N) v[j] += e.bias[n + j];
        if (n + j >= p.N) v[j] = 0.f;
      }
      if (e.q) {              // 8 neighbouring threads hold a block of 32 columns
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const uint32_t eb = a8_scale_byte(top);
        if (m < p.M && n < e.wide) {
          *reinterpret_cast<uint32_t*>(e.q + m * e.wide + n) = a8_pack4(v[0], v[1], v[2], v[3], a8_inverse(eb));
          if ((tx & 7) == 0) e.e[m * (e.wide / 32) + n / 32] = (uint8_t)eb;
        }
      }
    }
    if (m >= p.M) continue;
    float s[4];
    if (KIND == kEpiInput && e.q && n < e.wide)
      a8_unpack4(*reinterpret_cast<const uint32_t*>(e.q + m * e.wide + n), a8_step(e.e[m * (e.wide / 32) + n / 32]), s);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (n + j >= p.N) break;
      float y = v[j];
      if (KIND == kEpiForward) {
        y = act_value_rt(e.act, y);
        if (e.res) y += epi_read(e.res, e.out_f32, m * e.ldr + n + j);
      } else if (KIND == kEpiInput) {
        if (e.q) y *= act_slope_rt(e.act, s[j]);
      } else {
        y *= e.scale;
      }
      epi_write(e.out, e.out_f32, m * e.ldo + n + j, y);
    }
  }
}

template <int KIND, typename T>
sc_status simt_kind(const LinProblem& p, cudaStream_t s) {
  const int64_t tiles = ((p.M + kSimtTile - 1) / kSimtTile) * ((p.N + kSimtTile - 1) / kSimtTile);
  if (tiles > 0x7fffffff) return SC_ERR_TOO_LARGE;
  linear_simt_kernel<KIND, T, KIND != kEpiWeight, KIND == kEpiForward><<<(unsigned)tiles, 256, 0, s>>>(p);
  ++g_kernel_launches;
  return cudaGetLastError() == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}

// column sums of dY over a slice of the tokens, then over the slices in order
constexpr int kColSlices = 64;
template <typename T>
__global__ void __launch_bounds__(128)
column_sum_kernel(const T* __restrict__ dY, float* __restrict__ part, int64_t tokens, int64_t rows, int64_t ld) {
  const int64_t c = (int64_t)blockIdx.x * 128 + threadIdx.x;
  if (c >= rows) return;
  float s = 0.f;
  for (int64_t t = blockIdx.y; t < tokens; t += gridDim.y) s += (float)dY[t * ld + c];
  part[(int64_t)blockIdx.y * rows + c] = s;
}
__global__ void __launch_bounds__(128)
column_join_kernel(const float* __restrict__ part, float* __restrict__ out, int slices, int64_t rows) {
  const int64_t c = (int64_t)blockIdx.x * 128 + threadIdx.x;
  if (c >= rows) return;
  float s = 0.f;
  for (int i = 0; i < slices; ++i) s += part[(int64_t)i * rows + c];
  out[c] = s;
}

sc_status check_dims(int64_t tokens, int64_t rows, int64_t cols) {
  if (tokens < 0 || rows <= 0 || cols <= 0) return SC_ERR_SHAPE;
  if (tokens > (1 << 30) || rows > (1 << 30) || cols > (1 << 30)) return SC_ERR_TOO_LARGE;
  return SC_OK;
}
bool is_dtype(int d) { return d == SC_DTYPE_BF16 || d == SC_DTYPE_FP32; }
bool is_act(int a) { return a >= SC_ACT_NONE && a <= SC_ACT_SILU; }
bool off(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == SC_DTYPE_BF16 ? 1 : 3)) != 0; }
bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

}  // namespace

sc_status linear_simt(int kind, int operand_f32, const LinProblem& p, cudaStream_t s) {
  switch (kind) {
    case kEpiForward: return operand_f32 ? simt_kind<kEpiForward, float>(p, s) : simt_kind<kEpiForward, bf16>(p, s);
    case kEpiInput: return operand_f32 ? simt_kind<kEpiInput, float>(p, s) : simt_kind<kEpiInput, bf16>(p, s);
    default: return operand_f32 ? simt_kind<kEpiWeight, float>(p, s) : simt_kind<kEpiWeight, bf16>(p, s);
  }
}

// bf16 operands that TMA can describe: tensor cores; everything else: CUDA cores.
static sc_status linear_run(int kind, int operand_f32, const LinProblem& p, unsigned* status, cudaStream_t s) {
  if (!operand_f32 && linear_tc_supported(p)) return linear_tc(kind, p, status, s);
  return linear_simt(kind, operand_f32, p, s);
}

}  // namespace sc

using namespace sc;

extern "C" sc_status sc_linear_forward(const void* X_dev, const void* W_dev, int operand_dtype, const void* bias_dev,
                                       const void* residual_dev, void* Y_dev, int out_dtype, int act, void* act8_dev,
                                       int64_t tokens, int64_t rows, int64_t cols, int64_t ldx, int64_t ldw, int64_t ldr,
                                       int64_t ldy, void* status_dev, void* stream) {
  if (!is_dtype(operand_dtype) || !is_dtype(out_dtype)) return SC_ERR_DTYPE;
  const sc_status st = check_dims(tokens, rows, cols);
  if (st != SC_OK) return st;
  if (!is_act(act)) return SC_ERR_INVALID_ARG;
  if (ldx < cols || ldw < cols || ldy < rows || (residual_dev && ldr < rows)) return SC_ERR_SHAPE;
  if (tokens == 0) return SC_OK;
  if (!X_dev || !W_dev || !Y_dev) return SC_ERR_INVALID_ARG;
  if (off(X_dev, operand_dtype) || off(W_dev, operand_dtype) || off(Y_dev, out_dtype) || off(residual_dev, out_dtype) ||
      off(bias_dev, SC_DTYPE_FP32) || off16(act8_dev) || off(status_dev, SC_DTYPE_FP32))
    return SC_ERR_ALIGNMENT;
  LinProblem p{};
  p.A = {X_dev, ldx, 1};
  p.B = {W_dev, ldw, 1};
  p.M = tokens; p.N = rows; p.K = cols;
  p.epi.out = Y_dev;
  p.epi.bias = static_cast<const float*>(bias_dev);
  p.epi.res = residual_dev;
  p.epi.ldo = ldy; p.epi.ldr = ldr;
  p.epi.out_f32 = out_dtype == SC_DTYPE_FP32;
  p.epi.act = act;
  if (act8_dev) {
    const Act8View v = act8_view(act8_dev, tokens, rows);
    p.epi.q = v.q; p.epi.e = v.e; p.epi.wide = v.wide;
  }
  return linear_run(kEpiForward, operand_dtype == SC_DTYPE_FP32, p, static_cast<unsigned*>(status_dev),
                    static_cast<cudaStream_t>(stream));
}

extern "C" sc_status sc_linear_backward_input(const void* dY_dev, const void* W_dev, int operand_dtype,
                                              const void* act8_dev, int act, void* dX_dev, int out_dtype, int64_t tokens,
                                              int64_t rows, int64_t cols, int64_t lddy, int64_t ldw, int64_t lddx,
                                              void* status_dev, void* stream) {
  if (!is_dtype(operand_dtype) || !is_dtype(out_dtype)) return SC_ERR_DTYPE;
  const sc_status st = check_dims(tokens, rows, cols);
  if (st != SC_OK) return st;
  if (!is_act(act) || (!act8_dev && act != SC_ACT_NONE)) return SC_ERR_INVALID_ARG;
  if (lddy < rows || ldw < cols || lddx < cols) return SC_ERR_SHAPE;
  if (tokens == 0) return SC_OK;
  if (!dY_dev || !W_dev || !dX_dev) return SC_ERR_INVALID_ARG;
  if (off(dY_dev, operand_dtype) || off(W_dev, operand_dtype) || off(dX_dev, out_dtype) || off16(act8_dev) ||
      off(status_dev, SC_DTYPE_FP32))
    return SC_ERR_ALIGNMENT;
  LinProblem p{};
  p.A = {dY_dev, lddy, 1};
  p.B = {W_dev, 1, ldw};
  p.M = tokens; p.N = cols; p.K = rows;
  p.epi.out = dX_dev;
  p.epi.ldo = lddx;
  p.epi.out_f32 = out_dtype == SC_DTYPE_FP32;
  p.epi.act = act;
  if (act8_dev && act != SC_ACT_NONE) {
    const Act8View v = act8_view(const_cast<void*>(act8_dev), tokens, cols);
    p.epi.q = v.q; p.epi.e = v.e; p.epi.wide = v.wide;
  }
  return linear_run(kEpiInput, operand_dtype == SC_DTYPE_FP32, p, static_cast<unsigned*>(status_dev),
                    static_cast<cudaStream_t>(stream));
}

extern "C" size_t sc_linear_weight_grad_workspace_bytes(int operand_dtype, int64_t tokens, int64_t rows, int64_t cols) {
  if (!is_dtype(operand_dtype) || check_dims(tokens, rows, cols) != SC_OK) return 0;
  const size_t wide = ((size_t)cols + 31) / 32 * 32;
  return (size_t)kColSlices * (size_t)rows * sizeof(float) + 16 + (size_t)tokens * wide * (operand_dtype == SC_DTYPE_FP32 ? 4 : 2);
}

extern "C" sc_status sc_linear_weight_grad(const void* dY_dev, int operand_dtype, const void* act8_dev, int act,
                                           float scale, void* G_dev, int out_dtype, void* dbias_dev, int64_t tokens,
                                           int64_t rows, int64_t cols, int64_t lddy, void* workspace,
                                           size_t workspace_bytes, void* status_dev, void* stream) {
  if (!is_dtype(operand_dtype) || !is_dtype(out_dtype)) return SC_ERR_DTYPE;
  sc_status st = check_dims(tokens, rows, cols);
  if (st != SC_OK) return st;
  if (!is_act(act) || !G_dev) return SC_ERR_INVALID_ARG;
  if (lddy < rows) return SC_ERR_SHAPE;
  if (tokens > 0 && (!dY_dev || !act8_dev)) return SC_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < sc_linear_weight_grad_workspace_bytes(operand_dtype, tokens, rows, cols))
    return SC_ERR_WORKSPACE;
  if (off(dY_dev, operand_dtype) || off(G_dev, out_dtype) || off16(act8_dev) || off16(workspace) ||
      off(dbias_dev, SC_DTYPE_FP32) || off(status_dev, SC_DTYPE_FP32))
    return SC_ERR_ALIGNMENT;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int64_t wide = (cols + 31) / 32 * 32;
  const size_t a_bytes = (size_t)tokens * wide * (operand_dtype == SC_DTYPE_FP32 ? 4 : 2);
  float* part = reinterpret_cast<float*>(static_cast<char*>(workspace) + (a_bytes + 15) / 16 * 16);
  if (tokens > 0) {
    st = sc_act8_expand(act8_dev, act, workspace, operand_dtype, tokens, cols, wide, stream);
    if (st != SC_OK) return st;
  }
  LinProblem p{};
  p.A = {dY_dev, 1, lddy};
  p.B = {workspace, 1, wide};
  p.M = rows; p.N = cols; p.K = tokens;
  p.epi.out = G_dev;
  p.epi.ldo = cols;
  p.epi.out_f32 = out_dtype == SC_DTYPE_FP32;
  p.epi.scale = scale;
  if (tokens == 0) {
    if (dbias_dev && cudaMemsetAsync(dbias_dev, 0, (size_t)rows * sizeof(float), s) != cudaSuccess) return SC_ERR_CUDA;
    return cudaMemsetAsync(G_dev, 0, (size_t)rows * (size_t)cols * (out_dtype == SC_DTYPE_FP32 ? 4 : 2), s) == cudaSuccess
               ? SC_OK : SC_ERR_CUDA;
  }
  const bool tensor = operand_dtype == SC_DTYPE_BF16 && linear_tc_supported(p);
  if (dbias_dev && tensor) {            // by the product's own blocks
    p.epi.dy = dY_dev;
    p.epi.db = static_cast<float*>(dbias_dev);
    p.epi.tokens = tokens;
    p.epi.ld_dy = lddy;
  } else if (dbias_dev) {
    const int slices = tokens < kColSlices ? (int)tokens : kColSlices;
    const unsigned blocks = (unsigned)((rows + 127) / 128);
    if (operand_dtype == SC_DTYPE_FP32)
      column_sum_kernel<float><<<dim3(blocks, slices), 128, 0, s>>>(static_cast<const float*>(dY_dev), part, tokens, rows, lddy);
    else
      column_sum_kernel<bf16><<<dim3(blocks, slices), 128, 0, s>>>(static_cast<const bf16*>(dY_dev), part, tokens, rows, lddy);
    column_join_kernel<<<blocks, 128, 0, s>>>(part, static_cast<float*>(dbias_dev), slices, rows);
    g_kernel_launches += 2;
  }
  return linear_run(kEpiWeight, operand_dtype == SC_DTYPE_FP32, p, static_cast<unsigned*>(status_dev), s);
}
