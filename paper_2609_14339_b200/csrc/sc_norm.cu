// Layer norm: forward (y, the row statistics, optionally y as an 8-bit checkpoint) and backward (dx with the residual
// branch's gradient added, dweight, dbias).
#include "sc_act8.cuh"

namespace sc {
namespace {

constexpr int kNormThreads = 256;
constexpr int kNormSlices = 296;       // row slices of the column sums at most (fixed-order two-stage reduction)

template <typename T>
__device__ __forceinline__ float ld1(const T* p);
template <>
__device__ __forceinline__ float ld1<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float ld1<bf16>(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st1(float* p, float v) { *p = v; }
__device__ __forceinline__ void st1(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

// sum over the block, the same value in every thread (fixed order: lanes, then warps)
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const int warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[warp] = v;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < n_warps; ++w) s += red[w];
  return s;
}

template <typename T>
__global__ void __launch_bounds__(kNormThreads)
norm_forward_kernel(const T* __restrict__ X, const float* __restrict__ weight, const float* __restrict__ bias, float eps,
                    T* __restrict__ Y, float* __restrict__ stats, int8_t* __restrict__ q, uint8_t* __restrict__ qe,
                    int64_t wide, int64_t rows, int cols, int64_t ldx, int64_t ldy) {
  __shared__ float red[kNormThreads / 32];
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* x = X + r * ldx;
    float s = 0.f;
    for (int c = threadIdx.x; c < cols; c += kNormThreads) s += ld1(x + c);
    const float mean = block_sum(s, red) / (float)cols;
    s = 0.f;
    for (int c = threadIdx.x; c < cols; c += kNormThreads) { const float d = ld1(x + c) - mean; s += d * d; }
    const float rstd = 1.f / sqrtf(block_sum(s, red) / (float)cols + eps);
    if (stats && threadIdx.x == 0) { stats[r] = mean; stats[rows + r] = rstd; }
    // the padding of the last block of 32 is written too, as zeros
    const int width = q ? (int)wide : cols;
    for (int c = threadIdx.x; c < (width + 31) / 32 * 32; c += kNormThreads) {
      float y = 0.f;
      if (c < cols) {
        y = (ld1(x + c) - mean) * rstd;
        if (weight) y *= weight[c];
        if (bias) y += bias[c];
      }
      if (q) {       // 32 neighbouring columns are the 32 lanes of a warp
        const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(y) & 0x7fffffffu);
        const uint32_t e = a8_scale_byte(top);
        const float inv = a8_inverse(e);
        q[r * wide + c] = (int8_t)(inv == 0.f ? 0u : a8_round(y, inv) & 255u);
        if ((threadIdx.x & 31) == 0) qe[r * (wide / 32) + c / 32] = (uint8_t)e;
      }
      if (c < cols) st1(Y + r * ldy + c, y);
    }
    __syncthreads();
  }
}

template <typename T>
__global__ void __launch_bounds__(kNormThreads)
norm_backward_kernel(const T* dY, const T* __restrict__ X, const float* __restrict__ weight,
                     const float* __restrict__ stats, const T* R, T* dX, int64_t rows, int cols, int64_t lddy,
                     int64_t ldx, int64_t ldr, int64_t lddx) {
  __shared__ float red[kNormThreads / 32];
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const T *x = X + r * ldx, *dy = dY + r * lddy;
    const float mean = stats[r], rstd = stats[rows + r];
    float s0 = 0.f, s1 = 0.f;
    for (int c = threadIdx.x; c < cols; c += kNormThreads) {
      const float g = ld1(dy + c) * (weight ? weight[c] : 1.f);
      s0 += g;
      s1 += g * (ld1(x + c) - mean) * rstd;
    }
    const float m0 = block_sum(s0, red) / (float)cols, m1 = block_sum(s1, red) / (float)cols;
    for (int c = threadIdx.x; c < cols; c += kNormThreads) {
      const float g = ld1(dy + c) * (weight ? weight[c] : 1.f);
      float v = rstd * (g - m0 - (ld1(x + c) - mean) * rstd * m1);
      if (R) v += ld1(R + r * ldr + c);
      st1(dX + r * lddx + c, v);
    }
    __syncthreads();
  }
}

// column sums of dY n and dY over one slice of the rows
template <typename T>
__global__ void __launch_bounds__(128)
norm_columns_kernel(const T* __restrict__ dY, const T* __restrict__ X, const float* __restrict__ stats,
                    float* __restrict__ part, int64_t rows, int cols, int64_t lddy, int64_t ldx) {
  const int c = blockIdx.x * 128 + threadIdx.x;
  if (c >= cols) return;
  float sw = 0.f, sb = 0.f;
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
    const float d = ld1(dY + r * lddy + c);
    sw += d * ((ld1(X + r * ldx + c) - stats[r]) * stats[rows + r]);
    sb += d;
  }
  part[((size_t)blockIdx.y * 2 + 0) * cols + c] = sw;
  part[((size_t)blockIdx.y * 2 + 1) * cols + c] = sb;
}

__global__ void __launch_bounds__(128)
norm_columns_join_kernel(const float* __restrict__ part, int slices, float* __restrict__ dweight,
                         float* __restrict__ dbias, int cols) {
  const int c = blockIdx.x * 128 + threadIdx.x;
  if (c >= cols) return;
  float sw = 0.f, sb = 0.f;
  for (int s = 0; s < slices; ++s) {
    sw += part[((size_t)s * 2 + 0) * cols + c];
    sb += part[((size_t)s * 2 + 1) * cols + c];
  }
  if (dweight) dweight[c] = sw;
  if (dbias) dbias[c] = sb;
}

int norm_slices(int64_t rows) { return rows < kNormSlices ? (int)(rows > 0 ? rows : 1) : kNormSlices; }

sc_status check_rows(int64_t rows, int64_t cols) {
  if (rows < 0 || cols <= 0) return SC_ERR_SHAPE;
  if (rows > (1 << 30) || cols > (1 << 30)) return SC_ERR_TOO_LARGE;
  return SC_OK;
}
int elem(int dtype) { return dtype == SC_DTYPE_BF16 ? 2 : 4; }
bool off(const void* p, int n) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(n - 1)) != 0; }

template <typename T>
sc_status forward(const void* X, const void* w, const void* b, float eps, void* Y, void* stats, void* act8, int64_t rows,
                  int64_t cols, int64_t ldx, int64_t ldy, cudaStream_t s) {
  Act8View v{};
  if (act8) v = act8_view(act8, rows, cols);
  const unsigned grid = (unsigned)(rows < (1 << 20) ? rows : (1 << 20));
  norm_forward_kernel<T><<<grid, kNormThreads, 0, s>>>(static_cast<const T*>(X), static_cast<const float*>(w),
                                                       static_cast<const float*>(b), eps, static_cast<T*>(Y),
                                                       static_cast<float*>(stats), v.q, v.e, v.wide, rows, (int)cols, ldx,
                                                       ldy);
  ++g_kernel_launches;
  return cudaGetLastError() == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}

template <typename T>
sc_status backward(const void* dY, const void* X, const void* w, const void* stats, const void* R, void* dX, void* dw,
                   void* db, int64_t rows, int64_t cols, int64_t lddy, int64_t ldx, int64_t ldr, int64_t lddx, float* part,
                   cudaStream_t s) {
  const unsigned blocks = (unsigned)((cols + 127) / 128);
  int slices = 0;
  if (rows > 0 && (dw || db)) {       // before dX is written: dX may be dY
    slices = norm_slices(rows);
    norm_columns_kernel<T><<<dim3(blocks, slices), 128, 0, s>>>(static_cast<const T*>(dY), static_cast<const T*>(X),
                                                                static_cast<const float*>(stats), part, rows, (int)cols,
                                                                lddy, ldx);
    ++g_kernel_launches;
  }
  if (dw || db) {
    norm_columns_join_kernel<<<blocks, 128, 0, s>>>(part, slices, static_cast<float*>(dw), static_cast<float*>(db),
                                                    (int)cols);
    ++g_kernel_launches;
  }
  if (rows > 0) {
    const unsigned grid = (unsigned)(rows < (1 << 20) ? rows : (1 << 20));
    norm_backward_kernel<T><<<grid, kNormThreads, 0, s>>>(static_cast<const T*>(dY), static_cast<const T*>(X),
                                                          static_cast<const float*>(w), static_cast<const float*>(stats),
                                                          static_cast<const T*>(R), static_cast<T*>(dX), rows, (int)cols,
                                                          lddy, ldx, ldr, lddx);
    ++g_kernel_launches;
  }
  return cudaGetLastError() == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" sc_status sc_layernorm_forward(const void* X_dev, int dtype, const void* weight_dev, const void* bias_dev,
                                          float eps, void* Y_dev, void* stats_dev, void* act8_dev, int64_t rows,
                                          int64_t cols, int64_t ldx, int64_t ldy, void* stream) {
  if (dtype != SC_DTYPE_BF16 && dtype != SC_DTYPE_FP32) return SC_ERR_DTYPE;
  const sc_status st = check_rows(rows, cols);
  if (st != SC_OK) return st;
  if (!(eps >= 0.f)) return SC_ERR_INVALID_ARG;
  if (ldx < cols || ldy < cols) return SC_ERR_SHAPE;
  if (rows == 0) return SC_OK;
  if (!X_dev || !Y_dev) return SC_ERR_INVALID_ARG;
  if (off(X_dev, elem(dtype)) || off(Y_dev, elem(dtype)) || off(weight_dev, 4) || off(bias_dev, 4) || off(stats_dev, 4) ||
      off(act8_dev, 16))
    return SC_ERR_ALIGNMENT;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return dtype == SC_DTYPE_BF16
             ? forward<bf16>(X_dev, weight_dev, bias_dev, eps, Y_dev, stats_dev, act8_dev, rows, cols, ldx, ldy, s)
             : forward<float>(X_dev, weight_dev, bias_dev, eps, Y_dev, stats_dev, act8_dev, rows, cols, ldx, ldy, s);
}

extern "C" size_t sc_layernorm_workspace_bytes(int64_t rows, int64_t cols) {
  if (check_rows(rows, cols) != SC_OK) return 0;
  return (size_t)norm_slices(rows) * 2 * (size_t)cols * sizeof(float);
}

extern "C" sc_status sc_layernorm_backward(const void* dY_dev, const void* X_dev, int dtype, const void* weight_dev,
                                           const void* stats_dev, const void* residual_grad_dev, void* dX_dev,
                                           void* dweight_dev, void* dbias_dev, int64_t rows, int64_t cols, int64_t lddy,
                                           int64_t ldx, int64_t ldr, int64_t lddx, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  if (dtype != SC_DTYPE_BF16 && dtype != SC_DTYPE_FP32) return SC_ERR_DTYPE;
  const sc_status st = check_rows(rows, cols);
  if (st != SC_OK) return st;
  if (lddy < cols || ldx < cols || lddx < cols || (residual_grad_dev && ldr < cols)) return SC_ERR_SHAPE;
  if (rows > 0 && (!dY_dev || !X_dev || !stats_dev || !dX_dev)) return SC_ERR_INVALID_ARG;
  if ((dweight_dev || dbias_dev) && (!workspace || workspace_bytes < sc_layernorm_workspace_bytes(rows, cols)))
    return SC_ERR_WORKSPACE;
  if (off(dY_dev, elem(dtype)) || off(X_dev, elem(dtype)) || off(dX_dev, elem(dtype)) ||
      off(residual_grad_dev, elem(dtype)) || off(weight_dev, 4) || off(stats_dev, 4) || off(dweight_dev, 4) ||
      off(dbias_dev, 4) || off(workspace, 16))
    return SC_ERR_ALIGNMENT;
  if (rows == 0 && !dweight_dev && !dbias_dev) return SC_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  float* part = static_cast<float*>(workspace);
  return dtype == SC_DTYPE_BF16 ? backward<bf16>(dY_dev, X_dev, weight_dev, stats_dev, residual_grad_dev, dX_dev,
                                                 dweight_dev, dbias_dev, rows, cols, lddy, ldx, ldr, lddx, part, s)
                                : backward<float>(dY_dev, X_dev, weight_dev, stats_dev, residual_grad_dev, dX_dev,
                                                  dweight_dev, dbias_dev, rows, cols, lddy, ldx, ldr, lddx, part, s);
}
