// The linear layer around the step: forward with bias, activation, residual and an 8-bit checkpoint of the
// pre-activation in the epilogue; input gradient with the slope of a checkpointed activation in the epilogue; weight
// gradient from a checkpoint. One product D[m, n] = sum_k A(m, k) B(n, k) serves all three:
//   forward   A = X  (k fast)              B = W (k fast)              M = tokens, N = rows, K = cols
//   input     A = dY (k fast)              B = W (n fast)              M = tokens, N = cols, K = rows
//   weight    A = dY (m fast)              B = act(v) (n fast)         M = rows,   N = cols, K = tokens
#include "sc_linear.cuh"
#include "sc_ptx.cuh"

namespace sc {
namespace {

constexpr int kSimtM = 64, kSimtN = 128, kSimtK = 16;

// four neighbouring elements, n of them inside the row; vec: 8- or 16-byte accesses where all four are
__device__ __forceinline__ void load4(const void* p, int f32, int64_t i, bool vec, int n, float* r) {
  if (f32) {
    const float* s = static_cast<const float*>(p) + i;
    if (vec && n == 4) {
      const float4 f = *reinterpret_cast<const float4*>(s);
      r[0] = f.x; r[1] = f.y; r[2] = f.z; r[3] = f.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) r[j] = j < n ? s[j] : 0.f;
    }
  } else {
    const bf16* s = static_cast<const bf16*>(p) + i;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = j < n ? __bfloat162float(s[j]) : 0.f;
  }
}
__device__ __forceinline__ void store4(void* p, int f32, int64_t i, bool vec, int n, const float* v) {
  if (f32) {
    float* o = static_cast<float*>(p) + i;
    if (vec && n == 4) {
      *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < n) o[j] = v[j];
    }
  } else {
    bf16* o = static_cast<bf16*>(p) + i;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) o[j] = __float2bfloat16_rn(v[j]);
  }
}

// CUDA-core product in fp32: 64 x 128 tiles, 8 x 8 sums per thread, any strides. Serves fp32 operands and layouts that
// TMA cannot describe. 300 x 1001 x 999: 28 us, 21 TFLOP/s; 2.1 instructions a clock and SM, the loads and stores of shared
// and global memory being what they wait for. With 8 x 8 sums four of five instructions are multiply-adds, with 4 x 4 half
// of them (40 us then). Few tiles (that result has 40) would leave SMs idle and each block a long
// serial sum, so the contraction is split over a cluster of up to 8 blocks, joined through distributed shared memory in a
// fixed order; the next 16 terms are in flight (registers) while the present ones are summed.
constexpr int kSimtThreads = 128;
struct SimtTile {
  float a[kSimtK][kSimtM + 4], b[kSimtK][kSimtN + 4];
};

// This thread's elements of a ROWS x 16 operand tile. K fast: a warp takes 4 rows x 8 terms at a time (whole sectors, and
// no two lanes in one bank of the transposed store); otherwise 32 rows of one term. Element j lies a constant number of
// rows and terms from element 0, so an address is one multiply-add.
template <typename T, bool KFAST, int ROWS>
struct SimtLoader {
  static constexpr int kEach = ROWS * kSimtK / kSimtThreads, kBlocks = ROWS / 32;
  const T* at;                   // element 0 of the tile to come
  int64_t s_slow;                // stride of the dimension that is not contiguous
  int row, term;                 // element 0's place in the tile
  int rows_left;                 // rows of the operand from the tile's first on
  int64_t K;
  float x[kEach];
  __device__ SimtLoader(const LinOperand& o, int64_t rows, int64_t K_, int64_t row0, int64_t k0) : K(K_) {
    const int u = (threadIdx.x >> 5) * kEach, lane = threadIdx.x & 31;
    row = KFAST ? (u >> 1) * 4 + (lane >> 3) : (u % kBlocks) * 32 + lane;
    term = KFAST ? (lane & 7) : u / kBlocks;
    s_slow = KFAST ? o.s_row : o.s_k;
    const int64_t left = rows - row0;
    rows_left = left < ROWS ? (int)left : ROWS;
    at = static_cast<const T*>(o.base) + (row0 + row) * o.s_row + (k0 + term) * o.s_k;
  }
  __device__ static constexpr int drow(int j) { return KFAST ? (j >> 1) * 4 : (j % kBlocks) * 32; }
  __device__ static constexpr int dterm(int j) { return KFAST ? (j & 1) * 8 : j / kBlocks; }
  // the tile from term k0 on; moves on to the next
  __device__ void load(int64_t k0) {
    const int k_left = K - k0 < kSimtK ? (int)(K - k0) : kSimtK;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const T* src = KFAST ? at + drow(j) * s_slow + dterm(j) : at + dterm(j) * s_slow + drow(j);
      x[j] = row + drow(j) < rows_left && term + dterm(j) < k_left ? (float)*src : 0.f;
    }
    at += KFAST ? kSimtK : kSimtK * s_slow;
  }
  __device__ void store(float (*s)[ROWS + 4]) const {
#pragma unroll
    for (int j = 0; j < kEach; ++j) s[term + dterm(j)][row + drow(j)] = x[j];
  }
};

// what becomes of 4 neighbouring sums of row m, columns n..n+3; all 32 lanes of a warp call it together
template <int KIND>
__device__ __forceinline__ void simt_epilogue(const LinProblem& p, float* v, int64_t m, int64_t n, int tx, bool vec) {
  const LinEpilogue& e = p.epi;
  const int64_t room = p.N - n;
  const int left = m < p.M && room > 0 ? (room < 4 ? (int)room : 4) : 0;
  float aux[4] = {0.f, 0.f, 0.f, 0.f};
  if (KIND == kEpiForward && e.res) load4(e.res, e.out_f32, m * e.ldr + n, vec, left, aux);
  if (KIND == kEpiInput && e.q && left > 0) {
    a8_unpack4(*reinterpret_cast<const uint32_t*>(e.q + a8_at(p.M, m, n)), a8_step(e.e[a8_scale_at(p.M, m, n)]), aux);
    act_slopes<4>(e.act, aux);
  }
  if (KIND == kEpiForward) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = j < room ? v[j] + (e.bias ? __ldg(e.bias + n + j) : 0.f) : 0.f;
    if (e.q) {              // 8 neighbouring threads hold a block of 32 columns
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      const uint32_t eb = a8_scale_byte(top);
      if (m < p.M && n < e.wide) {
        *reinterpret_cast<uint32_t*>(e.q + a8_at(p.M, m, n)) = a8_pack4(v[0], v[1], v[2], v[3], a8_inverse(eb));
        if ((tx & 7) == 0) e.e[a8_scale_at(p.M, m, n)] = (uint8_t)eb;
      }
    }
    act_values<4>(e.act, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += aux[j];
  } else if (KIND == kEpiInput) {
    if (e.q)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] *= aux[j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] *= e.scale;
  }
  store4(e.out, e.out_f32, m * e.ldo + n, vec, left, v);
}

template <int KIND, typename T, bool A_KFAST, bool B_KFAST>
__global__ void __launch_bounds__(kSimtThreads)
linear_simt_kernel(const __grid_constant__ LinProblem p, unsigned split) {
  __shared__ __align__(16) union {
    SimtTile tile[2];
    float4 sums[kSimtM][kSimtN / 4];
  } sm;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;         // rows ty * 4 and 32 + ty * 4, columns tx * 4 and 64 + tx * 4
  const unsigned part = blockIdx.x % split;
  const unsigned t = blockIdx.x / split, tiles_n = (unsigned)((p.N + kSimtN - 1) / kSimtN);
  const int64_t m0 = (int64_t)(t / tiles_n) * kSimtM, n0 = (int64_t)(t % tiles_n) * kSimtN;
  const unsigned steps = (unsigned)((p.K + kSimtK - 1) / kSimtK);           // at most 2^26
  const int64_t first = steps * part / split, last = steps * (part + 1) / split;
  SimtLoader<T, A_KFAST, kSimtM> la(p.A, p.M, p.K, m0, first * kSimtK);
  SimtLoader<T, B_KFAST, kSimtN> lb(p.B, p.N, p.K, n0, first * kSimtK);
  float acc[8][8] = {};
  chain_wait();
  chain_go();
  if (first < last) {
    la.load(first * kSimtK);
    lb.load(first * kSimtK);
  }
  int buf = 0;
  for (int64_t step = first; step < last; ++step, buf ^= 1) {
    la.store(sm.tile[buf].a);
    lb.store(sm.tile[buf].b);
    __syncthreads();           // the other buffer's readers passed the barrier of the step before
    if (step + 1 < last) {
      la.load((step + 1) * kSimtK);
      lb.load((step + 1) * kSimtK);
    }
#pragma unroll 8
    for (int k = 0; k < kSimtK; ++k) {
      float av[8], bv[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 a = *reinterpret_cast<const float4*>(&sm.tile[buf].a[k][h * 32 + ty * 4]);
        const float4 b = *reinterpret_cast<const float4*>(&sm.tile[buf].b[k][h * 64 + tx * 4]);
        av[4 * h] = a.x; av[4 * h + 1] = a.y; av[4 * h + 2] = a.z; av[4 * h + 3] = a.w;
        bv[4 * h] = b.x; bv[4 * h + 1] = b.y; bv[4 * h + 2] = b.z; bv[4 * h + 3] = b.w;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
    }
  }
  // The tile's partial sums go to shared memory; each block of the cluster adds up its share of the rows. A lone block
  // takes the same way: the epilogue then exists once, in a loop (unrolled over the registers it was 15 us of instruction
  // fetches for the smallest call).
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h)
      sm.sums[(i >> 2) * 32 + ty * 4 + (i & 3)][h * 16 + tx] =
          make_float4(acc[i][4 * h], acc[i][4 * h + 1], acc[i][4 * h + 2], acc[i][4 * h + 3]);
  if (split > 1) cluster_sync_all();
  else __syncthreads();
  const int begin = (int)(kSimtM * part / split), end = (int)(kSimtM * (part + 1) / split);
  const bool vec = p.epi.ldo % 4 == 0 && p.epi.ldr % 4 == 0 &&
                   ((reinterpret_cast<uintptr_t>(p.epi.out) | reinterpret_cast<uintptr_t>(p.epi.res)) & 15) == 0;
#pragma unroll 2
  for (int i0 = begin * 2; i0 < end * 2; i0 += kSimtThreads / 16) {                 // half a row per 16 threads; whole warps
    const int i = i0 + ty, r = i >> 1, c = (i & 1) * 16 + tx;
    const bool mine = i < end * 2;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (mine && split > 1) {
      const uint32_t at = smem_u32(&sm.sums[r][c]);
      float4 w[8];
#pragma unroll
      for (unsigned s = 0; s < 8; ++s)              // all of them on their way before the first is added
        if (s < split) w[s] = ld_shared_cluster4(map_to_rank(at, s));
#pragma unroll
      for (unsigned s = 0; s < 8; ++s)
        if (s < split) { v[0] += w[s].x; v[1] += w[s].y; v[2] += w[s].z; v[3] += w[s].w; }
    } else if (mine) {
      const float4 f = sm.sums[r][c];
      v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
    }
    simt_epilogue<KIND>(p, v, mine ? m0 + r : p.M, n0 + c * 4, tx, vec);
  }
  if (split > 1) cluster_sync_all();            // the peers have read this block's sums
}

template <int KIND, typename T>
sc_status simt_kind(const LinProblem& p, cudaStream_t s) {
  const int64_t tiles = ((p.M + kSimtM - 1) / kSimtM) * ((p.N + kSimtN - 1) / kSimtN);
  const int64_t steps = (p.K + kSimtK - 1) / kSimtK;
  // Clocks of the SM with the most blocks, from measured ones: a step of one block alone takes 2500 (its four warps wait for
  // shared memory and for each other), of two side by side 2800, of three 3200; the epilogue 600 for each of a block's
  // share of 16 turns, a join 2500.
  int split = 1;
  double best = 1e30;
  for (int k = 1; k <= 8 && k <= steps; k += k == 6 ? 2 : 1) {        // clusters of 7 fit the chip badly
    const int64_t per_sm = (tiles * k + 147) / 148, rounds = (per_sm + 2) / 3, beside = per_sm < 3 ? per_sm : 3;
    const double step = beside == 1 ? 2500.0 : beside == 2 ? 2800.0 : 3200.0;
    const double cost = (double)rounds * ((double)((steps + k - 1) / k) * step + 600.0 * (16 / k + 1) + (k > 1 ? 2500.0 : 0.0));
    if (cost < best) { best = cost; split = k; }
  }
  if (tiles * split > 0x7fffffff) return SC_ERR_TOO_LARGE;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(tiles * split));
  cfg.blockDim = dim3(kSimtThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)split;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  chain_attribute(&attr[1]);
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, linear_simt_kernel<KIND, T, KIND != kEpiWeight, KIND == kEpiForward>, p, (unsigned)split) != cudaSuccess)
    return SC_ERR_CUDA;
  ++g_kernel_launches;
  return cudaGetLastError() == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}

// column sums of dY over a slice of the tokens, then over the slices in order
constexpr int kColSlices = 64;
template <typename T>
__global__ void __launch_bounds__(128)
column_sum_kernel(const T* __restrict__ dY, float* __restrict__ part, int64_t tokens, int64_t rows, int64_t ld) {
  chain_wait();
  chain_go();
  const int64_t c = (int64_t)blockIdx.x * 128 + threadIdx.x;
  if (c >= rows) return;
  float s = 0.f;
  for (int64_t t = blockIdx.y; t < tokens; t += gridDim.y) s += (float)dY[t * ld + c];
  part[(int64_t)blockIdx.y * rows + c] = s;
}
__global__ void __launch_bounds__(128)
column_join_kernel(const float* __restrict__ part, float* __restrict__ out, int slices, int64_t rows) {
  chain_wait();
  chain_go();
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
    // Rounded to the operands' type, as the forward product's operand was: without an activation that is exact (7 bits times
    // a power of two), with one it is the rounding of a bf16 activation (2^-8 of each value at most).
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
      launch_chained(column_sum_kernel<float>, dim3(blocks, slices), 128, 0, s, static_cast<const float*>(dY_dev), part, tokens, rows, lddy);
    else
      launch_chained(column_sum_kernel<bf16>, dim3(blocks, slices), 128, 0, s, static_cast<const bf16*>(dY_dev), part, tokens, rows, lddy);
    launch_chained(column_join_kernel, dim3(blocks), 128, 0, s, part, static_cast<float*>(dbias_dev), slices, rows);
    g_kernel_launches += 2;
  }
  return linear_run(kEpiWeight, operand_dtype == SC_DTYPE_FP32, p, static_cast<unsigned*>(status_dev), s);
}
