// Activations kept in 8 bits: compress, expand (with an activation applied) and the gradient through an activation whose
// argument was kept. Elementwise, bound by HBM: 3 bytes a value for bf16 tensors, 5 for the gradient.
#include "sc_act8.cuh"

namespace sc {
namespace {

constexpr int kA8Unroll = 4;

// Work is cut into units of 8 features (four neighbouring lanes hold a block of 32). A thread takes kA8Unroll units at a
// time, all of them loaded before the first is used: HBM latency times bandwidth is some 45 KB per SM, and one unit per
// thread in flight leaves much of it idle.
// FLAT: no row ends inside a unit's block and rows follow one another without a gap in the tensor and the checkpoint, so
// the unit's number is all that is needed; otherwise row and column advance from unit to unit without a division.
template <bool FLAT>
struct A8Walk {
  int64_t row, unit, step;
  int col8, step_col8, units_row;
  int64_t step_row;
  __device__ A8Walk(int64_t wide) {
    unit = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    step = (int64_t)gridDim.x * blockDim.x;
    if (!FLAT) {
      units_row = (int)(wide / 8);
      row = unit / units_row;
      col8 = (int)(unit - row * units_row);
      step_row = step / units_row;
      step_col8 = (int)(step - step_row * units_row);
    }
  }
  __device__ void next() {
    unit += step;
    if (!FLAT) {
      row += step_row;
      col8 += step_col8;
      if (col8 >= units_row) { col8 -= units_row; ++row; }
    }
  }
  __device__ int64_t at(int64_t ld) const { return FLAT ? unit * 8 : row * ld + col8 * 8; }
  __device__ int left(int features) const { return FLAT ? 8 : features - col8 * 8; }
};
// 8 elements as they lie in memory (16 or 32 bytes), loaded before they are converted
template <bool F32>
struct Raw8 {
  uint4 w[F32 ? 2 : 1];
  __device__ void load(const void* p, int64_t i) {
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const char*>(p) + i * (F32 ? 4 : 2));
    w[0] = src[0];
    if (F32) w[1] = src[1];
  }
  __device__ void get(float* x) const {
    const uint32_t* r = reinterpret_cast<const uint32_t*>(w);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      x[j] = F32 ? __uint_as_float(r[j]) : __uint_as_float(j & 1 ? r[j / 2] & 0xffff0000u : r[j / 2] << 16);
  }
};

__device__ __forceinline__ void a8_write_unit(const float* x, int8_t* q, uint8_t* qe, int64_t unit, bool live) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const uint32_t e = a8_scale_byte(top);
  const float inv = a8_inverse(e);
  if (live) {
    reinterpret_cast<uint2*>(q)[unit] = make_uint2(a8_pack4(x[0], x[1], x[2], x[3], inv), a8_pack4(x[4], x[5], x[6], x[7], inv));
    if ((threadIdx.x & 3) == 0) qe[unit / 4] = (uint8_t)e;
  }
}

// units: tokens * wide / 8. A checkpoint's rows follow one another without a gap, so a unit's number is its place in it.
template <bool F32, bool FLAT>
__global__ void __launch_bounds__(256)
a8_compress_kernel(const void* __restrict__ X, int8_t* __restrict__ q, uint8_t* __restrict__ qe, int64_t wide,
                   int64_t units, int features, int64_t ldx, bool vec) {
  A8Walk<FLAT> w(wide);
  // whole warps leave together: the shuffles need them (units is a multiple of 4, not of 32)
  while (__any_sync(0xffffffffu, w.unit < units)) {
    const int64_t unit0 = w.unit;
    if (FLAT) {
      Raw8<F32> r[kA8Unroll];
#pragma unroll
      for (int u = 0; u < kA8Unroll; ++u) {
        if (w.unit < units) r[u].load(X, w.unit * 8);
        else r[u] = Raw8<F32>{};
        w.next();
      }
#pragma unroll
      for (int u = 0; u < kA8Unroll; ++u) {
        float x[8];
        r[u].get(x);
        a8_write_unit(x, q, qe, unit0 + u * w.step, unit0 + u * w.step < units);
      }
    } else {
      float x[kA8Unroll][8];
#pragma unroll
      for (int u = 0; u < kA8Unroll; ++u) {
        load8(X, F32, w.at(ldx), vec, w.unit < units ? w.left(features) : 0, x[u]);
        w.next();
      }
#pragma unroll
      for (int u = 0; u < kA8Unroll; ++u) a8_write_unit(x[u], q, qe, unit0 + u * w.step, unit0 + u * w.step < units);
    }
  }
}

// Y = act(v), or GRAD: Y = dA * act'(v). dA and Y may be the same matrix.
template <bool F32, int ACT, bool GRAD, bool FLAT>
__global__ void __launch_bounds__(256)
a8_expand_kernel(const int8_t* __restrict__ q, const uint8_t* __restrict__ qe, int64_t wide, const void* dA, void* Y,
                 int64_t units, int features, int64_t ldda, int64_t ldy, bool vec) {
  A8Walk<FLAT> w(wide);
  while (w.unit < units) {
    A8Walk<FLAT> o = w;
    uint2 b[kA8Unroll];
    uint32_t e[kA8Unroll];
    Raw8<F32> raw[GRAD && FLAT ? kA8Unroll : 1];
#pragma unroll
    for (int u = 0; u < kA8Unroll; ++u) {
      if (w.unit < units) {
        b[u] = __ldcs(reinterpret_cast<const uint2*>(q) + w.unit);
        e[u] = qe[w.unit / 4];
        if (GRAD && FLAT) raw[u].load(dA, w.unit * 8);
      }
      w.next();
    }
#pragma unroll
    for (int u = 0; u < kA8Unroll; ++u) {
      const int n = o.unit < units ? o.left(features) : 0;
      if (n > 0) {
        float v[8], a[8];
        if (GRAD && FLAT) raw[u].get(a);
        if (GRAD && !FLAT) load8(dA, F32, o.at(ldda), vec, n, a);
        a8_unpack4(b[u].x, a8_step(e[u]), v);
        a8_unpack4(b[u].y, a8_step(e[u]), v + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = GRAD ? a[j] * act_slope<ACT>(v[j]) : act_value<ACT>(v[j]);
        store8(Y, F32, o.at(ldy), vec, n, v);
      }
      o.next();
    }
  }
}

unsigned grid_for(int64_t units) {
  const int64_t g = (units + 256 * kA8Unroll - 1) / (256 * kA8Unroll), most = 148 * 16;
  return (unsigned)(g < most ? g : most);
}
bool vec_ok(const void* p, int64_t ld, int dtype) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld * (dtype == SC_DTYPE_BF16 ? 2 : 4)) % 16 == 0;
}
// one stretch of memory whose blocks of 32 are the checkpoint's (a single row of full blocks too)
bool flat_ok(const void* p, int64_t ld, int64_t tokens, int64_t features) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && features % 32 == 0 && (ld == features || tokens == 1);
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

template <bool F32, int ACT, bool GRAD>
void expand_one(const Act8View& v, const void* dA, void* Y, int64_t tokens, int64_t features, int64_t ldda, int64_t ldy,
                cudaStream_t s) {
  const int dtype = F32 ? SC_DTYPE_FP32 : SC_DTYPE_BF16;
  const int64_t units = tokens * (v.wide / 8);
  const unsigned grid = grid_for(units);
  if (flat_ok(Y, ldy, tokens, features) && (!GRAD || flat_ok(dA, ldda, tokens, features))) {
    a8_expand_kernel<F32, ACT, GRAD, true><<<grid, 256, 0, s>>>(v.q, v.e, v.wide, dA, Y, units, (int)features, ldda, ldy, true);
  } else {
    const bool vec = vec_ok(Y, ldy, dtype) && (!GRAD || vec_ok(dA, ldda, dtype));
    a8_expand_kernel<F32, ACT, GRAD, false><<<grid, 256, 0, s>>>(v.q, v.e, v.wide, dA, Y, units, (int)features, ldda, ldy, vec);
  }
}
template <bool F32, bool GRAD>
void expand_act(const Act8View& v, int act, const void* dA, void* Y, int64_t tokens, int64_t features, int64_t ldda,
                int64_t ldy, cudaStream_t s) {
  switch (act) {
    case SC_ACT_RELU: expand_one<F32, SC_ACT_RELU, GRAD>(v, dA, Y, tokens, features, ldda, ldy, s); break;
    case SC_ACT_GELU: expand_one<F32, SC_ACT_GELU, GRAD>(v, dA, Y, tokens, features, ldda, ldy, s); break;
    case SC_ACT_SILU: expand_one<F32, SC_ACT_SILU, GRAD>(v, dA, Y, tokens, features, ldda, ldy, s); break;
    default: expand_one<F32, SC_ACT_NONE, GRAD>(v, dA, Y, tokens, features, ldda, ldy, s);
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
  const int64_t units = tokens * (v.wide / 8);
  const unsigned grid = grid_for(units);
  const bool vec = vec_ok(X_dev, ldx, dtype), flat = flat_ok(X_dev, ldx, tokens, features);
  const int n = (int)features;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == SC_DTYPE_BF16) {
    if (flat) a8_compress_kernel<false, true><<<grid, 256, 0, s>>>(X_dev, v.q, v.e, v.wide, units, n, ldx, vec);
    else a8_compress_kernel<false, false><<<grid, 256, 0, s>>>(X_dev, v.q, v.e, v.wide, units, n, ldx, vec);
  } else {
    if (flat) a8_compress_kernel<true, true><<<grid, 256, 0, s>>>(X_dev, v.q, v.e, v.wide, units, n, ldx, vec);
    else a8_compress_kernel<true, false><<<grid, 256, 0, s>>>(X_dev, v.q, v.e, v.wide, units, n, ldx, vec);
  }
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
  if (dtype == SC_DTYPE_BF16) expand_act<false, false>(v, act, nullptr, Y_dev, tokens, features, 0, ldy, s);
  else expand_act<true, false>(v, act, nullptr, Y_dev, tokens, features, 0, ldy, s);
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
  if (dtype == SC_DTYPE_BF16) expand_act<false, true>(v, act, dA_dev, dZ_dev, tokens, features, ldda, lddz, s);
  else expand_act<true, true>(v, act, dA_dev, dZ_dev, tokens, features, ldda, lddz, s);
  ++g_kernel_launches;
  return cudaGetLastError() == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}
