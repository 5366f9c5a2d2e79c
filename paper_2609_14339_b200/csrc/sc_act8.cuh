// Arithmetic of the 8-bit activation checkpoints and of the activations, shared by the kernels that write a checkpoint
// (compress, layer norm, the forward GEMM's epilogue) and those that read one.
#pragma once

#include "sc_internal.cuh"

namespace sc {

constexpr int kA8Block = 32;

// A checkpoint's two parts. Blocks of features are the slow index: block b of all tokens, 32 bytes a token, then block
// b + 1; the scale bytes lie the same way. A warp that holds 32 tokens' values of one block (a GEMM epilogue) then reads
// or writes 1 KB in one piece, and one that holds one token's (rows are 32 lanes there) 32 bytes, a whole sector.
struct Act8View {
  int8_t* q;
  uint8_t* e;
  int64_t tokens, wide;     // wide: features rounded up to 32
};
inline Act8View act8_view(void* blob, int64_t tokens, int64_t features) {
  Act8View v;
  v.tokens = tokens;
  v.wide = (features + kA8Block - 1) / kA8Block * kA8Block;
  v.q = static_cast<int8_t*>(blob);
  v.e = static_cast<uint8_t*>(blob) + (tokens * v.wide + 255) / 256 * 256;
  return v;
}
// places of feature f of token t, and of its block's scale byte
__device__ __forceinline__ int64_t a8_at(int64_t tokens, int64_t t, int64_t f) { return ((f >> 5) * tokens + t) * 32 + (f & 31); }
__device__ __forceinline__ int64_t a8_scale_at(int64_t tokens, int64_t t, int64_t f) { return (f >> 5) * tokens + t; }

// Scale byte of a block from the largest |x| (as bits; NaN and infinity compare above every finite value).
__device__ __forceinline__ uint32_t a8_scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return 255u;
  const int e = (int)(amax_bits >> 23) - 6;
  return e < 1 ? 1u : (uint32_t)e;
}
// 2^-e of a scale byte; 0 for a block of NaNs, whose integers are all stored as 0 (0 * inf = NaN on the way back).
__device__ __forceinline__ float a8_inverse(uint32_t byte) {
  return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23);
}
__device__ __forceinline__ float a8_step(uint32_t byte) { return __uint_as_float(byte << 23); }

// rint(x / 2^e) clamped to +-127, in the low byte. Adding 1.5 * 2^23 rounds to an integer (halves to even) that then
// stands in the low mantissa bits. fminf/fmaxf drop a NaN operand, so a NaN (its block's inverse is 0) gives a finite
// integer; a8_pack4's caller zeroes it through `keep`.
__device__ __forceinline__ uint32_t a8_round(float x, float inv) {
  const float v = fminf(fmaxf(x * inv, -127.f), 127.f);
  return __float_as_uint(v + 12582912.f);
}
// four integers' low bytes in one word
__device__ __forceinline__ uint32_t a8_pack4(float x0, float x1, float x2, float x3, float inv) {
  const uint32_t lo = __byte_perm(a8_round(x0, inv), a8_round(x1, inv), 0x0040);
  const uint32_t hi = __byte_perm(a8_round(x2, inv), a8_round(x3, inv), 0x0040);
  const uint32_t w = __byte_perm(lo, hi, 0x5410);
  return inv == 0.f ? 0u : w;
}
// the four values a word of integers stands for: byte b + 128 in the low mantissa bits of 2^23, minus 2^23 + 128
__device__ __forceinline__ void a8_unpack4(uint32_t w, float step, float* v) {
  const uint32_t u = w ^ 0x80808080u;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v[i] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7540 + i)) - 8388736.f) * step;
}

// ---- activations -----------------------------------------------------------------------------------------------
// One instruction each (the compiler's own forms spend several on denormal arguments, which cannot matter here: the
// reciprocal's argument is at least 1, and an exponential that small adds nothing).
__device__ __forceinline__ float fast_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2e = 1.4426950408889634f;

// Normal distribution function from Hastings' rational approximation of erfc (Abramowitz and Stegun 7.1.26, absolute error
// 1.5e-7 in erf): for x = |z| / sqrt(2), t = 1 / (1 + p x), erfc(x) = t (a1 + t (a2 + t (a3 + t (a4 + t a5)))) exp(-x^2).
// The lower tail comes out directly, not as 1 - (nearly 1), and the density the slope needs is the same exponential. Some
// 15 instructions, two of them on the special function unit (16 a clock and SM, which bounds the kernels that apply it).
__device__ __forceinline__ float normal_cdf(float z, float& exp_half_square) {
  const float t = fast_rcp(fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.f));
  exp_half_square = fast_exp2(z * z * (-0.5f * kLog2e));
  float p = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
  p = fmaf(t, p, 0.5f * 1.421413741f);
  p = fmaf(t, p, 0.5f * -0.284496736f);
  p = fmaf(t, p, 0.5f * 0.254829592f);
  const float tail = t * p * exp_half_square;
  return z >= 0.f ? 1.f - tail : tail;
}
__device__ __forceinline__ float sigmoid(float z) { return fast_rcp(1.f + fast_exp2(z * -kLog2e)); }
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if (ACT == SC_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
  if (ACT == SC_ACT_GELU) {
    float e;
    return z * normal_cdf(z, e);
  }
  if (ACT == SC_ACT_SILU) return z * sigmoid(z);
  return z;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if (ACT == SC_ACT_RELU) return z > 0.f ? 1.f : (z != z ? z : 0.f);
  if (ACT == SC_ACT_GELU) {
    float e;
    const float c = normal_cdf(z, e);
    return fmaf(z * 0.39894228040143268f, e, c);
  }
  if (ACT == SC_ACT_SILU) {
    const float s = sigmoid(z);
    return s * (1.f + z * (1.f - s));
  }
  return 1.f;
}

template <int N_, typename F>
__device__ __forceinline__ void each(float* v, F f) {
#pragma unroll
  for (int j = 0; j < N_; ++j) v[j] = f(v[j]);
}
// the activation is uniform over the launch: one branch per block of values
template <int N_>
__device__ __forceinline__ void act_values(int act, float* v) {
  switch (act) {
    case SC_ACT_RELU: each<N_>(v, [](float z) { return act_value<SC_ACT_RELU>(z); }); break;
    case SC_ACT_GELU: each<N_>(v, [](float z) { return act_value<SC_ACT_GELU>(z); }); break;
    case SC_ACT_SILU: each<N_>(v, [](float z) { return act_value<SC_ACT_SILU>(z); }); break;
    default: break;
  }
}
template <int N_>
__device__ __forceinline__ void act_slopes(int act, float* v) {
  switch (act) {
    case SC_ACT_RELU: each<N_>(v, [](float z) { return act_slope<SC_ACT_RELU>(z); }); break;
    case SC_ACT_GELU: each<N_>(v, [](float z) { return act_slope<SC_ACT_GELU>(z); }); break;
    case SC_ACT_SILU: each<N_>(v, [](float z) { return act_slope<SC_ACT_SILU>(z); }); break;
    default: each<N_>(v, [](float) { return 1.f; });
  }
}

// ---- eight neighbouring elements ---------------------------------------------------------------------------------
// n of them inside the row; vec: 16-byte accesses are allowed where all eight are
__device__ __forceinline__ void load8(const void* p, int f32, int64_t i, bool vec, int n, float* r) {
  if (vec && n >= 8) {
    if (f32) {
      const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
      const float4 b = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i + 4);
      r[0] = a.x; r[1] = a.y; r[2] = a.z; r[3] = a.w; r[4] = b.x; r[5] = b.y; r[6] = b.z; r[7] = b.w;
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const bf16*>(p) + i);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) { r[2 * j] = __uint_as_float(w[j] << 16); r[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      r[j] = j < n ? (f32 ? static_cast<const float*>(p)[i + j] : __bfloat162float(static_cast<const bf16*>(p)[i + j])) : 0.f;
  }
}
__device__ __forceinline__ void store8(void* p, int f32, int64_t i, bool vec, int n, const float* v) {
  if (vec && n >= 8) {
    if (f32) {
      float* o = static_cast<float*>(p) + i;
      *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&h);
      }
      *reinterpret_cast<uint4*>(static_cast<bf16*>(p) + i) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) {
        if (f32) static_cast<float*>(p)[i + j] = v[j];
        else static_cast<bf16*>(p)[i + j] = __float2bfloat16_rn(v[j]);
      }
  }
}

}  // namespace sc
