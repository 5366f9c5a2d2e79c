// Arithmetic of the 8-bit activation checkpoints and of the activations, shared by the kernels that write a checkpoint
// (compress, layer norm, the forward GEMM's epilogue) and those that read one.
#pragma once

#include "sc_internal.cuh"

namespace sc {

constexpr int kA8Block = 32;

struct Act8View {           // a checkpoint's two parts
  int8_t* q;                // tokens x wide
  uint8_t* e;               // tokens x wide / 32
  int64_t wide;             // features rounded up to 32
};
inline Act8View act8_view(void* blob, int64_t tokens, int64_t features) {
  Act8View v;
  v.wide = (features + kA8Block - 1) / kA8Block * kA8Block;
  v.q = static_cast<int8_t*>(blob);
  v.e = static_cast<uint8_t*>(blob) + (tokens * v.wide + 255) / 256 * 256;
  return v;
}

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
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if (ACT == SC_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
  if (ACT == SC_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
  if (ACT == SC_ACT_SILU) return __fdividef(z, 1.f + __expf(-z));
  return z;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if (ACT == SC_ACT_RELU) return z > 0.f ? 1.f : (z != z ? z : 0.f);
  if (ACT == SC_ACT_GELU)
    return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * 0.39894228040143268f * __expf(-0.5f * z * z);
  if (ACT == SC_ACT_SILU) {
    const float s = __fdividef(1.f, 1.f + __expf(-z));
    return s * (1.f + z * (1.f - s));
  }
  return 1.f;
}

}  // namespace sc
