// Pieces that the kernels of 16-bit rows share: pairs of 16-bit values as fp32 and back,
// reductions over groups of lanes, 8-bit codes of scaled values.
#pragma once
#include "mxmoe_internal.h"

namespace mxmoe {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));

#define LANES_INL __device__ __attribute__((always_inline)) inline

// a row whose largest magnitude is below this counts as zero: qmax / amax would overflow
constexpr float kTinyAmax = 0x1p-118f;

template <int ACT> LANES_INL f32x2 unpack2(uint32_t w) {
  if constexpr (ACT == MXMOE_BF16) return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
  const f16x2 h = __builtin_bit_cast(f16x2, w);
  return f32x2{(float)h[0], (float)h[1]};
}
template <int ACT> LANES_INL uint32_t pack2(float lo, float hi) {
  if constexpr (ACT == MXMOE_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
  // (a product that was rounded to fp32 must not be fused with the conversion)
  asm("" : "+v"(lo), "+v"(hi));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, f16x2));
}

// Sums and maxima over groups of L lanes (every lane ends with the result): DPP
// moves inside 16 lanes, cross-lane moves beyond.
template <int C> LANES_INL int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, C, 0xf, 0xf, true); }
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;
template <int C> LANES_INL double add_dpp(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)dpp<C>((int)(uint32_t)b), hi = (uint32_t)dpp<C>((int)(b >> 32));
  return v + __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
template <int L> LANES_INL double lanes_sum(double v) {
  if constexpr (L > 1) v = add_dpp<kXor1>(v);
  if constexpr (L > 2) v = add_dpp<kXor2>(v);
  if constexpr (L > 4) v = add_dpp<kHalfMirror>(v);
  if constexpr (L > 8) v = add_dpp<kMirror>(v);
  if constexpr (L > 16) v += __shfl_xor(v, 16, 64);
  if constexpr (L > 32) v += __shfl_xor(v, 32, 64);
  return v;
}
LANES_INL uint32_t max2(uint32_t a, uint32_t b) {  // of packed 16-bit pairs
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int L> LANES_INL uint32_t lanes_max(uint32_t v) {
  if constexpr (L > 1) v = max2(v, (uint32_t)dpp<kXor1>((int)v));
  if constexpr (L > 2) v = max2(v, (uint32_t)dpp<kXor2>((int)v));
  if constexpr (L > 4) v = max2(v, (uint32_t)dpp<kHalfMirror>((int)v));
  if constexpr (L > 8) v = max2(v, (uint32_t)dpp<kMirror>((int)v));
  if constexpr (L > 16) v = max2(v, (uint32_t)__shfl_xor((int)v, 16, 64));
  if constexpr (L > 32) v = max2(v, (uint32_t)__shfl_xor((int)v, 32, 64));
  return v;
}
template <int L> LANES_INL uint32_t lanes_umax(uint32_t v) {
  if constexpr (L > 1) v = max(v, (uint32_t)dpp<kXor1>((int)v));
  if constexpr (L > 2) v = max(v, (uint32_t)dpp<kXor2>((int)v));
  if constexpr (L > 4) v = max(v, (uint32_t)dpp<kHalfMirror>((int)v));
  if constexpr (L > 8) v = max(v, (uint32_t)dpp<kMirror>((int)v));
  if constexpr (L > 16) v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
  if constexpr (L > 32) v = max(v, (uint32_t)__shfl_xor((int)v, 32, 64));
  return v;
}

// Codes of 4 values times inv.  |v inv| <= qmax (1 + 2^-23) rounds to qmax at the most, so
// nothing is clamped.  int8: adding 1.5 2^23 leaves the integer nearest to the product
// (ties to even) in the low bits.  FP8: the conversion rounds to the nearest e4m3,
// ties to even; a zero loses its sign.
LANES_INL uint32_t codes4(float a, float b, float c, float d, float inv, bool f8) {
  float v[4] = {a * inv, b * inv, c * inv, d * inv};
  if (f8) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
    const uint32_t u = (uint32_t)w;
    return u & (0x7f7f7f7fu | ((u & 0x7f7f7f7fu) + 0x7f7f7f7fu));
  }
  uint32_t q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    asm("" : "+v"(v[i]));  // the product is rounded before the addition
    q[i] = __float_as_uint(v[i] + 12582912.0f);
  }
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[3], q[2], 0x0c0c0400u),
                               __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u), 0x05040100u);
}

}  // namespace
}  // namespace mxmoe
