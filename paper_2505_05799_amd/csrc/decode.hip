// One packed linear on the few rows of a decode step: out = a W^T + bias in one
// launch, no plan and no workspace.
//
// Weights stream as the fragment blocks of 16 channels by 128 k that the packer
// writes; the rows are the A operand (16 rows a fragment), the weights the B
// operand, so that a lane's four accumulators share one channel:
//   w4g128  per k block b:  out += s_b (sum_k a q - z_b sum_k a).  bf16: the codes become
//           128 + q (an OR), and 128 + z is taken off through the row sums, an MFMA of the rows
//           against ones; fp16: 1024 + q, from which a packed subtraction of
//           1024 + z leaves q - z.  Both are exact in their dtype.
//   w8a8    int8 MFMA, int32 sums; fp8  FP8 MFMA, fp32 sums; times s_a s_w at the end.
#include "mxmoe_internal.h"

namespace mxmoe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int ACT> __device__ inline f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (ACT == MXMOE_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <int ACT> __device__ inline float act_load(const uint16_t* p) {
  if constexpr (ACT == MXMOE_BF16) return __uint_as_float((uint32_t)*p << 16);
  else return (float)__builtin_bit_cast(_Float16, *p);
}
template <int ACT> __device__ inline uint16_t act_round(float f) {
  asm("" : "+v"(f));  // the fp32 value is rounded, not the expression it came from
  if constexpr (ACT == MXMOE_BF16) return __builtin_bit_cast(uint16_t, (__bf16)f);
  else return __builtin_bit_cast(uint16_t, (_Float16)f);
}

// One wavefront per 16 channels and 16 rows.
template <int KD, int ACT>
__global__ void __launch_bounds__(64) decode_kernel(DecodeArgs p) {
  const int lane = threadIdx.x, li = lane & 15, qd = lane >> 4;
  const int kb_n = p.k / 128;
  const int row = min((int)blockIdx.y * 16 + li, p.m - 1);  // rows past the last repeat it: their sums are dropped
  const uint8_t* wb = p.packed + (int64_t)blockIdx.x * kb_n * block_bytes(KD);
  f32x4 tot = {0.f, 0.f, 0.f, 0.f};
  i32x4 itot = {0, 0, 0, 0};
  for (int kb = 0; kb < kb_n; ++kb, wb += block_bytes(KD)) {
    const u32x4* wl = reinterpret_cast<const u32x4*>(wb + lane * lane_bytes(KD));
    if constexpr (KD == K_W4G) {
      const u32x4 d = wl[0];
      const uint32_t sz = reinterpret_cast<const uint32_t*>(wb + 64 * lane_bytes(KD))[li];
      const float s = (float)__builtin_bit_cast(_Float16, (uint16_t)sz);
      const _Float16 z = __builtin_bit_cast(_Float16, (uint16_t)(sz >> 16));
      const u32x4* ar = reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(p.a) + row * p.lda + kb * 128);
      f32x4 acc = {0.f, 0.f, 0.f, 0.f}, rs = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u32x4 a = ar[4 * j + qd];
        u32x4 b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t v = (d[j] >> (4 * i)) & 0x000F000Fu;
          if constexpr (ACT == MXMOE_BF16) {
            v |= 0x43004300u;
          } else {
            const _Float16 off = (_Float16)1024.f + z;
            v = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, v | 0x64006400u) - f16x2{off, off});
          }
          b[i] = v;
        }
        acc = mfma16<ACT>(a, b, acc);
        if constexpr (ACT == MXMOE_BF16) rs = mfma16<ACT>(a, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}, rs);
      }
      if constexpr (ACT == MXMOE_BF16) acc -= (128.f + (float)z) * rs;
      tot += s * acc;
    } else {
      const u32x4* ar = reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(p.a) + row * p.lda + kb * 128);
      const u32x4 a0 = ar[qd], a1 = ar[4 + qd], w0 = wl[0], w1 = wl[1];
      if constexpr (KD == K_W8A8) {
        itot = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a0), __builtin_bit_cast(i32x4, w0), itot, 0, 0, 0);
        itot = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a1), __builtin_bit_cast(i32x4, w1), itot, 0, 0, 0);
      } else {
        const i32x8 A = {(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
        const i32x8 B = {(int)w0[0], (int)w0[1], (int)w0[2], (int)w0[3], (int)w1[0], (int)w1[1], (int)w1[2], (int)w1[3]};
        tot = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, tot, 0, 0, 0, 127, 0, 127);
      }
    }
  }
  const int ch = blockIdx.x * 16 + li;
  const float bias = p.bias ? act_load<ACT>(reinterpret_cast<const uint16_t*>(p.bias) + ch) : 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = blockIdx.y * 16 + 4 * qd + i;
    if (r >= p.m) continue;
    float v = KD == K_W8A8 ? (float)itot[i] : tot[i];
    if constexpr (KD != K_W4G) v = v * p.a_scales[r] * p.wscale[ch];
    reinterpret_cast<uint16_t*>(p.out)[r * p.ldo + ch] = act_round<ACT>(v + bias);
  }
}

template <int KD> hipError_t launch_kind(const DecodeArgs& p, int act, hipStream_t s) {
  const dim3 grid(p.n / 16, (p.m + 15) / 16);
  if (act == MXMOE_BF16) hipLaunchKernelGGL((decode_kernel<KD, MXMOE_BF16>), grid, dim3(64), 0, s, p);
  else hipLaunchKernelGGL((decode_kernel<KD, MXMOE_F16>), grid, dim3(64), 0, s, p);
  return hipGetLastError();
}

}  // namespace

bool decode_kind(int kind) { return kind == K_W4G || kind == K_W8A8 || kind == K_F8A8; }

hipError_t launch_linear_decode(const DecodeArgs& p, int kind, int act, hipStream_t s) {
  switch (kind) {
    case K_W4G: return launch_kind<K_W4G>(p, act, s);
    case K_W8A8: return launch_kind<K_W8A8>(p, act, s);
    default: return launch_kind<K_F8A8>(p, act, s);
  }
}

}  // namespace mxmoe
