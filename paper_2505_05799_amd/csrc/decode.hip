// One packed linear on the few rows of a decode step: out = a W^T + bias in one
// launch, no plan and no workspace.
//
// Weights stream as the fragment blocks of 16 channels by 128 k that the packer
// writes; the rows are the A operand (16 rows a fragment), the weights the B
// operand, so that a lane's four accumulators share one channel:
//   w4g128  per k block b:  out += s_b (sum_k a q - z_b sum_k a).  bf16: the codes become
//           16 + q (an OR), and 16 + z is taken off through the row sums, an MFMA of the rows
//           against ones: the difference of two fp32 sums, which err by parts of
//           sum |a| (16 + q) and not of sum |a (q - z)|.  16 is the least offset that leaves 16
//           codes one exponent (128, where the codes need no shift of their own, errs five
//           times as much and overflows sooner; q - z itself takes 6 operations for two
//           codes, this takes 2).  fp16: 1024 + q, from which a packed subtraction of
//           1024 + z leaves q - z.  All of them are exact in their dtype.
//   w8a8    int8 MFMA, int32 sums; fp8  FP8 MFMA, fp32 sums; times s_a s_w at the end.
//
// The wavefronts of a workgroup take the k blocks of its channels in turn and meet once,
// through LDS, in wavefront order.  Rows past the last one repeat it (their sums are
// dropped).  A launch is bound by the weights' way from memory for few rows, and by the
// rows' way from the L2 to every CU for many.
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

#define DEC_INL __device__ __attribute__((always_inline)) inline

template <int ACT> DEC_INL f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (ACT == MXMOE_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
DEC_INL float act_load(const uint16_t* p, int act) {
  return act == MXMOE_BF16 ? __uint_as_float((uint32_t)*p << 16) : (float)__builtin_bit_cast(_Float16, *p);
}
DEC_INL uint16_t act_round(float f, int act) {
  asm("" : "+v"(f));  // the fp32 value is rounded, not the expression it came from
  return act == MXMOE_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)f) : __builtin_bit_cast(uint16_t, (_Float16)f);
}

// What a lane holds of one k block: its weights (and the group's scale and zero point),
// and the rows of a fragment (16-byte pieces: four of 16-bit rows, two of codes).
template <int KD> struct Wgt {
  static constexpr int N = lane_bytes(KD) / 16;
  u32x4 w[N];
  uint32_t sz;
  // block: the fragment block of the lane's channels and this k block
  DEC_INL void load(const uint8_t* block, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const u32x4*>(block + lane * lane_bytes(KD))[i];
    if constexpr (KD == K_W4G) sz = reinterpret_cast<const uint32_t*>(block + 64 * lane_bytes(KD))[lane & 15];
  }
};
template <int KD> constexpr int kPieces = KD == K_W4G ? 4 : 2;
template <int KD, int MF> using Rows = u32x4[MF][kPieces<KD>];
template <int KD> struct AccT { using type = f32x4; };
template <> struct AccT<K_W8A8> { using type = i32x4; };
template <int KD> using Acc = typename AccT<KD>::type;

// Row sums of a k block over the group (bf16 rows of w4g128), in the accumulators' layout.
template <int KD, int ACT, int MF> DEC_INL void row_sums(const Rows<KD, MF>& a, f32x4 (&rs)[MF]) {
  if constexpr (KD == K_W4G && ACT == MXMOE_BF16) {
#pragma unroll
    for (int f = 0; f < MF; ++f) {
      rs[f] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        rs[f] = mfma16<ACT>(a[f][j], u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}, rs[f]);
    }
  }
}

template <int KD, int ACT, int MF>
DEC_INL void use_block(const Wgt<KD>& s, const Rows<KD, MF>& a, const f32x4 (&rs)[MF], Acc<KD> (&tot)[MF]) {
  if constexpr (KD == K_W4G) {
    const float sc = (float)__builtin_bit_cast(_Float16, (uint16_t)s.sz);
    const _Float16 z = __builtin_bit_cast(_Float16, (uint16_t)(s.sz >> 16));
    f32x4 acc[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) acc[f] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u32x4 b;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t v;
        if constexpr (ACT == MXMOE_BF16) {  // 16 + q = 0x4180 | q << 3
          v = ((i ? s.w[0][j] >> (4 * i - 3) : s.w[0][j] << 3) & 0x00780078u) | 0x41804180u;
        } else {
          v = (s.w[0][j] >> (4 * i)) & 0x000F000Fu;
          const _Float16 off = (_Float16)1024.f + z;
          v = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, v | 0x64006400u) - f16x2{off, off});
        }
        b[i] = v;
      }
#pragma unroll
      for (int f = 0; f < MF; ++f) acc[f] = mfma16<ACT>(a[f][j], b, acc[f]);
    }
#pragma unroll
    for (int f = 0; f < MF; ++f) {
      if constexpr (ACT == MXMOE_BF16) acc[f] -= (16.f + (float)z) * rs[f];
      tot[f] += sc * acc[f];
    }
  } else if constexpr (KD == K_W8A8) {
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        tot[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a[f][j]), __builtin_bit_cast(i32x4, s.w[j]), tot[f], 0, 0, 0);
  } else {
    auto wide = [](u32x4 l, u32x4 h) { return i32x8{(int)l[0], (int)l[1], (int)l[2], (int)l[3], (int)h[0], (int)h[1], (int)h[2], (int)h[3]}; };
#pragma unroll
    for (int f = 0; f < MF; ++f)
      tot[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(a[f][0], a[f][1]), wide(s.w[0], s.w[1]), tot[f], 0, 0, 0, 127, 0, 127);
  }
}

// The wavefronts' sums of one block of channels, added in wavefront order, to the
// output.  red: [NW][MF][64] accumulators in LDS.  Output o = 64 (4 f + i) + l:
// fragment f, row 4 (l / 16) + i of it, channel l % 16.
template <int KD, int MF, int NW>
DEC_INL void write_out(const DecodeArgs& p, const Acc<KD>* red, int nb, int t, int threads) {
  for (int o = t; o < MF * 256; o += threads) {
    const int l = o & 63, i = (o >> 6) & 3, f = o >> 8, r = 16 * f + 4 * (l >> 4) + i;
    if (r >= p.m) continue;
    auto v = red[f * 64 + l][i];
#pragma unroll
    for (int j = 1; j < NW; ++j) v += red[(j * MF + f) * 64 + l][i];
    const int c = nb * 16 + (l & 15);
    float x = (float)v;
    if constexpr (KD != K_W4G) x = x * p.a_scales[r] * p.wscale[c];
    if (p.bias) x += act_load(reinterpret_cast<const uint16_t*>(p.bias) + c, p.act);
    reinterpret_cast<uint16_t*>(p.out)[(int64_t)r * p.ldo + c] = act_round(x, p.act);
  }
}

// LDS operations of a wavefront are done in order; this keeps the compiler to it between the
// lanes' writes and other lanes' reads.
DEC_INL void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---- One row, straight from memory.  NW wavefronts share 16 channels; a wavefront's
// next k block is asked for before this one is used.  4096 x 4096 w4g128 3.9 us a launch in
// a graph (one wavefront for all k blocks: 10.7); 20480 x 3584 9.9 us, 3.9 TB/s
// (14.4 us with weights that no cache holds).
template <int KD, int ACT, int NW>
__global__ void __launch_bounds__(64 * NW) decode_one_kernel(DecodeArgs p) {
  __shared__ Acc<KD> red[NW * 64];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), qd = lane >> 4;
  const int kbs = p.k / 128;
  const uint8_t* wb = p.packed + (int64_t)blockIdx.x * kbs * block_bytes(KD);
  const uint8_t* ar = reinterpret_cast<const uint8_t*>(p.a) + 16 * qd;
  Acc<KD> tot[1] = {Acc<KD>{0, 0, 0, 0}};
  struct Step { Wgt<KD> w; Rows<KD, 1> a; } cur, nxt;
  auto load = [&](Step& s, int kb) {
    s.w.load(wb + (int64_t)kb * block_bytes(KD), lane);
#pragma unroll
    for (int j = 0; j < kPieces<KD>; ++j)
      s.a[0][j] = *reinterpret_cast<const u32x4*>(ar + (int64_t)kb * (64 * kPieces<KD>) + 64 * j);
  };
  if (w < kbs) load(cur, w);
  for (int kb = w; kb < kbs; kb += NW) {
    if (kb + NW < kbs) load(nxt, kb + NW);
    f32x4 rs[1];
    row_sums<KD, ACT, 1>(cur.a, rs);
    use_block<KD, ACT, 1>(cur.w, cur.a, rs, tot);
    cur = nxt;
  }
  red[w * 64 + lane] = tot[0];
  __syncthreads();
  write_out<KD, 1, NW>(p, red, blockIdx.x, tid, 64 * NW);
}

// ---- Rows through a wavefront's own LDS.  A fragment straight from memory takes 64
// addresses a load, lane by lane, where the cache serves four lanes at a time that read 64
// bytes side by side (64 rows of fp8, 4096 x 14336: 28.9 us, bound by that).  So four lanes
// bring a row's 64 bytes, and the wavefront turns them into a fragment through 1 KB of LDS
// of its own, without a barrier: 16.0 us, 3.7 TB/s.  Its next k block, weights and rows, is on
// its way meanwhile.  NB blocks of channels use the fragments.
template <int KD, int ACT, int MF, int NW, int NB>
__global__ void __launch_bounds__(64 * NW) decode_wave_kernel(DecodeArgs p) {
  constexpr int P = kPieces<KD>, ES = KD == K_W4G ? 2 : 1;
  constexpr int kStage = NW * MF * P * 64, kRed = NW * MF * 64;
  __shared__ u32x4 buf[kStage > kRed ? kStage : kRed];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15, qd = lane >> 4;
  const int kbs = p.k / 128, nbs = p.n / 16, nb0 = (int)blockIdx.x * NB;
  const uint8_t* wb[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) wb[b] = p.packed + (int64_t)min(nb0 + b, nbs - 1) * kbs * block_bytes(KD);
  // lane 4 i + q brings piece 4 j + q of row i of a fragment, which lies at 16 q + (i ^ 2 q): the
  // lanes that a 16-byte LDS operation serves together, lanes 0-3 and 20-23, 4-7 and 16-19
  // and so on, then meet 8 different sets of banks both in the writes and in the reads
  // (with (i + 4 q) % 16 a third of the kernel's time were conflicts)
  const int mi = lane >> 2, mq = lane & 3;
  const uint8_t* src[MF];
#pragma unroll
  for (int f = 0; f < MF; ++f)
    src[f] = reinterpret_cast<const uint8_t*>(p.a) + (int64_t)min(16 * f + mi, p.m - 1) * p.lda * ES + 16 * mq;
  u32x4* put = buf + w * (MF * P * 64) + 16 * mq + (mi ^ (2 * mq));
  const u32x4* get = buf + w * (MF * P * 64) + 16 * qd + (li ^ (2 * qd));
  u32x4 st[MF][P];
  Wgt<KD> cur[NB], nxt[NB];
  auto load = [&](Wgt<KD> (&g)[NB], int kb) {
#pragma unroll
    for (int b = 0; b < NB; ++b) g[b].load(wb[b] + (int64_t)kb * block_bytes(KD), lane);
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
      for (int j = 0; j < P; ++j) st[f][j] = *reinterpret_cast<const u32x4*>(src[f] + (int64_t)kb * (64 * P) + 64 * j);
  };
  Acc<KD> tot[NB][MF];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int f = 0; f < MF; ++f) tot[b][f] = Acc<KD>{0, 0, 0, 0};
  if (w < kbs) load(cur, w);
  for (int kb = w; kb < kbs; kb += NW) {
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
      for (int j = 0; j < P; ++j) put[(f * P + j) * 64] = st[f][j];
    wave_order();
    if (kb + NW < kbs) load(nxt, kb + NW);
    Rows<KD, MF> a;
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
      for (int j = 0; j < P; ++j) a[f][j] = get[(f * P + j) * 64];
    wave_order();
    f32x4 rs[MF];
    row_sums<KD, ACT, MF>(a, rs);
#pragma unroll
    for (int b = 0; b < NB; ++b) use_block<KD, ACT, MF>(cur[b], a, rs, tot[b]);
#pragma unroll
    for (int b = 0; b < NB; ++b) cur[b] = nxt[b];
  }
  Acc<KD>* red = reinterpret_cast<Acc<KD>*>(buf);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    __syncthreads();
#pragma unroll
    for (int f = 0; f < MF; ++f) red[(w * MF + f) * 64 + lane] = tot[b][f];
    __syncthreads();
    if (nb0 + b < nbs) write_out<KD, MF, NW>(p, red, nb0 + b, tid, 64 * NW);
  }
}
template <int KD, int ACT, int MF, int NW, int NB> hipError_t go_wave(const DecodeArgs& p, hipStream_t s) {
  hipLaunchKernelGGL((decode_wave_kernel<KD, ACT, MF, NW, NB>), dim3((p.n / 16 + NB - 1) / NB), dim3(64 * NW), 0, s, p);
  return hipGetLastError();
}

// ---- Rows through LDS that the workgroup shares, for the widest linears: 8 wavefronts
// bring KC k blocks of all rows into LDS, and WN groups of wavefronts take NB blocks of
// 16 channels each, the WK wavefronts of a group one k block each.  Piece q of
// row r lies at q ^ (r % 16), so that both the writes along a row and the fragment reads
// across rows are free of bank conflicts.  The next k blocks' rows and weights are on
// their way in registers meanwhile, and workgroups start at different ones (all at the same
// lines, they waited for the same channels of the L2).  The rows come to a CU once for 64
// or 96 channels; the barriers, a chunk at a time, cost more where channels are few.
template <int KD, int ACT, int MF, int WN, int NB>
__global__ void __launch_bounds__(512) decode_rows_kernel(DecodeArgs p) {
  constexpr int NW = 8, WK = NW / WN, KC = WK, PP = 4 * kPieces<KD>, RP = KC * PP, RS = 512 / RP, NPT = 16 * MF / RS;
  constexpr int ES = KD == K_W4G ? 2 : 1;
  constexpr int kStage = 16 * MF * RP, kRed = NW * MF * 64;
  static_assert(512 % RP == 0 && NPT >= 1 && (16 * MF) % RS == 0, "staging covers the rows");
  __shared__ u32x4 buf[kStage > kRed ? kStage : kRed];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15, qd = lane >> 4;
  const int wn = w / WK, wk = w % WK;
  const int kbs = p.k / 128, nbs = p.n / 16, chunks = (kbs + KC - 1) / KC;
  const int nb0 = (int)blockIdx.x * (WN * NB) + wn * NB;
  const uint8_t* wb[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) wb[b] = p.packed + (int64_t)min(nb0 + b, nbs - 1) * kbs * block_bytes(KD);
  const int sq = tid % RP, sr = tid / RP;
  const uint8_t* src = reinterpret_cast<const uint8_t*>(p.a) + sr * p.lda * ES + 16 * sq;
  u32x4 st[NPT];
  auto stage_load = [&](int c) {
    const bool in = c * RP + sq < kbs * PP;
#pragma unroll
    for (int i = 0; i < NPT; ++i)
      if (in && sr + RS * i < p.m) st[i] = *reinterpret_cast<const u32x4*>(src + (int64_t)(RS * i) * p.lda * ES + (int64_t)c * (16 * RP));
  };
  Wgt<KD> cur[NB], nxt[NB];
  auto wgt_load = [&](Wgt<KD> (&g)[NB], int c) {
    const int kb = min(c * KC + wk, kbs - 1);
#pragma unroll
    for (int b = 0; b < NB; ++b) g[b].load(wb[b] + (int64_t)kb * block_bytes(KD), lane);
  };
  Acc<KD> tot[NB][MF];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int f = 0; f < MF; ++f) tot[b][f] = Acc<KD>{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < NPT; ++i) st[i] = u32x4{0u, 0u, 0u, 0u};
  int c = (int)(blockIdx.x >> 3) % chunks;
  wgt_load(cur, c);
  stage_load(c);
  for (int left = chunks; left > 0; --left) {
    const int next = c + 1 < chunks ? c + 1 : 0;
    __syncthreads();  // the last chunk's fragments are read
#pragma unroll
    for (int i = 0; i < NPT; ++i) {
      const int r = sr + RS * i;
      buf[r * RP + (sq ^ (r & 15))] = st[i];
    }
    __syncthreads();
    if (left > 1) {
      wgt_load(nxt, next);
      stage_load(next);
    }
    if (c * KC + wk < kbs) {
      Rows<KD, MF> a;
#pragma unroll
      for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int j = 0; j < kPieces<KD>; ++j) a[f][j] = buf[(16 * f + li) * RP + ((wk * PP + 4 * j + qd) ^ li)];
      f32x4 rs[MF];
      row_sums<KD, ACT, MF>(a, rs);
#pragma unroll
      for (int b = 0; b < NB; ++b) use_block<KD, ACT, MF>(cur[b], a, rs, tot[b]);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) cur[b] = nxt[b];
    c = next;
  }
  Acc<KD>* red = reinterpret_cast<Acc<KD>*>(buf);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    __syncthreads();
#pragma unroll
    for (int f = 0; f < MF; ++f) red[(w * MF + f) * 64 + lane] = tot[b][f];
    __syncthreads();
    if (nb0 + b < nbs) write_out<KD, MF, WK>(p, red + wn * WK * MF * 64, nb0 + b, tid - wn * WK * 64, WK * 64);
  }
}

template <int KD, int ACT, int NW> hipError_t go_one(const DecodeArgs& p, hipStream_t s) {
  hipLaunchKernelGGL((decode_one_kernel<KD, ACT, NW>), dim3(p.n / 16), dim3(64 * NW), 0, s, p);
  return hipGetLastError();
}
template <int KD, int ACT, int MF, int NB> hipError_t go_rows(const DecodeArgs& p, hipStream_t s) {
  hipLaunchKernelGGL((decode_rows_kernel<KD, ACT, MF, 2, NB>), dim3((p.n / 16 + 2 * NB - 1) / (2 * NB)), dim3(512), 0, s, p);
  return hipGetLastError();
}

// Rows of a call in MF fragments, nb blocks of 16 channels.
template <int KD, int ACT, int MF> hipError_t launch_rows(const DecodeArgs& p, hipStream_t s) {
  const int nb = p.n / 16;
  // 49 and more 16-bit rows, wide linears: a workgroup's rows shared by 4 or 6 blocks (64 x 20480 x
  // 3584 23.0 us, 26.0 by wavefronts; 64 x 16384 x 2048 12.6, 15.6; 64 x 12288 x 4096 19.7, 16.4)
  if constexpr (KD == K_W4G && MF == 4)
    if (nb > 768) return (nb + 1535) / 1536 * 4 <= (nb + 1023) / 1024 * 3 ? go_rows<KD, ACT, MF, 3>(p, s) : go_rows<KD, ACT, MF, 2>(p, s);
  // Blocks of a workgroup: what the busiest CU does, its workgroups times the rows (about the
  // weights of one block) and their blocks.  16 x 8192 x 4096 w4g128 with 1, 2, 3 blocks 6.7, 6.2,
  // 7.5; 32 x 12288 x 4096 14.0, 13.9, 10.7; 64 x 4096 x 14336 fp8 15.9, 18.8, 22.3.
  int NB = 1, best = 0;
  for (int b = 1; b <= 3; ++b) {
    const int cost = ((nb + b - 1) / b + 255) / 256 * (1 + b);
    if (b == 1 || cost < best) {
      NB = b;
      best = cost;
    }
  }
  // 8 wavefronts where a CU has one workgroup, else 4 (64 x 20480 x 3584 int8, 3 blocks: 21.2 and
  // 17.7; 64 x 8192 x 4096, 2 blocks: 9.8 and 10.1)
  const bool one = (nb + NB - 1) / NB <= 256;
  if (NB == 1) return go_wave<KD, ACT, MF, 8, 1>(p, s);
  if (NB == 2) return one ? go_wave<KD, ACT, MF, 8, 2>(p, s) : go_wave<KD, ACT, MF, 4, 2>(p, s);
  if constexpr (KD != K_W4G || MF < 4)  // (64 16-bit rows for 3 blocks do not fit the registers of 8)
    if (one) return go_wave<KD, ACT, MF, 8, 3>(p, s);
  return go_wave<KD, ACT, MF, 4, 3>(p, s);
}
template <int KD, int ACT> hipError_t launch(const DecodeArgs& p, hipStream_t s) {
  // One row straight from memory, with 16 wavefronts where few workgroups have much to read.
  // w4g128 that is wide and deep goes through LDS with two or three channel blocks to a
  // workgroup: a row's pieces and their sums serve all of them.  us with weights from the
  // caches / from memory, with 8 wavefronts, with 16, through LDS:
  //   bf16 w4g128  4096 x 4096 4.0 / 5.8, 4.0 / 5.0, 4.0 / 5.2;  4096 x 14336 10.0 / 14.2, 8.7 / 12.8,
  //     8.5 / 12.9;  16384 x 1024 3.8 / 5.2, 5.1 / 6.9, 4.0 / 4.8;  20480 x 256 3.2 / 4.0, 4.6 / 6.6, 3.4 / 4.1;
  //     14336 x 4096 9.3 / 12.3, 10.8 / 13.6, 8.4 / 11.0;  8192 x 14336 15.6 / 21.6, -, 13.2 / 16.5
  //   fp16 w4g128  20480 x 2048 5.9 / 8.7, -, 7.1 / 8.6;  20480 x 3584 9.5 / 13.8, -, 10.8 / 12.4;  24576 x 4096
  //     12.1 / 17.6, -, 12.2 / 14.1;  8192 x 14336 14.6 / 21.1, -, 13.2 / 16.5
  //   w8a8         2048 x 14336 6.1 / 12.0, 5.7 / 10.2, 6.0 / 11.5;  20480 x 3584 12.1 / 15.3, 12.4 / 15.7, 12.9 / 16.6
  if (p.m == 1 && !(KD == K_W4G && p.n >= 8192 && p.k >= 4096))
    return p.n <= 4096 && p.k >= 4096 ? go_one<KD, ACT, 16>(p, s) : go_one<KD, ACT, 8>(p, s);
  if (p.m <= 16) return launch_rows<KD, ACT, 1>(p, s);
  if (p.m <= 32) return launch_rows<KD, ACT, 2>(p, s);
  if (p.m <= 48) return launch_rows<KD, ACT, 3>(p, s);
  return launch_rows<KD, ACT, 4>(p, s);
}

}  // namespace

bool decode_kind(int kind) { return kind == K_W4G || kind == K_W8A8 || kind == K_F8A8; }

hipError_t launch_linear_decode(const DecodeArgs& p, int kind, hipStream_t s) {
  switch (kind) {
    case K_W4G: return p.act == MXMOE_BF16 ? launch<K_W4G, MXMOE_BF16>(p, s) : launch<K_W4G, MXMOE_F16>(p, s);
    case K_W8A8: return launch<K_W8A8, MXMOE_BF16>(p, s);  // (codes: the dtype is the output's only)
    default: return launch<K_F8A8, MXMOE_BF16>(p, s);
  }
}

}  // namespace mxmoe
