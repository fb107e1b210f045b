// Attention of a few query tokens a sequence over the paged cache.
//
//   out = softmax(x) v,  x = scale q k, capped by cap tanh(x / cap) where a cap is given
//
// Scores are formed as K Q^T (tokens by query rows), so that a lane holds one query row and
// four tokens of each 16: maxima, sums and weights need no other lane, and the weights of
// 32 tokens are, as they lie, the operand of V^T P^T (elements by query rows).  One
// pass over the tokens: the weights are powers of 2 against a reference of the row; a
// weight past 2^15 moves it, and the sums so far are scaled.
//
// 8-bit codes become fp16 in registers (both formats are exact there) and the products are
// fp16: queries in bf16 get a power of 2 a row that brings the largest to 2^14 (bf16 has
// fewer bits than fp16; what falls under fp16's least is under 2^-38 of the largest).  A
// key's scale multiplies its score.  A value's scale multiplies its weight, and the reference
// is that of the products, so that they keep their bits whatever the scales are; scales
// under 2^-80 move it no further than one of 2^-80 would.  The sum of the weights is of fp32 values, before any rounding.
//
// A weight enters its product as two, the rounded one and what it lacks (bf16 16 bits, fp16 22), or,
// where codes meet bf16 outputs, as one of fp16: its 11 bits lie under the output's 8 (errors grow by less
// than 1%).  With one part 16-bit bf16 rows were off by 1.4 times the output's own rounding, fp16 outputs by 1.3 times.
// The second product costs 0.5 to 1% where memory bounds a call, 5 to 11% where it does not.
//
// Tokens past a row's last are left out by selection, whatever they hold: their scores
// become -inf, their values zeros.  Where rows of a tile see different tokens and a value
// there is not finite, rows are added one by one, each with the values that it sees.
#include <algorithm>

#include "kvcache.h"
#include "lanes.h"

namespace mxmoe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Workgroups of 4 wavefronts that a CU holds (registers)
constexpr int cu_holds(bool wide, int mf_dim) { return wide && mf_dim >= 256 ? 1 : 2; }
enum CacheKind { C_BF16, C_F16, C_I8, C_F8, C_I8_F16, C_F8_F16 };  // (codes by the activations' type, bf16 first)
constexpr bool is_i8(int kind) { return kind == C_I8 || kind == C_I8_F16; }
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kBase = 8.f;              // weights are 2^8 at the reference ..
constexpr uint32_t kMostF16 = 0x7800u, kMostBf16 = 0x4700u;  // .. and move it past 2^15 (fp16 ends at 2^16)
constexpr float kLeastScale = 0x1p-80f;
constexpr float kMostSum = 0x1p96f;  // of a lane's weights of a block, without their values' scales, likewise
constexpr float kNoReference = -0x1p126f;  // of a row that has seen nothing: below any, and against it every weight is inf

template <int KIND> LANES_INL f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (KIND == C_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// 4 codes -> 4 fp16 values
template <int KIND> LANES_INL u32x2 widen(uint32_t w) {
  if constexpr (is_i8(KIND)) {  // 1024 + 128 + q, less 1152
    w ^= 0x80808080u;
    const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
    const f16x2 a = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) - off;
    const f16x2 b = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) - off;
    return u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
  } else {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
    return u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
  }
}
template <int KIND> LANES_INL u32x4 widen8(uint32_t lo, uint32_t hi) {
  const u32x2 a = widen<KIND>(lo), b = widen<KIND>(hi);
  return u32x4{a[0], a[1], b[0], b[1]};
}

// tanh y = 1 - 2 / (1 + e^(2 y)) for y > 0; below 1/4, where the difference takes the value's own
// digits (scores far below a cap), four terms more of the series.
LANES_INL float tanh_of(float y) {
  const float z = y * y;
  const float big = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(fabsf(y) * (2.f * kLog2e)));
  float s = __builtin_fmaf(z, 62.f / 2835.f, -17.f / 315.f);
  s = __builtin_fmaf(z, s, 2.f / 15.f);
  s = __builtin_fmaf(z, s, -1.f / 3.f);
  return fabsf(y) < 0.25f ? __builtin_fmaf(y * z, s, y) : __builtin_copysignf(big, y);
}

LANES_INL float quarters_max(float v) {  // over the four lanes of a query row
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
LANES_INL float quarters_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

LANES_INL float sum8(const float (&p)[8]) { return ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])); }

// Keys (or values) of 32 tokens as a lane holds them, and their scales.
template <int KIND, int D> struct Frag {
  static constexpr int ES = KIND <= C_F16 ? 2 : 1, N = D * ES / 32;
  u32x4 w[N];
  f32x4 s[ES == 1 ? 2 : 1];
  LANES_INL void load(const uint8_t* base, const float* scales, int64_t token, int lane) {
    const uint8_t* p = base + token * (D * ES) + lane * 16;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = *reinterpret_cast<const u32x4*>(p + 1024 * i);
    if constexpr (ES == 1) {
#pragma unroll
      for (int i = 0; i < 2; ++i) s[i] = *reinterpret_cast<const f32x4*>(scales + token + 4 * (lane >> 4) + 16 * i);
    }
  }
  LANES_INL u32x4 key(int tile, int step) const {  // 16 tokens, 32 elements
    if constexpr (ES == 2) return w[tile * (D / 32) + step];
    const u32x4 p = w[tile * (D / 64) + (step >> 1)];
    return step & 1 ? widen8<KIND>(p[2], p[3]) : widen8<KIND>(p[0], p[1]);
  }
  LANES_INL u32x4 value(int tile) const {  // 16 elements, 32 tokens
    if constexpr (ES == 2) return w[tile];
    const u32x4 p = w[tile >> 1];
    return tile & 1 ? widen8<KIND>(p[2], p[3]) : widen8<KIND>(p[0], p[1]);
  }
};

// What a block's tokens are to the rows of a wavefront: `some` 1 if a row does not see
// all 32 or the page is bad (NaN for whoever sees it); most, least: how many the rows see that
// see most and least of them.
struct Sight { int some, bad, most, least; };

// MF times 16 query rows of a wavefront: row 16 f + lane % 16.
template <int KIND, int D, int MF> struct Rows16 {
  static constexpr int ES = KIND <= C_F16 ? 2 : 1;
  static constexpr bool BOTH = KIND != C_I8 && KIND != C_F8;  // both parts of a weight
  u32x4 q[MF][D / 32];
  f32x4 acc[MF][D / 16];   // elements 16 i + 4 (lane / 16) + (0..3)
  float ref[MF], sum[MF];  // the row's reference, the sum of its weights (this lane's tokens)
  float mul[MF];           // from a product of codes to a score: in powers of 2, or (with a cap) parts of the cap
  float w[MF][8];          // products, then weights of the block in hand
  u32x4 pw[MF];            // weights as the second product takes them
  static constexpr int P = KIND == C_BF16 ? MXMOE_BF16 : MXMOE_F16;

  LANES_INL void clear() {
#pragma unroll
    for (int f = 0; f < MF; ++f) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) acc[f][i] = f32x4{0.f, 0.f, 0.f, 0.f};
      ref[f] = kNoReference;
      sum[f] = 0.f;
    }
  }
  LANES_INL void load(const AttnArgs& a, int f, const uint16_t* row, int lane) {
    const int qd = lane >> 4;
    float m = a.scale;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const int c = ES == 2 ? 4 * s + qd : 8 * (s >> 1) + 2 * qd + (s & 1);
      q[f][s] = row ? (u32x4) * reinterpret_cast<const u32x4_any*>(row + 8 * c) : u32x4{0u, 0u, 0u, 0u};
    }
    if constexpr (KIND == C_I8 || KIND == C_F8) {
      uint32_t b = 0u;
#pragma unroll
      for (int s = 0; s < D / 32; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) b = max2(b, q[f][s][i] & 0x7fff7fffu);
      b = max2(b, (uint32_t)__shfl_xor((int)b, 16, 64));
      b = max2(b, (uint32_t)__shfl_xor((int)b, 32, 64));
      const int e = (int)(max(b & 0xffffu, b >> 16) >> 7);  // exponent of the largest
      const int up = e == 255 ? 0 : min(127, 127 + 14 - max(e, 1));
      auto turned = [&](uint32_t b) {
        const f32x2 v = unpack2<MXMOE_BF16>(b);
        return pack2<MXMOE_F16>(__builtin_ldexpf(v[0], up), __builtin_ldexpf(v[1], up));
      };
#pragma unroll
      for (int s = 0; s < D / 32; ++s) q[f][s] = u32x4{turned(q[f][s][0]), turned(q[f][s][1]), turned(q[f][s][2]), turned(q[f][s][3])};
      m = __builtin_ldexpf(m, -up);
    }
    // (finite: 0 times it is 0)
    mul[f] = fminf(fmaxf(a.softcap > 0.f ? m / a.softcap : m * kLog2e, -0x1.fffffep127f), 0x1.fffffep127f);
  }

  // products of the rows and 32 keys: 16 keys of a tile, 32 elements of a step at a time
  template <class K> LANES_INL void scores(K key) {
    f32x4 s[MF][2];
#pragma unroll
    for (int f = 0; f < MF; ++f) s[f][0] = s[f][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const u32x4 b = key(t, i);
#pragma unroll
        for (int f = 0; f < MF; ++f) s[f][t] = mfma<KIND>(b, q[f][i], s[f][t]);
      }
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
      for (int i = 0; i < 8; ++i) w[f][i] = s[f][i >> 2][i & 3];
  }

  // weights of the 32 tokens, sums and references; ks, vs: the tokens' scales, limit: how many of
  // the tokens a row sees
  LANES_INL void weigh(const AttnArgs& a, const f32x4 (&ks)[2], const f32x4 (&vs)[2], const Sight& g, const int (&limit)[MF], int lane) {
    // A score is x k m, (k m) first: x k may pass the largest value where the score does not.
    float x[MF][8], p[MF][8], m[MF], total[ES == 1 ? MF : 1];
    f32x4 k[2] = {f32x4{1.f, 1.f, 1.f, 1.f}, f32x4{1.f, 1.f, 1.f, 1.f}};
    if constexpr (ES == 1) { k[0] = ks[0]; k[1] = ks[1]; }
#pragma unroll
    for (int f = 0; f < MF; ++f) {
      m[f] = mul[f];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[f][i] = w[f][i];
    }
    if (a.softcap > 0.f) {
#pragma unroll
      for (int f = 0; f < MF; ++f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[f][i] = a.softcap * kLog2e * tanh_of(x[f][i] * (ES == 1 ? k[i >> 2][i & 3] * m[f] : m[f]));
        m[f] = 1.f;
      }
      k[0] = k[1] = f32x4{1.f, 1.f, 1.f, 1.f};
    }
    auto factor = [&](int f, int i) { return ES == 1 ? k[i >> 2][i & 3] * m[f] : m[f]; };
    auto sees = [&](int f, int i) { return 4 * (lane >> 4) + (i & 3) + 16 * (i >> 2) < limit[f]; };
    auto weights = [&](int f) {
      const float off = kBase - ref[f];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[f][i] = __builtin_fmaf(x[f][i], factor(f, i), off);
      if (g.some) {  // (after the same arithmetic: a row's result does not hang on what others see)
#pragma unroll
        for (int i = 0; i < 8; ++i) p[f][i] = sees(f, i) ? (g.bad ? __builtin_nanf("") : p[f][i]) : -__builtin_inff();
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[f][i] = __builtin_amdgcn_exp2f(p[f][i]);
        w[f][i] = ES == 1 ? p[f][i] * vs[i >> 2][i & 3] : p[f][i];
      }
      if (ES == 1 && g.some) {  // (whatever the scale of a token that is not seen)
#pragma unroll
        for (int i = 0; i < 8; ++i) w[f][i] = sees(f, i) ? w[f][i] : 0.f;
      }
      const u32x4 o = {pack2<P>(w[f][0], w[f][1]), pack2<P>(w[f][2], w[f][3]), pack2<P>(w[f][4], w[f][5]), pack2<P>(w[f][6], w[f][7])};
      pw[f] = o;
      uint32_t t = max2(max2(o[0], o[1]), max2(o[2], o[3]));
      // Weights of values that are zeros, or whose scale is small, pass no limit with their scale in
      // them: their sum is looked at too, so that the row's stays finite (2^27 times 2^96).  Past the
      // limit a weight is 2^93 or more, its score at least 5 over what a scale of 2^-80 puts the
      // reference to: it moves, and a lane's sum is 2^91 then at the most.
      if constexpr (ES == 1) {
        total[f] = sum8(p[f]);
        if (total[f] > kMostSum) t = 0xffffffffu;
      }
      return t;
    };
    // (weights are not negative: the order of their bits is theirs, and inf and NaN come last; a
    // row without a reference has inf for its first tokens)
    constexpr uint32_t kMost = KIND == C_BF16 ? kMostBf16 : kMostF16;
    uint32_t top[MF], any = 0u;
#pragma unroll
    for (int f = 0; f < MF; ++f) any = max2(any, top[f] = weights(f));
    if (__ballot(max(any & 0xffffu, any >> 16) > kMost)) {
#pragma unroll
      for (int f = 0; f < MF; ++f) {
        // (a row moves for its own weights' sake alone: what it comes to does not hang on the others)
        uint32_t t = max(top[f] & 0xffffu, top[f] >> 16);
        t = max(t, (uint32_t)__shfl_xor((int)t, 16, 64));
        t = max(t, (uint32_t)__shfl_xor((int)t, 32, 64));
        float r = kNoReference;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!g.some || sees(f, i)) r = fmaxf(r, x[f][i] * factor(f, i) + (ES == 1 ? __builtin_amdgcn_logf(fmaxf(vs[i >> 2][i & 3], kLeastScale)) : 0.f));
        r = quarters_max(r);
        const float next = t > kMost ? fmaxf(ref[f], r) : ref[f], d = t > kMost ? __builtin_amdgcn_exp2f(ref[f] - next) : 1.f;
        ref[f] = next;
        sum[f] *= d;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) acc[f][i] *= d;
        weights(f);
      }
    }
#pragma unroll
    for (int f = 0; f < MF; ++f) sum[f] += ES == 1 ? total[ES == 1 ? f : 0] : sum8(p[f]);
  }

  // `what` in the 16-bit halves of the lane's tokens that come before a limit
  static LANES_INL u32x4 before(int lim, uint32_t what, int lane) {
    auto half = [&](int i) {
      const int t = 4 * (lane >> 4) + 2 * (i & 1) + 16 * (i >> 1);
      return (t < lim ? what : 0u) | (t + 1 < lim ? what << 16 : 0u);
    };
    const u32x4 m = {half(0), half(1), half(2), half(3)};
    return m;
  }
  static constexpr uint32_t kInf = KIND == C_BF16 ? 0x7f80u : 0x7c00u, kOne = KIND == C_BF16 ? 0x3f80u : 0x3c00u;
  // ones in the halves that are not finite.  (Fragments are changed whole: written element by element, results
  // were wrong for bf16, dim 64, 32 rows, by hipcc of ROCm 7.2, for a reason that was not found.)
  static LANES_INL uint32_t odd_half(uint32_t w) {
    return ((w & kInf) == kInf ? 0xffffu : 0u) | ((w & (kInf << 16)) == kInf << 16 ? 0xffff0000u : 0u);
  }
  static LANES_INL u32x4 odd_halves(u32x4 v) { return u32x4{odd_half(v[0]), odd_half(v[1]), odd_half(v[2]), odd_half(v[3])}; }

  // ones where a value of a 16-byte piece is not finite
  static LANES_INL uint32_t strange(uint32_t w) {
    if constexpr (ES == 2) return odd_half(w);
    const uint32_t top = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;  // bytes 0x7f, 0xff
    return (top >> 7) * 0xffu;
  }
  // ones for the values of a 16-byte piece whose tokens come before a limit
  static LANES_INL u32x4 kept(int lim, int lane) {
    if constexpr (ES == 2) return before(lim, 0xffffu, lane);
    auto four = [&](int t) {
      return (t < lim ? 0xffu : 0u) | (t + 1 < lim ? 0xff00u : 0u) | (t + 2 < lim ? 0xff0000u : 0u) | (t + 3 < lim ? 0xff000000u : 0u);
    };
    const uint32_t lo = four(4 * (lane >> 4)), hi = four(4 * (lane >> 4) + 16);
    return u32x4{lo, hi, lo, hi};
  }

  // Values for rows that do not see all of them.  Past the last token that any row sees they are
  // zeros.  One that is not finite must not reach the rows that do not see it (0 * inf): it
  // becomes zero, and rows become NaN where a product of ones counts such values among
  // the tokens they see.
  LANES_INL void sift(Frag<KIND, D>& v, const Sight& g, const int (&limit)[MF], int lane) {
    if constexpr (is_i8(KIND)) return;  // (every code is finite, the weights of what is not seen are 0)
    const u32x4 any = kept(g.most, lane);
    uint32_t odd = 0u;
#pragma unroll
    for (int i = 0; i < Frag<KIND, D>::N; ++i) {
      v.w[i] &= any;
#pragma unroll
      for (int j = 0; j < 4; ++j) odd |= strange(v.w[i][j]);
    }
    if (__ballot(odd != 0)) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) count(v.value(i), i, limit, lane);
#pragma unroll
      for (int i = 0; i < Frag<KIND, D>::N; ++i) {
        const u32x4 o = v.w[i];
        v.w[i] = o & ~u32x4{strange(o[0]), strange(o[1]), strange(o[2]), strange(o[3])};
      }
    }
  }
  // NaN for the rows that see a value of tile i that is not finite
  LANES_INL void count(u32x4 b, int i, const int (&limit)[MF], int lane) {
    __builtin_amdgcn_sched_barrier(0);  // (rare: one tile after another, in few registers)
    b = odd_halves(b) & (kOne | kOne << 16);
    constexpr float nan = __builtin_nanf("");
#pragma unroll
    for (int f = 0; f < MF; ++f) {
      const f32x4 n = mfma<KIND>(b, before(limit[f], kOne, lane), f32x4{0.f, 0.f, 0.f, 0.f}), o = acc[f][i];
      acc[f][i] = f32x4{n[0] > 0.f ? nan : o[0], n[1] > 0.f ? nan : o[1], n[2] > 0.f ? nan : o[2], n[3] > 0.f ? nan : o[3]};
    }
  }

  // weights times values, 16 elements of a tile at a time
  template <class V> LANES_INL void add(V value) {
    u32x4 rest[BOTH ? MF : 1];  // what the rounded weights lack
    if constexpr (BOTH) {
#pragma unroll
      for (int f = 0; f < MF; ++f) {
        auto lack = [&](int i) {
          const f32x2 r = unpack2<P>(pw[f][i]);
          return pack2<P>(w[f][2 * i] - r[0], w[f][2 * i + 1] - r[1]);
        };
        rest[f] = u32x4{lack(0), lack(1), lack(2), lack(3)};
      }
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const u32x4 b = value(i);
#pragma unroll
      for (int f = 0; f < MF; ++f) {
        acc[f][i] = mfma<KIND>(b, pw[f], acc[f][i]);
        if constexpr (BOTH) acc[f][i] = mfma<KIND>(b, rest[f], acc[f][i]);
      }
    }
  }

  // a block whose keys and values the lane holds; between: what is done when the keys are used
  template <class F>
  LANES_INL void block(const AttnArgs& a, Frag<KIND, D>& k, Frag<KIND, D>& v, const Sight& g, const int (&limit)[MF], int lane, F between) {
    scores([&](int t, int i) { return k.key(t, i); });
    f32x4 ks[2];
    if constexpr (ES == 1) { ks[0] = k.s[0]; ks[1] = k.s[1]; }
    between();
    f32x4 vs[2];
    if constexpr (ES == 1) { vs[0] = v.s[0]; vs[1] = v.s[1]; }
    weigh(a, ks, vs, g, limit, lane);
    if (g.some) sift(v, g, limit, lane);
    add([&](int i) { return v.value(i); });
  }
};

// How far a partial sum's factor is from the joint reference's
LANES_INL float join_factor(float ref, float top) { return __builtin_amdgcn_exp2f(ref - top); }

LANES_INL void store4(void* out, int64_t at, f32x4 o, int act) {
  typedef u32x2 u32x2_half __attribute__((aligned(2)));
  u32x2 w;
#pragma unroll
  for (int e = 0; e < 2; ++e)
    w[e] = act == MXMOE_BF16 ? pack2<MXMOE_BF16>(o[2 * e], o[2 * e + 1]) : pack2<MXMOE_F16>(o[2 * e], o[2 * e + 1]);
  *reinterpret_cast<u32x2_half*>(reinterpret_cast<uint16_t*>(out) + at) = w;
}

// Page ids and lengths: nothing writes them while a kernel runs, so that uniform ones come by
// scalar loads, whose wait does not wait for the keys and values that are on their way
// (as vector loads they did, once a block: 32 sequences up to 4000 tokens, 16 kv heads of 128 in bf16, 130 us against 123).
typedef const __attribute__((address_space(4))) int32_t* Fixed;
LANES_INL Fixed fixed(const int32_t* p) { return (Fixed)(uintptr_t)p; }
LANES_INL int length_of(const AttnArgs& a, int b) { return max(0, fixed(a.lengths)[b]); }

// Blocks of 32 tokens of a sequence's own pages (0 for a length past its table: its
// queries are NaN, which the joining launch writes).
LANES_INL int own_blocks(const AttnArgs& a, int b) {
  const int own = length_of(a, b) - a.prefix_len;
  return own <= 0 || own > a.width << a.page_log2 ? 0 : (own + 31) >> 5;
}

// 16 rows of a fragment that the wavefronts of a workgroup have summed, each over its blocks, joined
// through LDS: red [W][live][D + 4] (rows 4 banks apart) and a flag for each wavefront that has
// seen a block.  Every thread of the workgroup calls it; done(row, element, sums, weight,
// reference) gets 4 elements at a time.
template <int KIND, int D, int MF, int W, class F>
LANES_INL void meet(const Rows16<KIND, D, MF>& x, int f, int live, bool has, float* red, int* flag, int w, int lane, F done) {
  constexpr int RS = D + 4;
  const int n = lane & 15, qd = lane >> 4;
  const float s = quarters_sum(x.sum[f]);
  __syncthreads();  // what was there is read
  if (lane == 0) flag[w] = has;
  if (has && n < live) {
    float* row = red + (w * live + n) * RS;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) *reinterpret_cast<f32x4*>(row + 16 * e + 4 * qd) = x.acc[f][e];
    if (qd == 0) {
      row[D] = x.ref[f];
      row[D + 1] = s;
    }
  }
  __syncthreads();
  for (int o = w * 64 + lane; o < live * (D / 4); o += 64 * W) {
    const int r = o / (D / 4), d = 4 * (o % (D / 4));
    float top = kNoReference, l = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (flag[j]) top = fmaxf(top, red[(j * live + r) * RS + D]);
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (flag[j]) {
        const float* row = red + (j * live + r) * RS;
        const float c = join_factor(row[D], top);
        v += c * *reinterpret_cast<const f32x4*>(row + d);
        l += c * row[D + 1];
      }
    done(r, d, v, l, top);
  }
}

// What an item costs a workgroup beside its blocks (its queries, the wavefronts' meeting), in blocks.
// us with 4, 8, 16: 64 sequences up to 8192 tokens fp8 110.0, 108.5, 109.5, 16 up to 4000 with 40
// rows a kv head 38.3, 32.6, 30.5, one of 2000 12.7, 12.1, 13.8 (without: 123, 68, 13.0)
constexpr uint32_t kItemCost = 8;
LANES_INL uint32_t item_cost(int blocks) { return blocks ? blocks + kItemCost : 0u; }

// Sequences' own pages.  The costs of all items (sequence, row block, kv head), kItemCost and a unit
// for each block, form one list, which the workgroups share evenly: each takes `per` units in a
// row, across items as they come, its wavefronts every fourth block.  An item within a share is finished there; pieces of
// others go to the workspace: slot 2 g of workgroup g for a piece that continues an item,
// 2 g + 1 for one that begins one.  A wavefront asks for its next block's keys when this one's
// have made their scores, for its values when this one's are added, in the same registers, also
// into the next item, so that they are on their way while the wavefronts meet.
// Bound by memory: 64 sequences up to 8192 fp8 tokens of 8 heads of 128, 555 MB, 108 us with the join, 5.1 TB/s
// (a copy reaches 5.15, reading alone 6.0); 2 of 131072 int8 tokens in fp16 54 us, and 6 for the join of 64 pieces a row.
template <int KIND, int D, int MF>
__global__ void __launch_bounds__(256, cu_holds(KIND <= C_F16, MF * D)) attention_kernel(AttnArgs a) {
  constexpr int RS = D + 4;
  extern __shared__ float red[];
  __shared__ int flag[4];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15;
  const int group = a.q_heads / a.kv_heads, rows = a.n_q * group, piece_rows = min(rows, 16 * MF);
  const int per_seq = a.kv_heads * a.row_blocks;  // items of a sequence
  // this workgroup's share: all blocks, then the sequence in which it begins
  uint32_t total = 0;  // (fewer than 2^31: the host sees to it)
  for (int b = lane; b < a.batch; b += 64) total += item_cost(own_blocks(a, b));
#pragma unroll
  for (int d = 1; d < 64; d *= 2) total += __shfl_xor(total, d, 64);
  total = __builtin_amdgcn_readfirstlane(total * per_seq);
  const uint32_t per = max(4u + kItemCost, (total + gridDim.x - 1) / gridDim.x);
  const uint32_t at0 = min(total, per * blockIdx.x);
  int left = (int)min(total - at0, per);  // units of the share
  if (left <= 0 && blockIdx.x) return;
  uint32_t begin = 0;  // of the sequence, in the list
  int seq = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = b0 + lane;
    const uint32_t mine = (b < a.batch ? item_cost(own_blocks(a, b)) : 0u) * per_seq;
    uint32_t upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t o = __shfl_up(upto, d, 64);
      upto += lane >= d ? o : 0;
    }
    if (blockIdx.x == 0) {  // (the first workgroup writes all starts, others stop at their sequence)
      if (w == 0 && b < a.batch) a.starts[b] = begin + upto - mine;
    } else {
      const uint64_t past = __ballot(begin + upto > at0);
      if (past) {
        const int l = __builtin_ctzll(past);
        seq = b0 + l;
        begin += __shfl(upto - mine, l, 64);
        break;
      }
    }
    begin += __shfl(upto, 63, 64);
  }
  if (blockIdx.x == 0) {
    begin = 0;
    while (seq < a.batch && own_blocks(a, seq) == 0) ++seq;
    if (tid == 0) {
      a.starts[a.batch] = total;
      a.starts[a.batch + 1] = per;
    }
    if (left <= 0) return;
  }
  // item: of the sequence; i: a block of the item's
  struct Place { int seq, item, i, blocks, h; };
  auto next_item = [&](Place& p) {
    if (++p.item == per_seq) {
      p.item = 0;
      do ++p.seq;
      while ((p.blocks = own_blocks(a, p.seq)) == 0);
    }
    p.h = p.item % a.kv_heads;
  };
  Place s;  // the item in hand, i its first block in this share
  s.seq = __builtin_amdgcn_readfirstlane(seq);
  s.blocks = own_blocks(a, s.seq);
  {
    const uint32_t in = __builtin_amdgcn_readfirstlane(at0 - begin), cost = item_cost(s.blocks);
    s.item = in / cost;
    s.i = (int)(in - s.item * cost) - (int)kItemCost;
    s.h = s.item % a.kv_heads;
  }
  // (a share may end before an item's first block, or begin there: s.i < 0 units are its cost)
  auto blocks_of = [&](const Place& p, int units) { return min(p.blocks, p.i + units); };  // end of the share's
  auto page_of = [&](const Place& p) { return fixed(a.table)[(int64_t)p.seq * a.width + ((32 * p.i) >> a.page_log2)]; };
  auto token_of = [&](const Place& p, int id) {
    const int64_t rec = (int64_t)((unsigned)id < (unsigned)a.n_pages ? id : 0) * a.kv_heads + p.h;
    return (rec << a.page_log2) + ((32 * p.i) & ((1 << a.page_log2) - 1));
  };
  Rows16<KIND, D, MF> x;
  Frag<KIND, D> k, v;
  // c: the wavefront's next block, whose keys and values are on their way; ahead: units of the
  // share from c's item's place on (s.i as that item begins in the share)
  Place c = s;
  int ahead = left, id = 0, turn = w;  // turn: blocks to let pass
  bool mine = true;
  auto seek = [&]() {  // to the block `turn` further on, if the share has it
    while (true) {
      const int from = max(c.i, 0), end = blocks_of(c, ahead);
      if (from + turn < end) {
        ahead -= from + turn - c.i;
        c.i = from + turn;
        turn = 0;
        return;
      }
      turn -= max(end - from, 0);
      ahead -= c.blocks - c.i;
      if (ahead <= (int)kItemCost) {
        mine = false;
        return;
      }
      next_item(c);
      c.i = -(int)kItemCost;
    }
  };
  seek();
  if (mine) {
    id = page_of(c);
    const int64_t t = token_of(c, id);
    k.load(a.ck, a.cks, t, lane);
    v.load(a.cv, a.cvs, t, lane);
  }
  while (true) {
    const int first = max(s.i, 0), last = blocks_of(s, left);
    const int rb = s.item / a.kv_heads, own = length_of(a, s.seq) - a.prefix_len - a.n_q + 1;
    if (first < last) {
      const bool has = mine && c.seq == s.seq && c.item == s.item;
      x.clear();
      if (has) {
        int seen[MF];
#pragma unroll
        for (int f = 0; f < MF; ++f) {
          const int r = 16 * (MF * rb + f) + n, j = r / group;
          const bool live = r < rows;
          x.load(a, f, live ? reinterpret_cast<const uint16_t*>(a.q) + ((int64_t)s.seq * a.n_q + j) * a.ldq + ((int64_t)s.h * group + r % group) * D : nullptr, lane);
          seen[f] = live ? own + j : 0;
        }
        const int least = own + 16 * MF * rb / group, most = own + min(rows - 1, 16 * MF * rb + 16 * MF - 1) / group;
        bool here = true;
        while (here) {
          const int i = c.i;
          turn = 4;
          seek();
          here = mine && c.seq == s.seq && c.item == s.item;
          const int next_id = mine ? page_of(c) : 0;
          const int64_t next = token_of(c, next_id);
          Sight g;
          g.bad = (unsigned)id >= (unsigned)a.n_pages;
          g.least = least - 32 * i;
          g.most = most - 32 * i;
          g.some = g.bad || g.least < 32;
          int limit[MF];
#pragma unroll
          for (int f = 0; f < MF; ++f) limit[f] = seen[f] - 32 * i;
          x.block(a, k, v, g, limit, lane, [&]() {
            if (mine) k.load(a.ck, a.cks, next, lane);
          });
          if (mine) v.load(a.cv, a.cvs, next, lane);
          id = next_id;
        }
      }
      const bool whole = first == 0 && last == s.blocks;
#pragma unroll
      for (int f = 0; f < MF; ++f) {
        const int r0 = 16 * (MF * rb + f);
        meet<KIND, D, MF, 4>(x, f, min(16, rows - r0), has, red, flag, w, lane, [&](int r, int d, f32x4 v4, float l, float top) {
          const int row = r0 + r, q = row / group;
          const int64_t tok = (int64_t)s.seq * a.n_q + q, head = (int64_t)s.h * group + row % group;
          if (whole && !a.prefix_len) {
            store4(a.out, tok * a.ldo + head * D + d, v4 * (l == 0.f ? 0.f : 1.f / l), a.act);
          } else {
            float* part = whole ? a.own + (tok * a.q_heads + head) * RS
                                : a.part + ((2 * (int64_t)blockIdx.x + (first == 0)) * piece_rows + 16 * f + r) * RS;
            *reinterpret_cast<f32x4*>(part + d) = v4;
            if (d == 0) {
              part[D] = top;
              part[D + 1] = l;
            }
          }
        });
      }
    }
    left -= s.blocks - s.i;
    if (left <= (int)kItemCost) break;
    next_item(s);
    s.i = -(int)kItemCost;
  }
}

// Items of few blocks: a workgroup of W wavefronts takes an item, its wavefronts every Wth
// block, and they meet in LDS: one launch, nothing in the workspace.  A short prefix is taken along
// (a.fold), block by block in front of the item's own; beside a long one the sums go to the workspace.
// Bound by latency: one sequence of 300 int8 tokens, 8 heads, 6.6 us, of which a launch is 2.3 and the rest the chain
// length, page, keys, scores, weights, meeting; 8 sequences behind 1500 tokens 13.9 (32 workgroups, seven blocks to a
// wavefront).
template <int KIND, int D, int MF, int W>
__global__ void __launch_bounds__(64 * W, cu_holds(KIND <= C_F16, MF * D)) attention_item_kernel(AttnArgs a) {
  constexpr int RS = D + 4;
  extern __shared__ float red[];
  __shared__ int flag[W];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15;
  const int group = a.q_heads / a.kv_heads, rows = a.n_q * group, per_seq = a.kv_heads * a.row_blocks;
  const int seq = (int)blockIdx.x / per_seq, item = (int)blockIdx.x - seq * per_seq, rb = item / a.kv_heads, h = item - rb * a.kv_heads;
  const int length = length_of(a, seq), own = length - a.prefix_len - a.n_q + 1;
  const Fixed pages = fixed(a.table) + (int64_t)seq * a.width;
  const int pre = a.fold ? (min(length, a.prefix_len) + 31) >> 5 : 0;  // blocks of the prefix
  auto page_of = [&](int i) {
    const int t = 32 * (i < pre ? i : i - pre);
    return (i < pre ? fixed(a.prefix) : pages)[t >> a.page_log2];
  };
  auto token_of = [&](int i, int id) {
    const int64_t rec = (int64_t)((unsigned)id < (unsigned)a.n_pages ? id : 0) * a.kv_heads + h;
    return (rec << a.page_log2) + ((32 * (i < pre ? i : i - pre)) & ((1 << a.page_log2) - 1));
  };
  int i = w;
  int id = !a.fold && 32 * i < a.width << a.page_log2 ? page_of(i) : 0;  // (asked for beside the length)
  Rows16<KIND, D, MF> x;
  x.clear();
  int seen[MF];
#pragma unroll
  for (int f = 0; f < MF; ++f) {
    const int r = 16 * (MF * rb + f) + n, j = r / group;
    const bool live = r < rows;
    x.load(a, f, live ? reinterpret_cast<const uint16_t*>(a.q) + ((int64_t)seq * a.n_q + j) * a.ldq + ((int64_t)h * group + r % group) * D : nullptr, lane);
    seen[f] = live ? own + j : -(1 << 30);
  }
  const int blocks = pre + own_blocks(a, seq);
  if (a.fold && i < blocks) id = page_of(i);
  const bool past = (int64_t)length > a.prefix_len + ((int64_t)a.width << a.page_log2);
  const int least = own + 16 * MF * rb / group, most = own + min(rows - 1, 16 * MF * rb + 16 * MF - 1) / group;
  Frag<KIND, D> k, v;
  if (i < blocks) {
    const int64_t t = token_of(i, id);
    k.load(a.ck, a.cks, t, lane);
    v.load(a.cv, a.cvs, t, lane);
  }
  while (i < blocks) {
    const int next = i + W;
    const int next_id = next < blocks ? page_of(next) : 0;
    // what lies before the block, and how many tokens of its part there are
    const int from = i < pre ? 32 * i - a.prefix_len : 32 * (i - pre), part = i < pre ? a.prefix_len - 32 * i : 1 << 30;
    Sight g;
    g.bad = (unsigned)id >= (unsigned)a.n_pages;
    g.least = min(least - from, part);
    g.most = min(most - from, part);
    g.some = g.bad || g.least < 32;
    int limit[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) limit[f] = min(seen[f] - from, part);
    x.block(a, k, v, g, limit, lane, [&]() {
      if (next < blocks) k.load(a.ck, a.cks, token_of(next, next_id), lane);
    });
    if (next < blocks) v.load(a.cv, a.cvs, token_of(next, next_id), lane);
    i = next;
    id = next_id;
  }
#pragma unroll
  for (int f = 0; f < MF; ++f) {
    const int r0 = 16 * (MF * rb + f);
    meet<KIND, D, MF, W>(x, f, min(16, rows - r0), w < blocks, red, flag, w, lane, [&](int r, int d, f32x4 v4, float l, float top) {
      const int row = r0 + r, q = row / group;
      const int64_t tok = (int64_t)seq * a.n_q + q, head = (int64_t)h * group + row % group;
      if (!a.prefix_len || a.fold) {
        store4(a.out, tok * a.ldo + head * D + d, v4 * (past ? __builtin_nanf("") : l == 0.f ? 0.f : 1.f / l), a.act);
      } else {
        float* part = a.own + (tok * a.q_heads + head) * RS;
        *reinterpret_cast<f32x4*>(part + d) = v4;
        if (d == 0) {
          part[D] = top;
          part[D + 1] = l;
        }
      }
    });
  }
}

// Keys and values of a stage in LDS, as the products take them (codes widened to fp16): fragments of
// 1 KB that a wavefront reads side by side.
template <int KIND, int D> struct Stage {
  static constexpr int ES = KIND <= C_F16 ? 2 : 1;
  static constexpr int NB = D == 256 ? 1 : 2;                       // blocks of a stage
  static constexpr int KF = NB * 2 * (D / 32), VF = NB * (D / 16);  // fragments of keys, of values
  static constexpr int LP = NB * D * ES / 64;                       // 1 KB loads of a wavefront (keys and values)
  u32x4 k[KF][64], v[VF][64];
  float s[ES == 1 ? 2 : 1][NB * 32];
};

// The shared prefix: rows of all sequences (sequence by sequence, a query's heads of the kv
// head side by side) against it.  A workgroup takes one share of the prefix's blocks, its four
// wavefronts 16 MF rows each; keys and values go through LDS, two stages of them, where they come
// once for all wavefronts and codes are widened once.  Workgroups with the same blocks, for other
// rows, have indexes 8 apart: one XCD's, so that its L2 has them.
// 128 sequences of 4 rows a kv head behind 32768 fp8 tokens, 8 heads of 128, bf16: 115 us for 69 GFLOP, 0.60 PFLOP/s (a bf16
// product of 8192^3: 1.16).  Neither memory (71 MB) nor the matrix cores (29% busy) are its limit, but the order of its
// work: scores, weights (some 8 vector instructions and a quarter-rate exponential a score) and products follow one
// another in each of two wavefronts a SIMD (the registers hold no third), which wait 33% of the time, together at a
// barrier each 64 tokens.
template <int KIND, int D, int MF>
__global__ void __launch_bounds__(256, 2) attention_prefix_kernel(AttnArgs a) {
  using S = Stage<KIND, D>;
  using R = Rows16<KIND, D, MF>;
  constexpr int RS = D + 4, ES = S::ES, NB = S::NB;
  __shared__ S stage[2];
  __shared__ uint32_t odd_values;  // 1: some were not finite (in LDS they are zeros)
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, qd = lane >> 4;
  const int group = a.q_heads / a.kv_heads, rows = a.batch * a.n_q * group;
  const int teams = (rows + 64 * MF - 1) / (64 * MF);  // workgroups with the same blocks
  const int of8 = (int)blockIdx.x / (8 * teams), rem = (int)blockIdx.x - of8 * 8 * teams, pair = of8 * 8 + (rem & 7);
  if (pair >= a.kv_heads * a.shares) return;
  const int h = pair % a.kv_heads, share = pair / a.kv_heads;
  const int r0 = ((rem >> 3) * 4 + w) * 16 * MF;
  const int blocks = (a.prefix_len + 31) >> 5;
  const int first = (int)((int64_t)blocks * share / a.shares), last = (int)((int64_t)blocks * (share + 1) / a.shares);
  Rows16<KIND, D, MF> x;
  x.clear();
  int seen[MF], most = 0, least = 1 << 30;
#pragma unroll
  for (int f = 0; f < MF; ++f) {
    const int r = r0 + 16 * f + n, tok = min(r, rows - 1) / group;
    const bool live = r < rows;
    x.load(a, f, live ? reinterpret_cast<const uint16_t*>(a.q) + tok * a.ldq + ((int64_t)h * group + r % group) * D : nullptr, lane);
    const int b = tok / a.n_q;
    seen[f] = live ? max(0, min(a.prefix_len, length_of(a, b) - a.n_q + 1 + tok % a.n_q)) : 0;
    most = max(most, seen[f]);
    least = min(least, live ? seen[f] : 1 << 30);
  }
#pragma unroll
  for (int d = 1; d < 16; d *= 2) {
    most = max(most, __shfl_xor(most, d, 64));
    least = min(least, __shfl_xor(least, d, 64));
  }
  most = __builtin_amdgcn_readfirstlane(most);
  least = __builtin_amdgcn_readfirstlane(least);
  auto id_of = [&](int i) { return fixed(a.prefix)[(32 * i) >> a.page_log2]; };
  auto token_of = [&](int i, int id) {
    const int64_t rec = (int64_t)((unsigned)id < (unsigned)a.n_pages ? id : 0) * a.kv_heads + h;
    return (rec << a.page_log2) + ((32 * i) & ((1 << a.page_log2) - 1));
  };
  // A stage's keys, then its values: load j of wavefront w is the KB 4 j + w of either.
  constexpr int KB = NB * D * ES / 32;  // KB of keys (and of values) in a stage
  static_assert(KB % 4 == 0 && KB / 4 * 2 == S::LP, "every wavefront brings as much");
  u32x4 in[S::LP];
  f32x4 in_s;
  int ids[NB];
  auto ask = [&](int i0) {  // blocks i0 .. (the last one again past the share's end)
    int64_t t[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int i = min(i0 + b, last - 1);
      t[b] = token_of(i, ids[b] = id_of(i));
    }
#pragma unroll
    for (int j = 0; j < S::LP; ++j) {
      const int p = 4 * (j % (S::LP / 2)) + w, b = p / (KB / NB);
      const uint8_t* base = j < S::LP / 2 ? a.ck : a.cv;
      in[j] = *reinterpret_cast<const u32x4*>(base + (NB > 1 && b ? t[NB - 1] : t[0]) * (D * ES) + (p % (KB / NB)) * 1024 + lane * 16);
    }
    if constexpr (ES == 1)
      if (tid < 16 * NB) {
        const int j = tid & 7, b = NB > 1 ? (tid >> 3) & 1 : 0;
        const float* base = tid < 8 * NB ? a.cks : a.cvs;
        in_s = *reinterpret_cast<const f32x4*>(base + (NB > 1 && b ? t[NB - 1] : t[0]) + 4 * j);
      }
  };
  // Values enter LDS as finite ones, tokens past the prefix as zeros: rows that do not see a token
  // then need no more than a weight of 0.
  auto put = [&](S& to, int i0) {
    if constexpr (!is_i8(KIND)) {
      uint32_t seen16 = 0u, any = 0u;
      if (32 * (i0 + NB) > a.prefix_len) {
#pragma unroll
        for (int j = S::LP / 2; j < S::LP; ++j) {
          const int p = 4 * (j % (S::LP / 2)) + w;
          in[j] &= R::kept(a.prefix_len - 32 * (i0 + p / (KB / NB)), lane);
        }
      }
#pragma unroll
      for (int j = S::LP / 2; j < S::LP; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (ES == 2) seen16 = max2(seen16, in[j][e] & 0x7fff7fffu);
          else any |= (in[j][e] & 0x7f7f7f7fu) + 0x01010101u;
        }
      const bool odd = ES == 2 ? max(seen16 & 0xffffu, seen16 >> 16) >= R::kInf : (any & 0x80808080u) != 0;
      if (__ballot(odd)) {
#pragma unroll
        for (int j = S::LP / 2; j < S::LP; ++j) {
          const u32x4 o = in[j];
          in[j] = o & ~u32x4{R::strange(o[0]), R::strange(o[1]), R::strange(o[2]), R::strange(o[3])};
        }
        if (lane == 0) odd_values = 1u;
      }
    }
#pragma unroll
    for (int j = 0; j < S::LP; ++j) {
      const int p = 4 * (j % (S::LP / 2)) + w;
      u32x4(*dst)[64] = j < S::LP / 2 ? to.k : to.v;
      if constexpr (ES == 2) {
        dst[p][lane] = in[j];
      } else {
        dst[2 * p][lane] = widen8<KIND>(in[j][0], in[j][1]);
        dst[2 * p + 1][lane] = widen8<KIND>(in[j][2], in[j][3]);
      }
    }
    if constexpr (ES == 1)
      if (tid < 16 * NB) *reinterpret_cast<f32x4*>(&to.s[tid / (8 * NB)][4 * (tid % (8 * NB))]) = in_s;
  };
  if (tid == 0) odd_values = 0u;
  __syncthreads();
  if (first < last) {
    ask(first);
    put(stage[0], first);
  }
  __syncthreads();
  for (int i0 = first, at = 0; i0 < last; i0 += NB, at ^= 1) {
    const S& st = stage[at];
    bool bad[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) bad[b] = (unsigned)ids[b] >= (unsigned)a.n_pages;
    if (i0 + NB < last) ask(i0 + NB);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int i = i0 + b;
      Sight g;
      g.bad = bad[b];
      g.least = least - 32 * i;
      g.most = most - 32 * i;
      g.some = g.bad || g.least < 32;
      if (i >= last || g.most <= 0) continue;
      int limit[MF];
#pragma unroll
      for (int f = 0; f < MF; ++f) limit[f] = seen[f] - 32 * i;
      x.scores([&](int t, int s) { return st.k[(b * 2 + t) * (D / 32) + s][lane]; });
      f32x4 ks[2], vs[2];
      if constexpr (ES == 1) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          ks[t] = *reinterpret_cast<const f32x4*>(&st.s[0][32 * b + 16 * t + 4 * qd]);
          vs[t] = *reinterpret_cast<const f32x4*>(&st.s[1][32 * b + 16 * t + 4 * qd]);
        }
      }
      x.weigh(a, ks, vs, g, limit, lane);
      x.add([&](int e) { return st.v[b * (D / 16) + e][lane]; });
    }
    if (i0 + NB < last) put(stage[at ^ 1], i0 + NB);
    __syncthreads();
  }
  if (!is_i8(KIND) && odd_values) {  // (rare: the values once more, as memory has them)
    for (int i = first; i < min(last, (most + 31) >> 5); ++i) {
      const int64_t t = token_of(i, id_of(i));
      const u32x4 any = R::kept(a.prefix_len - 32 * i, lane);
      int limit[MF];
#pragma unroll
      for (int f = 0; f < MF; ++f) limit[f] = seen[f] - 32 * i;
#pragma unroll
      for (int e = 0; e < D / 16; ++e) {
        __builtin_amdgcn_sched_barrier(0);
        const u32x4 v = *reinterpret_cast<const u32x4*>(a.cv + t * (D * ES) + (ES == 2 ? e : e >> 1) * 1024 + lane * 16) & any;
        x.count(ES == 2 ? v : e & 1 ? widen8<KIND>(v[2], v[3]) : widen8<KIND>(v[0], v[1]), e, limit, lane);
      }
    }
  }
#pragma unroll
  for (int f = 0; f < MF; ++f) {
    const int r = r0 + 16 * f + n;
    const float s = quarters_sum(x.sum[f]);
    if (r >= rows) continue;
    const int tok = r / group;
    float* part = a.pre + (((int64_t)share * a.batch * a.n_q + tok) * a.q_heads + (int64_t)h * group + r % group) * RS;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) *reinterpret_cast<f32x4*>(part + 16 * e + 4 * qd) = x.acc[f][e];
    if (qd == 0) {
      part[D] = x.ref[f];
      part[D + 1] = s;
    }
  }
}

// Pieces of a query row joined: of the prefix's shares, of the workgroups that shared its
// item.  D / 4 lanes hold a row; GP groups of them take the pieces of one row in turn, four at
// a time, and meet in LDS.  Bound by memory where rows are many: 17 pieces of 4096 rows, 37 MB, 9.2 us.
template <int D, int GP>
__global__ void __launch_bounds__(GP == 32 ? 32 * D / 4 : 256) attention_join_kernel(AttnArgs a) {
  constexpr int RS = D + 4, L = D / 4, T = GP == 32 ? 32 * L : 256, R = T / (L * GP);  // rows of a workgroup
  __shared__ float red[GP > 1 ? GP : 1][RS];
  const int tid = threadIdx.x, d = 4 * (tid % L), gr = tid / L % GP;
  const int group = a.q_heads / a.kv_heads;
  const int rank = (int)blockIdx.x * R + tid / (L * GP);  // (fewer than 2^26)
  if (R > 1 && rank >= a.batch * a.n_q * a.q_heads) return;
  const int64_t tok = rank / a.q_heads;
  const int head = rank - (int)tok * a.q_heads, b = (int)tok / a.n_q, h = head / group;
  const int row = ((int)tok - b * a.n_q) * group + head % group, frag_rows = 16 * a.frags, rb = row / frag_rows;
  const int piece_rows = min(a.n_q * group, frag_rows);
  const int length = length_of(a, b);
  const int blocks = own_blocks(a, b);
  uint32_t g0 = 0;
  int pieces = blocks > 0;  // of the item
  if (!a.direct && blocks) {
    const uint32_t per = a.starts[a.batch + 1], s0 = a.starts[b] + (rb * a.kv_heads + h) * item_cost(blocks) + kItemCost;
    g0 = s0 / per;
    pieces = (int)((s0 + blocks - 1) / per - g0) + 1;
  }
  if (pieces == 1 && !a.prefix_len) return;  // written where it was computed
  const int shares = length > 0 ? a.shares : 0, n = shares + pieces;
  float top = kNoReference, l = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = gr; i0 < n; i0 += 4 * GP) {
    f32x4 o[4];
    float r[4], s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + j * GP;
      if (i < n) {
        const int64_t g = g0 + (uint32_t)(i - shares);
        const float* p = i < shares ? a.pre + (((int64_t)i * a.batch * a.n_q + tok) * a.q_heads + head) * RS
                         : pieces == 1 ? a.own + (tok * a.q_heads + head) * RS
                                       : a.part + ((2 * g + (i == shares)) * piece_rows + row % frag_rows) * RS;
        o[j] = *reinterpret_cast<const f32x4*>(p + d);
        r[j] = p[D];
        s[j] = p[D + 1];
      } else {
        o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        r[j] = kNoReference;
        s[j] = 0.f;
      }
    }
    float next = top;
#pragma unroll
    for (int j = 0; j < 4; ++j) next = fmaxf(next, r[j]);
    const float c = join_factor(top, next);
    v *= c;
    l *= c;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float e = join_factor(r[j], next);
      v += o[j] * e;
      l += s[j] * e;
    }
    top = next;
  }
  if constexpr (GP > 1) {
    *reinterpret_cast<f32x4*>(&red[gr][d]) = v;
    if (d == 0) {
      red[gr][D] = top;
      red[gr][D + 1] = l;
    }
    __syncthreads();
    if (gr) return;
    const int used = min(GP, n);
    for (int i = 0; i < used; ++i) top = fmaxf(top, red[i][D]);
    l = 0.f;
    v = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < used; ++i) {
      const float c = join_factor(red[i][D], top);
      v += c * *reinterpret_cast<const f32x4*>(&red[i][d]);
      l += c * red[i][D + 1];
    }
  }
  const bool past = (int64_t)length > a.prefix_len + ((int64_t)a.width << a.page_log2);
  store4(a.out, tok * a.ldo + (int64_t)head * D + d, v * (past ? __builtin_nanf("") : l == 0.f ? 0.f : 1.f / l), a.act);
}

// Fragments of 16 rows that a wavefront takes.  us with 1 and 2 (32 heads of 128, 8 kv heads): 16 sequences up to 4000
// tokens, 20 rows int8 32.4, 31.3, bf16 48.1, 39.3; 64 of 1000, 32 rows int8 36.6, 31.2, bf16 52, 55.  (40 rows, which fill
// three of one and four of two: 28.0, 32.6, bf16 38.1, 38.1: for them one would be the better.)  FP8 codes with both parts of fp16 weights fit the
// registers with one alone at dim 128: 20 rows 30.9, 98; 32 rows 35.6, 138.
constexpr bool two_frags(int kind, int dim) { return dim == 64 || (dim == 128 && kind != C_F8_F16); }
int kind_of(const AttnArgs& a) {
  const bool bf16 = a.act == MXMOE_BF16;
  return a.qmax == kQmaxF8 ? (bf16 ? C_F8 : C_F8_F16) : a.qmax ? (bf16 ? C_I8 : C_I8_F16) : bf16 ? C_BF16 : C_F16;
}
int frags_of(int64_t rows, int kind, int dim) { return rows > 16 && two_frags(kind, dim) ? 2 : 1; }

// Wavefronts to an item, or 0 where the list of costs is shared.  An item to a workgroup is one launch
// and needs no search for its place; from 64 blocks on its length is what the launch waits for, and
// few long items leave CUs idle.  us with 4 wavefronts to an item, 8, shared (int8, dim 128, 4 rows; sequences of
// 3/4 to all of the length): 8 items of 4 blocks 4.9, 5.0, 8.2; 8 of 63 17.5, 14.7, 12.1; 128 of 63 20.4, 16.7,
// 20.1; 512 of 4 7.6, 10.2, 14.4; 512 of 63 47.3, 49.0, 54.3; 2048 of 16 51.0, 67.1, 62.9.  (By the table's
// width, all that the host knows: short sequences behind a wide table take the shared list.)
int direct_of(int64_t items, int64_t longest) {
  if (longest > 64 || (longest > 48 && items < 16)) return 0;
  return items <= 256 ? 8 : 4;
}

struct Plan { int fold, direct, frags, row_blocks, pre_frags, shares, grid, pieces; size_t starts, part, own, pre, total; };
Plan plan_of(const AttnArgs& a, int dim) {
  Plan p = {};
  const int group = a.q_heads / a.kv_heads, rows = a.n_q * group;
  const int64_t rs = 4 * (int64_t)(dim + 4), all = (int64_t)a.batch * a.n_q * a.q_heads;
  p.frags = frags_of(rows, kind_of(a), dim);
  p.row_blocks = (rows + 16 * p.frags - 1) / (16 * p.frags);
  const int64_t items = (int64_t)a.batch * a.kv_heads * p.row_blocks, longest = ((int64_t)a.width << a.page_log2) / 32, most = items * longest;
  const int64_t pre = ((int64_t)a.prefix_len + 31) / 32;
  // A prefix is taken along by every item where that costs less than two launches more: few blocks to
  // read again (by its bytes), and items not much longer.  us, taken along or apart (int8, dim 128, 4 rows): 8 sequences
  // behind 1500 tokens 13.6, 17.7; 64 22.7, 33.3; 128 38.1, 42.0; 256 66, 54; 512 behind 300 58, 68; 64 behind 2500 32, 38;
  // 4 18.6, 17.3; dim 256, 128 behind 300 27.7, 39, behind 1500 63, 51
  p.fold = pre > 0 && (pre + longest <= 64 || (items >= 64 && pre <= 80 && longest <= 64)) && pre * items * dim <= 50000 * 128;
  p.direct = p.fold ? direct_of(items, std::min<int64_t>(pre + longest, 48)) : direct_of(items, longest);
  p.grid = (int)std::min<int64_t>(256 * cu_holds(a.qmax == 0, p.frags * dim), std::max<int64_t>(1, (most + 3) / 4));  // a block to a wavefront
  if (a.prefix_len && !p.fold) {
    const int64_t prows = (int64_t)a.batch * rows;
    // (us with 1 and 2 behind 16000 int8 tokens: 128 rows a kv head 37.9, 41.1, 256 54.0, 54.3, 512 85, 77)
    p.pre_frags = prows <= 128 || dim == 256 ? 1 : 2;
    const int64_t wgs = ((prows + 64 * p.pre_frags - 1) / (64 * p.pre_frags)) * a.kv_heads;
    const int64_t blocks = ((int64_t)a.prefix_len + 31) / 32;
    p.shares = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>((blocks + 3) / 4, 64), 512 / wgs));
  }
  // pieces of a row at the most, if all sequences are as long as the table allows
  p.pieces = p.shares + 1 + (p.direct ? 0 : (int)(p.grid / items));
  auto align = [](size_t n) { return (n + 255) / 256 * 256; };
  size_t o = 0;
  p.starts = o; o = align(o + (p.direct ? 0 : 4 * ((size_t)a.batch + 2)));
  p.part = o; o = align(o + (p.direct ? 0 : 2) * (size_t)p.grid * std::min(rows, 16 * p.frags) * rs);
  p.own = o; o = align(o + (a.prefix_len && !p.fold ? (size_t)all * rs : 0));
  p.pre = o; o = align(o + (size_t)p.shares * all * rs);
  p.total = o;
  return p;
}

// LDS of meet
size_t meet_bytes(const AttnArgs& a, int dim, int w) { return 4 * (size_t)w * std::min(16, a.n_q * (a.q_heads / a.kv_heads)) * (dim + 4); }

template <int KIND, int D, int MF, int W> hipError_t go_item(const AttnArgs& a, const Plan& p, hipStream_t s) {
  hipLaunchKernelGGL((attention_item_kernel<KIND, D, MF, W>), dim3((unsigned)(a.batch * a.kv_heads * p.row_blocks)), dim3(64 * W),
                     meet_bytes(a, D, W), s, a);
  return hipGetLastError();
}
template <int KIND, int D, int MF> hipError_t go_own(const AttnArgs& a, const Plan& p, hipStream_t s) {
  if (p.direct) {
    if constexpr (D < 256)  // (8 wavefronts of 256 elements: their rows in LDS are for one workgroup alone)
      if (p.direct == 8) return go_item<KIND, D, MF, 8>(a, p, s);
    return go_item<KIND, D, MF, 4>(a, p, s);
  }
  hipLaunchKernelGGL((attention_kernel<KIND, D, MF>), dim3(p.grid), dim3(256), meet_bytes(a, D, 4), s, a);
  return hipGetLastError();
}
template <int KIND, int D, int MF> hipError_t go_prefix(const AttnArgs& a, hipStream_t s) {
  const int64_t rows = (int64_t)a.batch * a.n_q * (a.q_heads / a.kv_heads);
  const unsigned teams = (unsigned)((rows + 64 * MF - 1) / (64 * MF)), pairs = (unsigned)(a.kv_heads * a.shares);
  hipLaunchKernelGGL((attention_prefix_kernel<KIND, D, MF>), dim3((pairs + 7) / 8 * 8 * teams), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <int KIND, int D> hipError_t go(const AttnArgs& a, const Plan& p, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (a.prefix_len && !p.fold) {
    if constexpr (D <= 128)
      if (p.pre_frags == 2) e = go_prefix<KIND, D, 2>(a, s);
    if (p.pre_frags == 1) e = go_prefix<KIND, D, 1>(a, s);
    if (e != hipSuccess) return e;
  }
  if constexpr (two_frags(KIND, D))
    if (p.frags == 2) e = go_own<KIND, D, 2>(a, p, s);
  if (p.frags == 1) e = go_own<KIND, D, 1>(a, p, s);
  if (e != hipSuccess || (p.direct && (!a.prefix_len || p.fold))) return e;
  const unsigned all = (unsigned)(a.batch * a.n_q * a.q_heads);
  // groups to a row: all pieces of few rows at once, many rows without a meeting.  us with 1, 1024 / dim, 32 (behind 16000
  // int8 tokens, 32 heads of 128): 4 sequences, 64 pieces 41.7, 26.1, 25.1; 32, 64 pieces 44, 37.8, 42.4; 64, 33 pieces 56.2,
  // 54.4, 63.1; 128, 17 pieces 77.4, 79.6, 96
  if (p.pieces <= 8 || (p.pieces <= 32 && all >= 4096))
    hipLaunchKernelGGL((attention_join_kernel<D, 1>), dim3((all * (D / 4) + 255) / 256), dim3(256), 0, s, a);
  else if (p.pieces <= 32 || all > 512 || D == 256)
    hipLaunchKernelGGL((attention_join_kernel<D, 1024 / D>), dim3(all), dim3(256), 0, s, a);
  else if constexpr (D < 256)
    hipLaunchKernelGGL((attention_join_kernel<D, 32>), dim3(all), dim3(8 * D), 0, s, a);
  return hipGetLastError();
}
template <int KIND> hipError_t by_dim(const AttnArgs& a, const Plan& p, int dim, hipStream_t s) {
  return dim == 64 ? go<KIND, 64>(a, p, s) : dim == 128 ? go<KIND, 128>(a, p, s) : go<KIND, 256>(a, p, s);
}

}  // namespace

size_t attention_workspace(const AttnArgs& a, int dim) { return plan_of(a, dim).total; }

hipError_t launch_attention(AttnArgs a, int dim, hipStream_t s) {
  const Plan p = plan_of(a, dim);
  uint8_t* ws = reinterpret_cast<uint8_t*>(a.workspace);
  a.starts = reinterpret_cast<uint32_t*>(ws + p.starts);
  a.part = reinterpret_cast<float*>(ws + p.part);
  a.own = reinterpret_cast<float*>(ws + p.own);
  a.pre = reinterpret_cast<float*>(ws + p.pre);
  a.frags = p.frags;
  a.row_blocks = p.row_blocks;
  a.shares = p.shares;
  a.direct = p.direct;
  a.fold = p.fold;
  switch (kind_of(a)) {
    case C_BF16: return by_dim<C_BF16>(a, p, dim, s);
    case C_F16: return by_dim<C_F16>(a, p, dim, s);
    case C_I8: return by_dim<C_I8>(a, p, dim, s);
    case C_F8: return by_dim<C_F8>(a, p, dim, s);
    case C_I8_F16: return by_dim<C_I8_F16>(a, p, dim, s);
    default: return by_dim<C_F8_F16>(a, p, dim, s);
  }
}

}  // namespace mxmoe
