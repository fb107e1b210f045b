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
// is that of the products, so that they keep 11 bits whatever the scales are; scales
// under 2^-80 do not move it.  The sum of the weights is of fp32 values, before any rounding.
// 16-bit rows: weights are rounded to the rows' dtype (half a step each, of random
// sign: the sum over many tokens errs by less than the output's own rounding).
//
// Tokens past a row's last are left out by selection, whatever they hold: their scores
// become -inf, their values zeros.  Where rows of a tile see different tokens and a value
// there is not finite, rows are added one by one, each with the values that it sees.
#include "kvcache.h"
#include "lanes.h"

namespace mxmoe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

enum CacheKind { C_BF16, C_F16, C_I8, C_F8 };
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kBase = 8.f;              // weights are 2^8 at the reference ..
constexpr float kMostWeight = 0x1p15f;    // .. and move it past 2^15 (fp16 ends at 2^16)
constexpr float kLeastScale = 0x1p-80f;

template <int KIND> LANES_INL f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (KIND == C_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// 4 codes -> 4 fp16 values
template <int KIND> LANES_INL u32x2 widen(uint32_t w) {
  if constexpr (KIND == C_I8) {  // 1024 + 128 + q, less 1152
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

LANES_INL float quarters_max(float v) {  // over the four lanes of a query row
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
LANES_INL float quarters_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// Keys and values of 32 tokens as a lane holds them.
template <int KIND, int D> struct Block {
  static constexpr int ES = KIND <= C_F16 ? 2 : 1, N = D * ES / 32;
  u32x4 k[N], v[N];
  f32x4 ks[2], vs[2];
  LANES_INL void load(const AttnArgs& a, int64_t rec, int at, int lane) {
    const uint8_t* kp = a.ck + ((rec << a.page_log2) + at) * (D * ES) + lane * 16;
    const uint8_t* vp = a.cv + ((rec << a.page_log2) + at) * (D * ES) + lane * 16;
#pragma unroll
    for (int i = 0; i < N; ++i) k[i] = *reinterpret_cast<const u32x4*>(kp + 1024 * i);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = *reinterpret_cast<const u32x4*>(vp + 1024 * i);
    if constexpr (ES == 1) {
      const int64_t s = (rec << a.page_log2) + at + 4 * (lane >> 4);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        ks[i] = *reinterpret_cast<const f32x4*>(a.cks + s + 16 * i);
        vs[i] = *reinterpret_cast<const f32x4*>(a.cvs + s + 16 * i);
      }
    }
  }
  LANES_INL u32x4 key(int tile, int step) const {
    if constexpr (ES == 2) return k[tile * (D / 32) + step];
    const u32x4 p = k[tile * (D / 64) + (step >> 1)];
    return step & 1 ? widen8<KIND>(p[2], p[3]) : widen8<KIND>(p[0], p[1]);
  }
  LANES_INL u32x4 value(int tile) const {
    if constexpr (ES == 2) return v[tile];
    const u32x4 p = v[tile >> 1];
    return tile & 1 ? widen8<KIND>(p[2], p[3]) : widen8<KIND>(p[0], p[1]);
  }
};

// 16 query rows of a wavefront: row lane % 16.
template <int KIND, int D> struct Rows16 {
  static constexpr int ES = KIND <= C_F16 ? 2 : 1;
  u32x4 q[D / 32];
  f32x4 acc[D / 16];   // elements 16 i + 4 (lane / 16) + (0..3)
  float ref, sum;      // the row's reference, the sum of its weights (this lane's tokens)
  float mul;           // from a product of codes to a score, in powers of 2 (without a cap)

  LANES_INL void init(const AttnArgs& a, const uint16_t* row, int lane) {
    const int qd = lane >> 4;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    ref = -__builtin_inff();
    sum = 0.f;
    mul = a.scale;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const int c = ES == 2 ? 4 * s + qd : 8 * (s >> 1) + 2 * qd + (s & 1);
      q[s] = row ? (u32x4) * reinterpret_cast<const u32x4_any*>(row + 8 * c) : u32x4{0u, 0u, 0u, 0u};
    }
    if (ES == 1 && a.act == MXMOE_BF16) {
      uint32_t m = 0u;
#pragma unroll
      for (int s = 0; s < D / 32; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = max2(m, q[s][i] & 0x7fff7fffu);
      m = max2(m, (uint32_t)__shfl_xor((int)m, 16, 64));
      m = max2(m, (uint32_t)__shfl_xor((int)m, 32, 64));
      const int e = (int)(max(m & 0xffffu, m >> 16) >> 7);  // exponent of the largest
      const int up = e == 255 ? 0 : min(127, 127 + 14 - max(e, 1));
#pragma unroll
      for (int s = 0; s < D / 32; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x2 w = unpack2<MXMOE_BF16>(q[s][i]);
          q[s][i] = pack2<MXMOE_F16>(__builtin_ldexpf(w[0], up), __builtin_ldexpf(w[1], up));
        }
      mul = __builtin_ldexpf(mul, -up);
    }
    if (a.softcap > 0.f) mul = mul / a.softcap; else mul *= kLog2e;
  }

  // 32 tokens; limit: how many of them the lane's row sees.  MASK: some row sees fewer than
  // 32 (or the page is bad: NaN for whoever sees it); most: what the row that sees most of
  // them does, least: the real row that sees least.
  template <bool MASK>
  LANES_INL void add(const AttnArgs& a, const Block<KIND, D>& b, int lane, int limit, int most, int least, bool bad) {
    const int t0 = 4 * (lane >> 4);
    float x[8], w[8];
    {
      f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) s[t] = mfma<KIND>(b.key(t, i), q[i], s[t]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = s[i >> 2][i & 3] * mul;
        if constexpr (ES == 1) x[i] *= b.ks[i >> 2][i & 3];
      }
    }
    if (a.softcap > 0.f) {
      const float c = a.softcap * kLog2e;
#pragma unroll
      for (int i = 0; i < 8; ++i)  // tanh y = 1 - 2 / (1 + e^(2 y))
        x[i] = c - 2.f * c * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x[i] * (2.f * kLog2e)));
    }
    float vs[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (ES == 1) vs[i] = b.vs[i >> 2][i & 3]; else vs[i] = 1.f;
      if constexpr (MASK) {
        const bool in = t0 + (i & 3) + 16 * (i >> 2) < limit;
        x[i] = in ? (bad ? __builtin_nanf("") : x[i]) : -__builtin_inff();
        vs[i] = in ? vs[i] : 0.f;
      }
    }
    auto weights = [&](float r, float (&p)[8]) {
      float most_w = 0.f;
      const float off = kBase - (r == -__builtin_inff() ? 0.f : r);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(x[i] + off);
        w[i] = ES == 1 ? p[i] * vs[i] : p[i];
        most_w = fmaxf(most_w, w[i]);
      }
      return most_w;
    };
    float p[8];
    const float top = weights(ref, p);
    // a row without a reference takes one from its first tokens
    bool move = top > kMostWeight;
    if (ref == -__builtin_inff()) {
#pragma unroll
      for (int i = 0; i < 8; ++i) move |= x[i] > -__builtin_inff();
    }
    if (__ballot(move)) {
      float m = -__builtin_inff();
#pragma unroll
      for (int i = 0; i < 8; ++i)
        m = fmaxf(m, x[i] + (ES == 1 ? __builtin_amdgcn_logf(fmaxf(vs[i], kLeastScale)) : 0.f));
      m = quarters_max(m);
      const float next = fmaxf(ref, m);
      const float f = ref == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(ref - next);  // (nothing summed yet)
      ref = next;
      sum *= f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) acc[i] *= f;
      weights(ref, p);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += p[i];
    u32x4 pw;
#pragma unroll
    for (int i = 0; i < 4; ++i) pw[i] = pack2<KIND == C_BF16 ? MXMOE_BF16 : MXMOE_F16>(w[2 * i], w[2 * i + 1]);
    if constexpr (!MASK) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) acc[i] = mfma<KIND>(b.value(i), pw, acc[i]);
    } else {
      // tokens j of the lane's eight that come before a limit, as a mask of 16-bit halves
      auto cut = [&](u32x4 v, int lim) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = t0 + 2 * (i & 1) + 16 * (i >> 1);
          v[i] &= (t < lim ? 0xffffu : 0u) | (t + 1 < lim ? 0xffff0000u : 0u);
        }
        return v;
      };
      constexpr uint32_t kInf = KIND == C_BF16 ? 0x7f80u : 0x7c00u;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const u32x4 v = cut(b.value(i), most);
        bool odd = false;
        if (least < most) {
#pragma unroll
          for (int j = 0; j < 4; ++j) odd |= (v[j] & kInf) == kInf || (v[j] & (kInf << 16)) == kInf << 16;
        }
        if (!__ballot(odd)) {
          acc[i] = mfma<KIND>(v, pw, acc[i]);
        } else {
          f32x4 out = acc[i];
          for (int r = 0; r < 16; ++r) {
            const f32x4 o = mfma<KIND>(cut(v, __builtin_amdgcn_readlane(limit, r)), pw, acc[i]);
            if ((lane & 15) == r) out = o;
          }
          acc[i] = out;
        }
      }
    }
  }
};

// A wavefront takes 16 query rows of a sequence and kv head, and all tokens they see.
template <int KIND, int D>
__global__ void __launch_bounds__(64) attention_kernel(AttnArgs a) {
  const int lane = threadIdx.x, n = lane & 15, qd = lane >> 4;
  const int group = a.q_heads / a.kv_heads, rows = a.n_q * group, frags = (rows + 15) / 16;
  const int frag = (int)blockIdx.x % frags, item = (int)blockIdx.x / frags;
  const int h = item % a.kv_heads, s = item / a.kv_heads;
  const int page = 1 << a.page_log2;
  const int length = a.lengths[s];
  const bool beyond = (int64_t)length > a.prefix_len + (int64_t)a.width * page;
  const int r = 16 * frag + n, j = r / group;
  const bool live = r < rows;
  const int64_t head = (int64_t)h * group + r % group;
  const int64_t tok = (int64_t)s * a.n_q + j;
  Rows16<KIND, D> x;
  x.init(a, live ? reinterpret_cast<const uint16_t*>(a.q) + tok * a.ldq + head * D : nullptr, lane);
  const int seen = live ? max(0, length - a.n_q + 1 + j) : 0;  // tokens that the row sees
  const int j0 = (16 * frag) / group, j1 = min(rows - 1, 16 * frag + 15) / group;
  const int least = max(0, length - a.n_q + 1 + j0), most = beyond ? 0 : max(0, length - a.n_q + 1 + j1);
  for (int part = 0; part < 2; ++part) {
    const int first = part ? a.prefix_len : 0;  // position of the part's first token
    const int end = part ? most - first : min(most, a.prefix_len);
    const int32_t* pages = part ? a.table + (int64_t)s * a.width : a.prefix;
    for (int t = 0; t < end; t += 32) {
      const int id = pages[t >> a.page_log2];
      const bool bad = id < 0 || id >= a.n_pages;
      Block<KIND, D> b;
      b.load(a, (int64_t)(bad ? 0 : id) * a.kv_heads + h, t & (page - 1), lane);
      // (the prefix may end inside a block)
      const int full = part ? 1 << 30 : a.prefix_len;
      const int lo = min(least - first, full) - t, hi = min(end, full) - t;
      if (lo >= 32 && !bad) x.template add<false>(a, b, lane, 32, 32, 32, false);
      else x.template add<true>(a, b, lane, min(seen - first, full) - t, hi, lo, bad);
    }
  }
  const float sum = quarters_sum(x.sum);
  if (!live) return;
  const float f = beyond ? __builtin_nanf("") : sum == 0.f ? 0.f : 1.f / sum;
  uint16_t* out = reinterpret_cast<uint16_t*>(a.out) + tok * a.ldo + head * D + 4 * qd;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const f32x4 o = x.acc[i] * f;
    u32x2 w;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      w[e] = a.act == MXMOE_BF16 ? pack2<MXMOE_BF16>(o[2 * e], o[2 * e + 1]) : pack2<MXMOE_F16>(o[2 * e], o[2 * e + 1]);
    typedef u32x2 u32x2_half __attribute__((aligned(2)));
    *reinterpret_cast<u32x2_half*>(out + 16 * i) = w;
  }
}

template <int KIND, int D> hipError_t go(const AttnArgs& a, hipStream_t s) {
  const int64_t frags = (a.n_q * (a.q_heads / a.kv_heads) + 15) / 16;
  hipLaunchKernelGGL((attention_kernel<KIND, D>), dim3((unsigned)(frags * a.batch * a.kv_heads)), dim3(64), 0, s, a);
  return hipGetLastError();
}
template <int KIND> hipError_t by_dim(const AttnArgs& a, int dim, hipStream_t s) {
  return dim == 64 ? go<KIND, 64>(a, s) : dim == 128 ? go<KIND, 128>(a, s) : go<KIND, 256>(a, s);
}

}  // namespace

size_t attention_workspace(const AttnArgs&, int) { return 0; }

hipError_t launch_attention(const AttnArgs& a, int dim, hipStream_t s) {
  if (a.qmax == kQmaxF8) return by_dim<C_F8>(a, dim, s);
  if (a.qmax) return by_dim<C_I8>(a, dim, s);
  return a.act == MXMOE_BF16 ? by_dim<C_BF16>(a, dim, s) : by_dim<C_F16>(a, dim, s);
}

}  // namespace mxmoe
