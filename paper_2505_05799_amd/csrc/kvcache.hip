// Heads of new tokens into the paged cache (norm, rotation, 8-bit codes in one pass),
// and rows of the cache back.
//
//   y = x r w,  r = 1 / sqrt(mean x^2 + eps)       (64-bit sum and root; queries and keys)
//   (a, b) -> (a cos - b sin, b cos + a sin)        angle = position * frequency, in 64 bits
//   codes, scale: the per-token recipe of rowquant.h on the fp32 values of a head's row
//
// dim / 8 lanes hold a head's row, 8 elements each.  Keys are written in the 16-byte pieces that a
// row consists of.  A value's elements lie 16 bytes apart there, next to those of other tokens:
// 32 tokens whose slots are one block of the cache go through LDS and leave as whole pieces (and come
// back that way), others element by element.  The tokens are counted off by 32 from where the call's first slot
// says, so that one sequence's tokens fall into blocks; where a call holds several, those after the first
// do as a rule not.  65536 tokens of 8 int8 heads of 128 in one sequence and in 16: in 119 and 182 us, back 85 and
// 224; 16-bit rows in 129 and 249, back 94 and 222 (a call to a sequence has each fall into blocks).
#include <algorithm>

#include "kvcache.h"
#include "lanes.h"

namespace mxmoe {
namespace {

// The row's factor of the norm: 1 / sqrt(mean + eps) in 64 bits, by an approximate root and one step
// of Newton's (relative error below 2^-40), rounded to fp32.
template <int D> LANES_INL float norm_factor(const float (&v)[8], double eps) {
  double ss = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) ss = __builtin_fma((double)v[i], (double)v[i], ss);
  const double m = __builtin_fma(lanes_sum<D / 8>(ss), 1.0 / D, eps);
  double r = __builtin_amdgcn_rsq(m);
  const double e = __builtin_fma(-m * r, r, 1.0);
  r = __builtin_fma(0.5 * r, e, r);
  // (the step turns the root of inf, 0, into NaN)
  return m < __builtin_inf() ? (float)r : m != m ? __builtin_nanf("") : 0.f;
}

// Codes and scale of a head's row that dim / 8 lanes hold
struct Coded { u32x2 q; float scale; };
template <int D> LANES_INL Coded encode(const float (&v)[8], int qmax) {
  uint32_t mb = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) mb = max(mb, __float_as_uint(v[i]) & 0x7fffffffu);
  mb = lanes_umax<D / 8>(mb);
  const float amax = __uint_as_float(mb), qm = (float)qmax;
  Coded c = {{0u, 0u}, 0.f};
  if (mb >= 0x7f800000u) {
    c.scale = __builtin_nanf("");
  } else if (amax >= kTinyAmax) {
    const float inv = __fdiv_rn(qm, amax);
    const bool f8 = qmax == kQmaxF8;
    c.scale = __fdiv_rn(amax, qm);
    c.q = u32x2{codes4(v[0], v[1], v[2], v[3], inv, f8), codes4(v[4], v[5], v[6], v[7], inv, f8)};
  }
  return c;
}
template <int ACT> LANES_INL u32x4 rounded(const float (&v)[8]) {
  return u32x4{pack2<ACT>(v[0], v[1]), pack2<ACT>(v[2], v[3]), pack2<ACT>(v[4], v[5]), pack2<ACT>(v[6], v[7])};
}
template <int ACT> LANES_INL void widened(u32x4 w, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 a = unpack2<ACT>(w[i]);
    v[2 * i] = a[0];
    v[2 * i + 1] = a[1];
  }
}
LANES_INL u32x4 row_piece(const void* p, int64_t at) { return *reinterpret_cast<const u32x4_any*>(reinterpret_cast<const uint16_t*>(p) + at); }

// The slots of 32 tokens of a call from t0 on (of those that there are): the first slot of the block of the
// cache that they are side by side in, each at its place, or -1.  Every wavefront finds out for itself.
LANES_INL int block_of(const int32_t* slots, int t0, int tokens, int n_slots) {
  const int l = threadIdx.x & 31, t = t0 + l;
  const bool live = t >= 0 && t < tokens;
  const int at = live ? slots[t] - l : 0;
  const uint64_t all = __ballot(live);
  const int base = __builtin_amdgcn_readlane(at, __builtin_ctzll(all));  // (t0 < tokens: there is one)
  return base >= 0 && base < n_slots && base % 32 == 0 && __ballot(live && at != base) == 0 ? base : -1;
}

// Pieces of values in LDS: 256 bytes of (dim tile, q), 16 bytes further apart than in the cache, so that
// lanes that read different tiles meet different banks.
constexpr int kTile = 256 + 16;
template <int ES> LANES_INL int lds_at(int t, int d) {
  const int q = (t >> 2) & 3, j = (t & 3) + ((t >> 4) & 1) * 4;
  if (ES == 2) return ((d >> 4) * 4 + q) * kTile + (d & 15) * 16 + 2 * j;
  return ((d >> 5) * 4 + q) * kTile + (d & 15) * 16 + ((d >> 4) & 1) * 8 + j;
}

// 32 tokens' values of one head into the cache
template <int D, int ES, int ACT> LANES_INL void append_values(const KvAppendArgs& a, int t0, int h, uint8_t* lds) {
  constexpr int GL = D / 8, RP = 256 / GL;
  const int tid = threadIdx.x, c = tid % GL;
  const int first = block_of(a.slots, t0, a.tokens, a.n_slots);
  const int page = (1 << a.page_log2) - 1;
  const int64_t rec0 = first < 0 ? 0 : ((int64_t)(first >> a.page_log2) * a.kv_heads + h) << a.page_log2;
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += RP) {
    const int i = r0 + tid / GL, t = t0 + i;
    const bool live = i < 32 && t >= 0 && t < a.tokens;
    const u32x4 w = live ? row_piece(a.v, t * a.ldv + h * D + 8 * c) : u32x4{0u, 0u, 0u, 0u};
    const int slot = live ? a.slots[t] : -1;
    const bool keep = slot >= 0 && slot < a.n_slots;
    const int64_t rec = keep ? ((int64_t)(slot >> a.page_log2) * a.kv_heads + h) << a.page_log2 : 0;
    uint8_t* to = first >= 0 ? lds : reinterpret_cast<uint8_t*>(a.cv) + rec * (D * ES);
    auto place = [&](int e) { return first >= 0 ? lds_at<ES>(i, 8 * c + e) : value_at<ES>(slot & page, 8 * c + e, D); };
    if constexpr (ES == 1) {
      float v[8];
      widened<ACT>(w, v);
      const Coded q = encode<D>(v, a.qmax);
      if (keep) {
        if (c == 0) a.cvs[rec + (slot & page)] = q.scale;
#pragma unroll
        for (int e = 0; e < 8; ++e) to[place(e)] = (uint8_t)(q.q[e >> 2] >> (8 * (e & 3)));
      }
    } else if (keep) {
#pragma unroll
      for (int e = 0; e < 8; ++e) *reinterpret_cast<uint16_t*>(to + place(e)) = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
  }
  if (first < 0) return;
  __syncthreads();
  uint8_t* base = reinterpret_cast<uint8_t*>(a.cv) + (rec0 + (first & page)) * (D * ES);
  const int lo = max(0, -t0), hi = min(32, a.tokens - t0);  // tokens of the block that are the call's
  for (int o = tid; o < 2 * D * ES; o += 256) {
    const uint8_t* piece = lds + (o >> 4) * kTile + (o & 15) * 16;
    uint8_t* to = base + 16 * o;
    if (lo == 0 && hi == 32) {
      *reinterpret_cast<u32x4*>(to) = *reinterpret_cast<const u32x4*>(piece);
      continue;
    }
    const int q = (o >> 4) & 3;
#pragma unroll
    for (int g = 0; g < 4; ++g) {  // 4 bytes: 2 or 4 tokens of an element
      const int t = 4 * q + (ES == 2 ? 2 * (g & 1) + 16 * (g >> 1) : 16 * (g & 1));
      if (t >= lo && t + 4 / ES <= hi) {
        *reinterpret_cast<uint32_t*>(to + 4 * g) = *reinterpret_cast<const uint32_t*>(piece + 4 * g);
      } else {
#pragma unroll
        for (int e = 0; e < 4 / ES; ++e)
          if (t + e >= lo && t + e < hi) {
            if (ES == 2) *reinterpret_cast<uint16_t*>(to + 4 * g + 2 * e) = *reinterpret_cast<const uint16_t*>(piece + 4 * g + 2 * e);
            else to[4 * g + e] = piece[4 * g + e];
          }
      }
    }
  }
}

// The first `value_jobs` workgroups take 32 tokens' values of one head each.  The others take `tb`
// tokens and every `parts`-th set of heads of a token's q | k (and v, where values have no jobs of
// their own): the groups of dim / 8 lanes share the tokens and take heads in turn, the next
// row on its way meanwhile.  The rotations' cosines and sines go through LDS, one pair of a
// token to a thread, into the registers of the lanes that need them for all heads.
// Bound by memory where there are many tokens: 28 + 2 x 4 heads of 128 of 16384 tokens, bf16 in, int8 out,
// 68.2 us, 4.9 TB/s (a copy of as much: 5.15); by its launch and three memory latencies (slot and row,
// positions and frequencies, weights) where there are few: one token 3.7 us.
template <int D, int ACT>
__global__ void __launch_bounds__(256) kv_append_kernel(KvAppendArgs a) {
  constexpr int GL = D / 8, RP = 256 / GL;
  __shared__ __attribute__((aligned(16))) uint8_t lds[D / 4 * kTile > RP * D / 2 * 8 ? D / 4 * kTile : RP * D / 2 * 8];
  if ((int)blockIdx.x < a.value_jobs) {
    // (blocks begin where the first token's slot says, so that the tokens of one sequence fall into them)
    const int job = (int)blockIdx.x / a.kv_heads, h = (int)blockIdx.x - job * a.kv_heads;
    const int t0 = 32 * job - (a.slots[0] & 31);
    if (t0 >= a.tokens) return;
    if (a.qmax) append_values<D, 1, ACT>(a, t0, h, lds);
    else append_values<D, 2, ACT>(a, t0, h, lds);
    return;
  }
  float2* turn = reinterpret_cast<float2*>(lds);  // [tb][rot / 2]
  const int tid = threadIdx.x, c = tid % GL, half = a.rot / 2, job = (int)blockIdx.x - a.value_jobs;
  const int part = job % a.parts, t0 = job / a.parts * a.tb;
  const int per = RP / a.tb, tl = tid / GL / per, t = t0 + tl;  // groups to a token, this group's token
  const bool live = t < a.tokens;
  const int step = per * a.parts;
  int h = part * per + tid / GL % per;
  auto row_of = [&](int h) {
    return h < a.q_heads ? row_piece(a.q, t * a.ldq + h * D + 8 * c)
           : h < a.q_heads + a.kv_heads ? row_piece(a.k, t * a.ldk + (h - a.q_heads) * D + 8 * c)
                                        : row_piece(a.v, t * a.ldv + (h - a.q_heads - a.kv_heads) * D + 8 * c);
  };
  u32x4 next = live && h < a.heads ? row_of(h) : u32x4{0u, 0u, 0u, 0u};
  const int slot = live ? a.slots[t] : -1;
  // Row element i, times the row's factor, becomes x own[i] + partner turned[i]: weight times cosine,
  // partner's weight times sine (with its sign), of queries first, of keys when they come.  (The factor
  // first: a large row's products with its weight may pass the largest value.)
  float own[8], turned[8];
  int kind = -1;
  const int hc = a.rot / 16;
  const bool in = 8 * c < a.rot, low = c < hc;
  const int pc = !in || a.interleaved ? c : low ? c + hc : c - hc;
  u32x4 weights[2][2] = {};  // (asked for before the angles)
  if (a.q_weight) {
    weights[0][0] = row_piece(a.q_weight, 8 * c);
    weights[0][1] = row_piece(a.q_weight, 8 * pc);
  }
  if (a.k_weight) {
    weights[1][0] = row_piece(a.k_weight, 8 * c);
    weights[1][1] = row_piece(a.k_weight, 8 * pc);
  }
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    cs[i] = 1.f;
    sn[i] = 0.f;
  }
  if (a.rot) {
    for (int i = tid; i < a.tb * half; i += 256) {
      const int k = i / half, p = i - k * half;
      if (t0 + k < a.tokens) {
        const double turns = (double)a.positions[t0 + k] * a.freqs[p] * 0.15915494309189533577;
        float s1, c1;
        sincospif(2.f * (float)(turns - rint(turns)), &s1, &c1);
        turn[i] = make_float2(c1, s1);
      }
    }
    __syncthreads();
    if (in) {
      const float2* z = turn + tl * half + (a.interleaved ? 4 * c : 8 * (low ? c : c - hc));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 w = z[a.interleaved ? i >> 1 : i];
        cs[i] = w.x;
        sn[i] = (a.interleaved ? (i & 1) == 0 : low) ? -w.y : w.y;
      }
    }
  }
  const int other = (tid & 63) - c + pc;
  const bool keep = slot >= 0 && slot < a.n_slots;
  const int page = (1 << a.page_log2) - 1, at = slot & page;
  // (all groups go round as often: the cross-lane moves take whole wavefronts)
  for (int h0 = part * per; h0 < a.heads; h0 += step, h += step) {
    const bool here = live && h < a.heads;
    const u32x4 w = next;
    if (live && h + step < a.heads) next = row_of(h + step);
    const int what = h < a.q_heads ? 0 : h < a.q_heads + a.kv_heads ? 1 : 2;
    float v[8];
    widened<ACT>(w, v);
    if (what < 2 && what != kind) {
      kind = what;
      float g[8], o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = o[i] = 1.f;
      if (what ? a.k_weight : a.q_weight) {
        widened<ACT>(what ? weights[1][0] : weights[0][0], g);
        widened<ACT>(what ? weights[1][1] : weights[0][1], o);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        own[i] = g[i] * cs[i];
        turned[i] = (a.interleaved ? o[i ^ 1] : o[i]) * sn[i];
      }
    }
    const bool norm = (what == 0 && a.q_weight) || (what == 1 && a.k_weight);
    const float f = norm ? norm_factor<D>(v, a.eps) : 1.f;
    float o[8];
    if (a.rot) {
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = v[i ^ 1];
      } else {
        u32x4 pw;
#pragma unroll
        for (int i = 0; i < 4; ++i) pw[i] = (uint32_t)__shfl((int)w[i], other, 64);
        widened<ACT>(pw, o);
      }
    }
    if (what < 2 && (norm || a.rot)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = v[i] * f * own[i];
        v[i] = in ? __builtin_fmaf(o[i] * f, turned[i], y) : y;
      }
    }
    if (what == 0) {
      if (here) *reinterpret_cast<u32x4_any*>(reinterpret_cast<uint16_t*>(a.q_out) + t * a.ldo + h * D + 8 * c) = rounded<ACT>(v);
      continue;
    }
    const int hk = h - a.q_heads - (what == 2 ? a.kv_heads : 0);
    const int64_t rec = (int64_t)((keep ? slot >> a.page_log2 : 0) * (int64_t)a.kv_heads + hk) << a.page_log2;
    if (a.qmax) {
      const Coded q = encode<D>(v, a.qmax);
      if (here && keep) {
        uint8_t* base = reinterpret_cast<uint8_t*>(what == 1 ? a.ck : a.cv) + rec * D;
        if (c == 0) (what == 1 ? a.cks : a.cvs)[rec + at] = q.scale;
        if (what == 1) {
          *reinterpret_cast<u32x2*>(base + key_at<1>(at, c, D)) = q.q;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) base[value_at<1>(at, 8 * c + e, D)] = (uint8_t)(q.q[e >> 2] >> (8 * (e & 3)));
        }
      }
    } else if (here && keep) {
      uint8_t* base = reinterpret_cast<uint8_t*>(what == 1 ? a.ck : a.cv) + rec * (2 * D);
      if (what == 1) {
        *reinterpret_cast<u32x4*>(base + key_at<2>(at, c, D)) = rounded<ACT>(v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) *reinterpret_cast<uint16_t*>(base + value_at<2>(at, 8 * c + e, D)) = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}

LANES_INL void decoded(u32x2 q, float s, int qmax, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = q[i >> 2] >> (8 * (i & 3)) & 0xffu;
    v[i] = (qmax == kQmaxF8 ? __builtin_amdgcn_cvt_f32_fp8((int)b, 0) : (float)(int8_t)b) * s;
  }
}

// Rows at slots back in 16 bits.  32 tokens' keys or values of one head to a workgroup: whole pieces
// where their slots are one block, else piece by piece and element by element.  65536 tokens of 8 int8
// heads of 128: 85-89 us, 4.6-4.8 TB/s (copy 5.15; 177 without LDS), bf16 94, 5.7; 1237 of one bf16 head of 256, 80 workgroups, 4.3 us: latency.
template <int D, int ES, int ACT>
__global__ void __launch_bounds__(256) kv_read_kernel(KvReadArgs a) {
  constexpr int GL = D / 8, RP = 256 / GL, kRow = D * ES + 16;  // (rows of keys 16 bytes apart)
  __shared__ __attribute__((aligned(16))) uint8_t lds[D * ES / 8 * kTile > 32 * kRow ? D * ES / 8 * kTile : 32 * kRow];
  const int tid = threadIdx.x, c = tid % GL;
  const int job = (int)blockIdx.x / (2 * a.kv_heads), row = (int)blockIdx.x - job * (2 * a.kv_heads);
  const bool what = row >= a.kv_heads;
  const int h = row - (what ? a.kv_heads : 0);
  const int t0 = 32 * job - (a.slots[0] & 31);
  if (t0 >= a.tokens) return;
  const int first = block_of(a.slots, t0, a.tokens, a.n_slots);
  const int page = (1 << a.page_log2) - 1;
  const uint8_t* from = reinterpret_cast<const uint8_t*>(what ? a.cv : a.ck);
  const float* scales = what ? a.cvs : a.cks;
  uint16_t* to = reinterpret_cast<uint16_t*>(what ? a.v : a.k);
  if (first >= 0) {
    const int64_t rec = (((int64_t)(first >> a.page_log2) * a.kv_heads + h) << a.page_log2) + (first & page);
    const uint8_t* base = from + rec * (D * ES);
    constexpr int N = (2 * D * ES + 255) / 256;  // 16-byte pieces to a thread
    u32x4 w[N];
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (tid + 256 * j < 2 * D * ES) w[j] = *reinterpret_cast<const u32x4*>(base + 16 * (tid + 256 * j));
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int o = tid + 256 * j;
      // (a key's piece: token o % 16 of tile o / (16 pieces a row))
      const int at = what ? (o >> 4) * kTile + (o & 15) * 16 : ((o & 15) + 16 * (o / (D * ES))) * kRow + o % (D * ES) / 16 * 16;
      if (o < 2 * D * ES) *reinterpret_cast<u32x4*>(lds + at) = w[j];
    }
    __syncthreads();
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += RP) {
      const int i = r0 + tid / GL;
      if (i >= 32 || t0 + i < 0 || t0 + i >= a.tokens) continue;
      uint16_t* out = to + ((int64_t)(t0 + i) * a.kv_heads + h) * D + 8 * c;
      if constexpr (ES == 2) {
        u32x4 v;
        if (!what) {
          v = *reinterpret_cast<const u32x4*>(lds + i * kRow + 16 * c);
        } else {
          uint32_t e[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] = *reinterpret_cast<const uint16_t*>(lds + lds_at<2>(i, 8 * c + j));
          v = u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
        }
        *reinterpret_cast<u32x4_any*>(out) = v;
      } else {
        u32x2 q;
        if (!what) {
          q = *reinterpret_cast<const u32x2*>(lds + i * kRow + 8 * c);
        } else {
          uint32_t e[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] = lds[lds_at<1>(i, 8 * c + j)];
          q = u32x2{e[0] | e[1] << 8 | e[2] << 16 | e[3] << 24, e[4] | e[5] << 8 | e[6] << 16 | e[7] << 24};
        }
        float f[8];
        decoded(q, scales[rec + i], a.qmax, f);
        *reinterpret_cast<u32x4_any*>(out) = rounded<ACT>(f);
      }
    }
    return;
  }
  for (int i = tid / GL; i < 32; i += RP) {
    const int t = t0 + i;
    if (t < 0 || t >= a.tokens) continue;
    const int slot = a.slots[t];
    uint16_t* out = to + ((int64_t)t * a.kv_heads + h) * D + 8 * c;
    if (slot < 0 || slot >= a.n_slots) {
      *reinterpret_cast<u32x4_any*>(out) = u32x4{0u, 0u, 0u, 0u};
      continue;
    }
    const int64_t rec = ((int64_t)(slot >> a.page_log2) * a.kv_heads + h) << a.page_log2;
    const int at = slot & page;
    const uint8_t* base = from + rec * (D * ES);
    if constexpr (ES == 1) {
      u32x2 q;
      if (!what) {
        q = *reinterpret_cast<const u32x2*>(base + key_at<1>(at, c, D));
      } else {
        uint32_t e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = base[value_at<1>(at, 8 * c + j, D)];
        q = u32x2{e[0] | e[1] << 8 | e[2] << 16 | e[3] << 24, e[4] | e[5] << 8 | e[6] << 16 | e[7] << 24};
      }
      float f[8];
      decoded(q, scales[rec + at], a.qmax, f);
      *reinterpret_cast<u32x4_any*>(out) = rounded<ACT>(f);
    } else if (!what) {
      *reinterpret_cast<u32x4_any*>(out) = *reinterpret_cast<const u32x4*>(base + key_at<2>(at, c, D));
    } else {
      uint32_t e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = *reinterpret_cast<const uint16_t*>(base + value_at<2>(at, 8 * c + j, D));
      *reinterpret_cast<u32x4_any*>(out) = u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
    }
  }
}

template <int D, int ACT> hipError_t go_append(KvAppendArgs a, hipStream_t s) {
  constexpr int RP = 2048 / D;
  // 32 tokens and more: values by blocks (us of a run of 256 slots, 4 heads of 128, int8: 4.8, without
  // 6.9; 16384: 68, 73; below, a call is its launch, and 31 slots of dim 256 would take 5.3 for 3.9)
  const int blocks = a.tokens >= 32 ? (a.tokens + 31) / 32 + 1 : 0;  // (they may begin anywhere in one)
  a.value_jobs = blocks * a.kv_heads;
  a.heads = a.q_heads + (blocks ? 1 : 2) * a.kv_heads;
  // tokens to a workgroup: more of them share angles and weights, fewer fill the CUs.  us with 1, 4, 8, 16 (28 + 4 heads
  // of 128, int8): 16 tokens 3.9, 4.2, 4.5, 5.0, 1024 10.4, 8.6, 9.1, 9.8, 8192 -, 37.3, 33.2, 45.1, 16384 102, 72.4, 67.7, 68.2; 262144
  // tokens of 4 keys and values alone -, -, 293, 264; 16384 of dim 64 -, 43.7, 37.4, 33.8
  a.tb = a.tokens >= 16384 ? std::min(RP, 16) : a.tokens >= 8192 ? 8 : a.tokens >= 32 ? 4 : 1;
  const int teams = (a.tokens + a.tb - 1) / a.tb, per = RP / a.tb;
  const int most = (a.heads + per - 1) / per, want = (512 + teams - 1) / teams;
  a.parts = want < most ? want : most;
  const int64_t grid = a.value_jobs + (int64_t)teams * a.parts;
  hipLaunchKernelGGL((kv_append_kernel<D, ACT>), dim3((unsigned)grid), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <int D, int ACT> hipError_t go_read(const KvReadArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(((a.tokens + 31) / 32 + 1) * 2 * a.kv_heads));
  if (a.qmax) hipLaunchKernelGGL((kv_read_kernel<D, 1, ACT>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv_read_kernel<D, 2, ACT>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(const KvAppendArgs& a, int dim, hipStream_t s) {
  if (a.act == MXMOE_BF16)
    return dim == 64 ? go_append<64, MXMOE_BF16>(a, s) : dim == 128 ? go_append<128, MXMOE_BF16>(a, s) : go_append<256, MXMOE_BF16>(a, s);
  return dim == 64 ? go_append<64, MXMOE_F16>(a, s) : dim == 128 ? go_append<128, MXMOE_F16>(a, s) : go_append<256, MXMOE_F16>(a, s);
}
hipError_t launch_kv_read(const KvReadArgs& a, int dim, hipStream_t s) {
  if (a.act == MXMOE_BF16)
    return dim == 64 ? go_read<64, MXMOE_BF16>(a, s) : dim == 128 ? go_read<128, MXMOE_BF16>(a, s) : go_read<256, MXMOE_BF16>(a, s);
  return dim == 64 ? go_read<64, MXMOE_F16>(a, s) : dim == 128 ? go_read<128, MXMOE_F16>(a, s) : go_read<256, MXMOE_F16>(a, s);
}

}  // namespace mxmoe
