// Heads of new tokens into the paged cache (norm, rotation, 8-bit codes in one pass),
// and rows of the cache back.
//
//   y = x r w,  r = 1 / sqrt(mean x^2 + eps)       (64-bit sum and root; queries and keys)
//   (a, b) -> (a cos - b sin, b cos + a sin)        angle = position * frequency, in 64 bits
//   codes, scale: the per-token recipe of rowquant.h on the fp32 values of a head's row
//
// dim / 8 lanes hold a head's row, 8 elements each.
#include "kvcache.h"
#include "lanes.h"

namespace mxmoe {
namespace {

LANES_INL void store_act(uint16_t* p, const float (&v)[8], int act) {
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = act == MXMOE_BF16 ? pack2<MXMOE_BF16>(v[2 * i], v[2 * i + 1]) : pack2<MXMOE_F16>(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<u32x4_any*>(p) = o;
}
LANES_INL void load_act(const uint16_t* p, float (&v)[8], int act) {
  const u32x4 w = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 a = act == MXMOE_BF16 ? unpack2<MXMOE_BF16>(w[i]) : unpack2<MXMOE_F16>(w[i]);
    v[2 * i] = a[0];
    v[2 * i + 1] = a[1];
  }
}

// A workgroup takes `tb` tokens and the heads hs .. he of a token's q | k | v heads.  The
// rotations' cosines and sines of its tokens are in LDS, one pair of a token to a thread.
template <int D>
__global__ void __launch_bounds__(256) kv_append_kernel(KvAppendArgs a) {
  constexpr int GL = D / 8, RP = 256 / GL;
  extern __shared__ float2 turn[];  // [tb][rot / 2]
  const int tid = threadIdx.x, c = tid % GL, half = a.rot / 2;
  const int t0 = (int)blockIdx.x * a.tb, nt = min(a.tb, a.tokens - t0);
  for (int i = tid; i < nt * half; i += 256) {
    const int t = i / half, p = i - t * half;
    const double turns = (double)a.positions[t0 + t] * a.freqs[p] * 0.15915494309189533577;
    const float f = 2.f * (float)(turns - rint(turns));
    float sn, cs;
    sincospif(f, &sn, &cs);
    turn[i] = make_float2(cs, sn);
  }
  __syncthreads();
  const int per = (a.heads + (int)gridDim.y - 1) / (int)gridDim.y;
  const int h0 = (int)blockIdx.y * per, nh = min(per, a.heads - h0);
  const int rows = nt * nh;
  for (int r0 = 0; r0 < rows; r0 += RP) {
    const int r = r0 + tid / GL;
    const bool live = r < rows;  // (lanes of no row go along: the cross-lane moves take whole groups)
    const int tl = live ? r / nh : 0, h = h0 + (live ? r - tl * nh : 0), t = t0 + tl;
    const int what = h < a.q_heads ? 0 : h < a.q_heads + a.kv_heads ? 1 : 2;
    const int hk = h - a.q_heads - (what == 2 ? a.kv_heads : 0);
    const uint16_t* src = what == 0 ? reinterpret_cast<const uint16_t*>(a.q) + t * a.ldq + h * D
                        : reinterpret_cast<const uint16_t*>(what == 1 ? a.k : a.v) + t * (what == 1 ? a.ldk : a.ldv) + hk * D;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (live) load_act(src + 8 * c, v, a.act);
    const void* w = what == 0 ? a.q_weight : what == 1 ? a.k_weight : nullptr;
    if (w) {
      float g[8];
      load_act(reinterpret_cast<const uint16_t*>(w) + 8 * c, g, a.act);
      double ss = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fma((double)v[i], (double)v[i], ss);
      ss = lanes_sum<GL>(ss);
      const float f = (float)(1.0 / __builtin_sqrt(ss / D + a.eps));
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = v[i] * f * g[i];
    }
    if (a.rot) {  // (q, k and v rows may share a wavefront: every lane moves, v keeps its own)
      const float2* cs = turn + tl * half;
      if (a.interleaved) {
        if (what < 2 && 8 * c < a.rot) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 z = cs[4 * c + i];
            const float x = v[2 * i], y = v[2 * i + 1];
            v[2 * i] = x * z.x - y * z.y;
            v[2 * i + 1] = y * z.x + x * z.y;
          }
        }
      } else {
        const int hc = a.rot / 16;
        const bool first = c < hc, in = c < 2 * hc;
        const int other = (int)(threadIdx.x & 63) + (in ? (first ? hc : -hc) : 0);
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = __shfl(v[i], other, 64);
        if (what < 2 && in) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float2 z = cs[8 * (first ? c : c - hc) + i];
            v[i] = first ? v[i] * z.x - o[i] * z.y : v[i] * z.x + o[i] * z.y;
          }
        }
      }
    }
    if (what == 0) {
      if (live) store_act(reinterpret_cast<uint16_t*>(a.q_out) + t * a.ldo + h * D + 8 * c, v, a.act);
    }
    const int slot = live && what ? a.slots[t] : -1;
    const bool keep = slot >= 0 && slot < a.n_slots;
    const int64_t rec = (int64_t)(keep ? slot >> a.page_log2 : 0) * a.kv_heads + (what ? hk : 0);
    const int at = keep ? slot & ((1 << a.page_log2) - 1) : 0;
    if (a.qmax) {
      uint32_t mb = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) mb = max(mb, __float_as_uint(v[i]) & 0x7fffffffu);
      mb = lanes_umax<GL>(mb);
      const float amax = __uint_as_float(mb), qm = (float)a.qmax;
      float inv = 0.f, scale = 0.f;
      if (mb >= 0x7f800000u) {
        scale = __builtin_nanf("");
      } else if (amax >= kTinyAmax) {
        inv = __fdiv_rn(qm, amax);
        scale = __fdiv_rn(amax, qm);
      }
      if (keep) {
        const bool f8 = a.qmax == kQmaxF8;
        u32x2 q = {0u, 0u};
        if (inv > 0.f) q = u32x2{codes4(v[0], v[1], v[2], v[3], inv, f8), codes4(v[4], v[5], v[6], v[7], inv, f8)};
        uint8_t* base = reinterpret_cast<uint8_t*>(what == 1 ? a.ck : a.cv) + (rec << a.page_log2) * D;
        float* sc = (what == 1 ? a.cks : a.cvs) + (rec << a.page_log2) + at;
        if (c == 0) *sc = scale;
        if (what == 1) {
          *reinterpret_cast<u32x2*>(base + key_at<1>(at, c, D)) = q;
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) base[value_at<1>(at, 8 * c + i, D)] = (uint8_t)(q[i >> 2] >> (8 * (i & 3)));
        }
      }
    } else if (keep) {
      uint8_t* base = reinterpret_cast<uint8_t*>(what == 1 ? a.ck : a.cv) + (rec << a.page_log2) * (2 * D);
      uint16_t o[8];
      store_act(o, v, a.act);
      if (what == 1) {
        *reinterpret_cast<u32x4*>(base + key_at<2>(at, c, D)) = *reinterpret_cast<const u32x4_any*>(o);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) *reinterpret_cast<uint16_t*>(base + value_at<2>(at, 8 * c + i, D)) = o[i];
      }
    }
  }
}

// Rows at slots back in 16 bits: a row of one head (keys, then values) to dim / 8 lanes.
template <int D>
__global__ void __launch_bounds__(256) kv_read_kernel(KvReadArgs a) {
  constexpr int GL = D / 8, RP = 256 / GL;
  const int c = threadIdx.x % GL;
  const int64_t rows = (int64_t)a.tokens * a.kv_heads * 2;
  for (int64_t r = (int64_t)blockIdx.x * RP + threadIdx.x / GL; r < rows; r += (int64_t)gridDim.x * RP) {
    const int64_t t = r / (2 * a.kv_heads);
    const int j = (int)(r - t * (2 * a.kv_heads)), what = j >= a.kv_heads, h = j - (what ? a.kv_heads : 0);
    const int slot = a.slots[t];
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    uint16_t* out = reinterpret_cast<uint16_t*>(what ? a.v : a.k) + (t * a.kv_heads + h) * D + 8 * c;
    if (slot < 0 || slot >= a.n_slots) {
      store_act(out, v, a.act);
      continue;
    }
    const int64_t rec = (int64_t)(slot >> a.page_log2) * a.kv_heads + h;
    const int at = slot & ((1 << a.page_log2) - 1);
    if (a.qmax) {
      const uint8_t* base = reinterpret_cast<const uint8_t*>(what ? a.cv : a.ck) + (rec << a.page_log2) * D;
      const float s = (what ? a.cvs : a.cks)[(rec << a.page_log2) + at];
      uint8_t q[8];
      if (!what) {
        *reinterpret_cast<u32x2_any*>(q) = *reinterpret_cast<const u32x2*>(base + key_at<1>(at, c, D));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = base[value_at<1>(at, 8 * c + i, D)];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v[i] = (a.qmax == kQmaxF8 ? __builtin_amdgcn_cvt_f32_fp8((int)q[i], 0) : (float)(int8_t)q[i]) * s;
      store_act(out, v, a.act);
    } else {
      const uint8_t* base = reinterpret_cast<const uint8_t*>(what ? a.cv : a.ck) + (rec << a.page_log2) * (2 * D);
      if (!what) {
        *reinterpret_cast<u32x4_any*>(out) = *reinterpret_cast<const u32x4*>(base + key_at<2>(at, c, D));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = *reinterpret_cast<const uint16_t*>(base + value_at<2>(at, 8 * c + i, D));
      }
    }
  }
}

}  // namespace

hipError_t launch_kv_append(KvAppendArgs a, int dim, hipStream_t s) {
  a.heads = a.q_heads + 2 * a.kv_heads;
  a.tb = 4;
  const dim3 grid((a.tokens + a.tb - 1) / a.tb, a.tokens <= 256 ? (a.heads * dim / 8 + 255) / 256 : 1);
  const size_t lds = sizeof(float2) * a.tb * (a.rot / 2);
  switch (dim) {
    case 64: hipLaunchKernelGGL(kv_append_kernel<64>, grid, dim3(256), lds, s, a); break;
    case 128: hipLaunchKernelGGL(kv_append_kernel<128>, grid, dim3(256), lds, s, a); break;
    default: hipLaunchKernelGGL(kv_append_kernel<256>, grid, dim3(256), lds, s, a); break;
  }
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvReadArgs& a, int dim, hipStream_t s) {
  const int64_t rows = (int64_t)a.tokens * a.kv_heads * 2, rp = 2048 / dim, grid = (rows + rp - 1) / rp;
  const dim3 g((unsigned)(grid < (1 << 20) ? grid : 1 << 20));
  switch (dim) {
    case 64: hipLaunchKernelGGL(kv_read_kernel<64>, g, dim3(256), 0, s, a); break;
    case 128: hipLaunchKernelGGL(kv_read_kernel<128>, g, dim3(256), 0, s, a); break;
    default: hipLaunchKernelGGL(kv_read_kernel<256>, g, dim3(256), 0, s, a); break;
  }
  return hipGetLastError();
}

}  // namespace mxmoe
