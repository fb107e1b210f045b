// Balance loss of the router, with per-expert counts, mean probabilities and the
// gradient of the logits.  Over the n tokens that the mask keeps:
//   c_e = number of (token, slot) pairs with expert e,  f_e = c_e / (k n)
//   P_e = 1/n sum_t p[t,e],  p[t] = softmax of the token's logits
//   L = alpha E sum_e f_e P_e
//   dL/dlogits[t,e] = alpha E / n * p[t,e] (f_e - sum_j f_j p[t,j])
// The counts are constants of the gradient (a choice of experts has none), so a token's
// gradient needs all counts and its own logits.  Two launches: the first counts and sums
// the probabilities, the second writes the gradient, and its first workgroup adds the
// shares of the first in their order, to counts, mean probabilities and loss.  Where shares times
// experts are many, a launch between them folds the shares into one.  The logits are
// read twice, the second time from the caches: with one pass over them and a launch for
// the counts before it and one for the shares behind it, 65536 x 64 took 20.9 us and
// 4096 x 60 12.9, and a workgroup that finishes last adding the shares waits for the L2s to
// be written back (29 us).  Small batches take one workgroup and one launch.
//
// A token is held by LT lanes, V consecutive logits to a lane and chunk, so that a
// wavefront reads 64 / LT tokens side by side; sums over a token are butterflies
// over its lanes.
//
// Sums over tokens are 64-bit in a lane and wherever they are added up, so that their error
// does not grow with the batch.  They are kept as fp32 in between, a wavefront's in LDS, a
// workgroup's share in the workspace and the folded one: each rounds a sum of positive terms
// once, within 2^-24 of it, and halves what the last launch reads (summed in fp32 throughout,
// 2^22 like tokens of 8 experts came out 19 x 2^-24 off).
#include <algorithm>
#include "mxmoe_internal.h"

namespace mxmoe {
namespace {

#define BAL_INL __device__ __attribute__((always_inline)) inline

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_any __attribute__((aligned(4)));

constexpr int kThreads = 512;

template <int C> BAL_INL float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), C, 0xf, 0xf, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;
template <int L, typename F> BAL_INL float lanes(float v, F f) {
  if constexpr (L > 1) v = f(v, dpp<kXor1>(v));
  if constexpr (L > 2) v = f(v, dpp<kXor2>(v));
  if constexpr (L > 4) v = f(v, dpp<kHalfMirror>(v));
  if constexpr (L > 8) v = f(v, dpp<kMirror>(v));
  if constexpr (L > 16) v = f(v, __shfl_xor(v, 16, 64));
  if constexpr (L > 32) v = f(v, __shfl_xor(v, 32, 64));
  return v;
}
template <int L> BAL_INL float lanes_sum(float v) { return lanes<L>(v, [](float a, float b) { return a + b; }); }
template <int L> BAL_INL float lanes_max(float v) { return lanes<L>(v, [](float a, float b) { return fmaxf(a, b); }); }
// exp(d) for d <= 0 within 2 units in the last place where it is a normal number, and 0
// below (d < -87.3): 2^(d log2 e) with the rounding error of the product put back (the
// library's expf takes three times the instructions; with it and a quotient a
// probability, one workgroup took 14.4 us for 512 tokens of 64 experts)
BAL_INL float exp_diff(float d) {
  constexpr float kL2e = 1.44269504f, kL2eLow = 1.92596303e-8f, kLn2 = 0.693147181f;
  d = d < -104.f ? -104.f : d;  // 0 from here on, and -inf makes no NaN below (a NaN stays)
  const float hi = d * kL2e, lo = fmaf(d, kL2e, -hi) + d * kL2eLow;
  const float x = __builtin_amdgcn_exp2f(hi);
  return fmaf(x, lo * kLn2, x);
}

// Logits of a token in a lane: chunk j holds experts V (LT j + l) .. + V - 1 (V = 1: LT j + l).
template <int LT, int V, int J> struct Tok {
  float v[J][V] = {};
  BAL_INL static int expert(int l, int j) { return V * (LT * j + l); }
  // (V = 4: E >= 4; the chunk that E ends in is read from E - 4 on and moved into place, so
  // that every lane has one load to a chunk)
  BAL_INL void load(const float* row, int l, int E) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int e = expert(l, j);
      if constexpr (V == 1) {
        v[j][0] = e < E ? row[e] : -INFINITY;
      } else {
        const int at = min(e, E - 4), d = e - at;
        const f32x4 x = *reinterpret_cast<const f32x4_any*>(row + at);
        if ((E & 3) == 0) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[j][i] = d == 0 ? x[i] : -INFINITY;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float y = -INFINITY;
#pragma unroll
            for (int q = 3; q >= i; --q) y = d == q - i ? x[q] : y;
            v[j][i] = y;
          }
        }
      }
    }
  }
  BAL_INL void store(float* row, int l, int E) const {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int e = expert(l, j);
      if constexpr (V == 1) {
        if (e < E) row[e] = v[j][0];
      } else {
        if (e + 4 <= E) *reinterpret_cast<f32x4_any*>(row + e) = f32x4{v[j][0], v[j][1], v[j][2], v[j][3]};
        if (E & 3) {
#pragma unroll
          for (int i = 0; i < 3; ++i)
            if (e + 4 > E && e + i < E) row[e + i] = v[j][i];
        }
      }
    }
  }
  // softmax in place; a token of nothing but -inf has probabilities 0
  BAL_INL void softmax() {
    float m = v[0][0];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) m = fmaxf(m, v[j][i]);  // (a NaN makes the sum below NaN)
    m = lanes_max<LT>(m);
    if (m == -INFINITY) m = 0.f;  // (then every exp is 0)
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[j][i] = V == 1 ? expf(v[j][i] - m) : exp_diff(v[j][i] - m);
        s += v[j][i];
      }
    s = lanes_sum<LT>(s);
    if (s == 0.f) s = 1.f;
    // A product with 1 / s where a lane holds many: one more rounding for ten fewer
    // instructions each.  Where it holds one or two (up to 8 experts), the definition's own
    // operations, each rounded, as they cost little there (with the others 4096 x 8 8.0 us
    // and not 8.1, 300000 x 8 18.5 and not 19.0, 10^6 x 8 39.8 and not 41.4): equal counts,
    // whose gradient is 0 but for roundings, are common there.
    const float inv = __fdiv_rn(1.f, s);
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) v[j][i] = V == 1 ? __fdiv_rn(v[j][i], s) : v[j][i] * inv;
  }
  BAL_INL float dot(const float (&f)[J][V]) const {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float x = v[j][i] * f[j][i];
        if (V == 1) asm("" : "+v"(x));  // (rounded before it is added)
        s += x;
      }
    return lanes_sum<LT>(s);
  }
};

// Shared memory of a workgroup of W wavefronts, for at most NE experts
template <int W, int NE> struct Lds {
  int32_t hist[NE + 1];  // counts; hist[E]: kept tokens
  float col[W][NE];      // sums of probabilities of the wavefronts
  double loss[W];        // of the loss
};

BAL_INL double wave_sum(double v) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// Counts of a share of the pairs, and of the kept tokens among them, into hist (cleared
// here): four pairs to a load.
template <int W> BAL_INL void count_pairs(int32_t* hist, const BalanceArgs& a, int64_t part, int64_t parts) {
  for (int e = threadIdx.x; e <= a.E; e += 64 * W) hist[e] = 0;
  __syncthreads();
  const int64_t P = (int64_t)a.T * a.k, step = 4 * parts * (64 * W);
#pragma unroll 4
  for (int64_t p = 4 * (part * (64 * W) + threadIdx.x); p < P; p += step) {
    i32x4 e = {-1, -1, -1, -1};
    if (p + 4 <= P) e = *reinterpret_cast<const i32x4_any*>(a.ids + p);
    else
      for (int i = 0; i < 3; ++i)
        if (p + i < P) e[i] = a.ids[p + i];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (a.mask) {
        if (p + i >= P) continue;
        const uint32_t t = (uint32_t)(p + i) / (uint32_t)a.k;
        if (!a.mask[t]) continue;
        if (t * (uint32_t)a.k == (uint32_t)(p + i)) atomicAdd(&hist[a.E], 1);
      }
      if ((uint32_t)e[i] < (uint32_t)a.E) atomicAdd(&hist[e[i]], 1);
    }
  }
  if (!a.mask && part == 0 && threadIdx.x == 0) hist[a.E] = a.T;
  __syncthreads();
}

// The tokens of this workgroup's share, U of a lane at a time.  SUM: probabilities summed
// into col[w] of every wavefront.  GRAD: gradients out, from the counts and kept tokens in hist.
template <int LT, int V, int J, int U, int W, bool SUM, bool GRAD>
BAL_INL void tokens(Lds<W, LT * V * J>& L, const BalanceArgs& a, int64_t part, int64_t parts) {
  constexpr int G = 64 / LT;  // tokens of a wavefront
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, l = lane % LT, g = lane / LT;
  float f[J][V], gs = 0.f;
  double sum[J][V];
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) sum[j][i] = 0.0;
  if constexpr (GRAD) {
    const int n = L.hist[a.E];
    const double per = n > 0 ? 1.0 / n : 0.0;
    const double per_pair = per / a.k;
    gs = (float)((double)a.alpha * a.E * per);
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = Tok<LT, V, J>::expert(l, j) + i;
        const double c = e < a.E ? (double)L.hist[e] : 0.0;
        f[j][i] = (float)(V == 1 ? c * per / a.k : c * per_pair);
      }
  }
  const int64_t step = parts * (W * G);
  for (int64_t t0 = part * (W * G) + w * G; t0 < a.T; t0 += U * step) {
    Tok<LT, V, J> x[U];
    bool kept[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t t = t0 + g + u * step;
      kept[u] = t < a.T;
      if (kept[u]) {
        x[u].load(a.logits + t * a.E, l, a.E);  // (padding's too: it need not wait for the mask)
        if (a.mask) kept[u] = a.mask[t] != 0;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t t = t0 + g + u * step;
      if (t - g >= a.T) continue;  // (of the whole wavefront)
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) x[u].v[j][i] = kept[u] ? x[u].v[j][i] : -INFINITY;  // probabilities 0
      x[u].softmax();
      if constexpr (SUM) {
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) sum[j][i] += (double)x[u].v[j][i];
      }
      if constexpr (GRAD) {
        if (SUM && !a.grad) continue;
        const float fp = x[u].dot(f);
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) x[u].v[j][i] = kept[u] ? gs * x[u].v[j][i] * (f[j][i] - fp) : 0.f;
        if (t < a.T) x[u].store(a.grad + t * a.E, l, a.E);
      }
    }
  }
  if constexpr (SUM) {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        double s = sum[j][i];
        for (int d = LT; d < 64; d <<= 1) s += __shfl_xor(s, d, 64);
        const int e = Tok<LT, V, J>::expert(l, j) + i;
        if (g == 0 && e < a.E) L.col[w][e] = (float)s;
      }
    __syncthreads();
  }
}

// Small batches: everything by one workgroup.
template <int LT, int V, int J, int U>
__global__ void __launch_bounds__(1024) balance_small_kernel(BalanceArgs a) {
  constexpr int W = 16;
  __shared__ Lds<W, LT * V * J> L;
  count_pairs<W>(L.hist, a, 0, 1);
  tokens<LT, V, J, U, W, true, true>(L, a, 0, 1);
  const int tid = threadIdx.x, n = L.hist[a.E];
  const double per = n > 0 ? 1.0 / n : 0.0;
  double s = 0.0;
  for (int e = tid; e < a.E; e += 64 * W) {
    double p = 0.0;
#pragma unroll
    for (int i = 0; i < W; ++i) p += (double)L.col[i][e];
    p *= per;
    a.probs[e] = (float)p;
    a.counts[e] = L.hist[e];
    s += (double)L.hist[e] * per / a.k * p;
  }
  s = wave_sum(s);
  if ((tid & 63) == 0) L.loss[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) {
    s = 0.0;
#pragma unroll
    for (int i = 0; i < W; ++i) s += L.loss[i];
    a.loss[0] = (float)((double)a.alpha * a.E * s);
  }
}

template <int LT, int V, int J, int U>
__global__ void __launch_bounds__(1024) balance_sums_kernel(BalanceArgs a) {
  constexpr int W = 16;
  __shared__ Lds<W, LT * V * J> L;
  count_pairs<W>(L.hist, a, blockIdx.x, gridDim.x);
  for (int e = threadIdx.x; e <= a.E; e += 64 * W) a.part_counts[(int64_t)blockIdx.x * (a.E + 1) + e] = L.hist[e];
  tokens<LT, V, J, U, W, true, false>(L, a, blockIdx.x, gridDim.x);
  for (int e = threadIdx.x; e < a.E; e += 64 * W) {
    double s = (double)L.col[0][e];
#pragma unroll
    for (int i = 1; i < W; ++i) s += (double)L.col[i][e];
    a.part_probs[(int64_t)blockIdx.x * a.E + e] = (float)s;
  }
}

// p[i * stride] of the shares i = first, first + step, ..., added in that order, eight on their
// way at a time, the last ones too (one by one, each costs a trip to memory).
template <typename S, typename P> BAL_INL S add_shares(const P* p, int stride, int first, int step, int n_part) {
  S s = 0;
  int i = first;
  for (; i + 7 * step < n_part; i += 8 * step)
#pragma unroll
    for (int u = 0; u < 8; ++u) s += (S)p[(i + u * step) * stride];
  if (i < n_part) {
    P v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = p[min(i + u * step, n_part - 1) * stride];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += i + u * step < n_part ? (S)v[u] : (S)0;
  }
  return s;
}

// Many shares of many experts, added in their order to the first one: 32 columns to a
// workgroup, 16 threads each a run of the shares.
__global__ void __launch_bounds__(512) balance_fold_kernel(BalanceArgs a, int n_part) {
  __shared__ double sum[16][32];
  __shared__ int32_t cnt[32];
  const int tid = threadIdx.x, c = tid & 31, r = tid >> 5, e = blockIdx.x * 32 + c;
  if (tid < 32) cnt[tid] = 0;
  __syncthreads();
  if (e <= a.E) {
    atomicAdd(&cnt[c], add_shares<int32_t>(a.part_counts + e, a.E + 1, r, 16, n_part));
    sum[r][c] = e < a.E ? add_shares<double>(a.part_probs + e, a.E, r, 16, n_part) : 0.0;
  }
  __syncthreads();
  if (tid < 32 && e <= a.E) {
    a.part_counts[e] = cnt[c];
    if (e == a.E) return;
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += sum[i][c];
    a.part_probs[e] = (float)s;
  }
}

// The first workgroup: counts, mean probabilities and loss from the shares; the others: the
// gradient of their tokens.
template <int LT, int V, int J, int U>
__global__ void __launch_bounds__(kThreads) balance_grad_kernel(BalanceArgs a) {
  constexpr int W = kThreads / 64;
  __shared__ Lds<W, LT * V * J> L;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (a.n_part == 1) {
    for (int e = tid; e <= a.E; e += kThreads) L.hist[e] = a.part_counts[e];
  } else {  // a wavefront adds up some of the shares, lanes along the experts
    for (int e = tid; e <= a.E; e += kThreads) L.hist[e] = 0;
    __syncthreads();
    for (int e = lane; e <= a.E; e += 64) atomicAdd(&L.hist[e], add_shares<int32_t>(a.part_counts + e, a.E + 1, w, W, a.n_part));
  }
  if (blockIdx.x > 0) {
    __syncthreads();
    tokens<LT, V, J, U, W, false, true>(L, a, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  // EP threads (a power of two) along the experts, the rest of the workgroup along the shares
  int EP = 32;
  while (EP < a.E && EP < kThreads) EP *= 2;
  const int c = tid & (EP - 1), r = tid / EP, R = kThreads / EP;
  __shared__ double share[kThreads];
  __syncthreads();
  const int n = L.hist[a.E];
  const double per = n > 0 ? 1.0 / n : 0.0;
  double s = 0.0;
  for (int e0 = 0; e0 < a.E; e0 += EP) {
    const int e = e0 + c;
    double p = e < a.E ? add_shares<double>(a.part_probs + e, a.E, r, R, a.n_part) : 0.0;
    share[tid] = p;
    __syncthreads();
    if (r == 0 && e < a.E) {
      for (int i = 1; i < R; ++i) p += share[i * EP + c];
      p *= per;
      a.probs[e] = (float)p;
      a.counts[e] = L.hist[e];
      s += (double)L.hist[e] * per / a.k * p;
    }
    __syncthreads();
  }
  s = wave_sum(s);
  if (lane == 0) L.loss[w] = s;
  __syncthreads();
  if (tid == 0) {
    s = 0.0;
#pragma unroll
    for (int i = 0; i < W; ++i) s += L.loss[i];
    a.loss[0] = (float)((double)a.alpha * a.E * s);
  }
}

template <int LT, int V, int J> hipError_t go(const BalanceArgs& a, hipStream_t s) {
  constexpr int U = V * J > 8 ? 2 : 4;  // tokens of a lane in flight
  if (a.n_part == 0) {
    hipLaunchKernelGGL((balance_small_kernel<LT, V, J, U>), dim3(1), dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((balance_sums_kernel<LT, V, J, U>), dim3(a.n_part), dim3(1024), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  BalanceArgs b = a;
  // (every gradient workgroup reads all shares of the counts: where they are many, a launch
  // adds them up once.  us without / with it, shares x experts: 256 x 128 18.0 / 15.6, 256 x 256
  // 27.8 / 21.7, 128 x 160 13.1 / 11.9, 256 x 64 19.6 / 20.5, 64 x 256 11.2 / 11.5, 64 x 128
  // 10.0 / 11.4; and, as a wavefront goes through the experts 64 at a time, 32 x 512 14.2 / 13.2,
  // 10 x 1000 19.9 / 15.5)
  if (a.n_part > 1 && (a.n_part * a.E > 16384 || a.E > 256)) {
    hipLaunchKernelGGL(balance_fold_kernel, dim3((a.E + 32) / 32), dim3(512), 0, s, a, a.n_part);
    const hipError_t f = hipGetLastError();
    if (f != hipSuccess) return f;
    b.n_part = 1;
  }
  hipLaunchKernelGGL((balance_grad_kernel<LT, V, J, U>), dim3(1 + (a.grad ? a.n_grad : 0)), dim3(kThreads), 0, s, b);
  return hipGetLastError();
}

}  // namespace

// Lanes of a token.  Few experts: a lane to an expert (or two), lanes a power of two.
static int token_lanes(int E) {
  if (E <= 8) return E == 8 ? 8 : (E > 3 ? 4 : (E > 1 ? 2 : 1));
  int lt = 4;
  while (lt < 64 && 4 * lt < E) lt *= 2;
  return lt;
}

// Workgroups of a call.  One for everything up to 64 wavefronts' worth of tokens (a launch costs
// more than they do: 64 tokens of 60 experts 5.0 us, 6.6 in two launches; 256 7.3 and 7.5; 512
// of 64 11.1 and 8.2).  Otherwise a token to a lane of a summing workgroup up to 64 of them (4096 x
// 60: 64 of them 9.1 us, 32 9.8, 16 11.2; 1000 x 512: 63 of them 11.8, 32 13.3), then two, as the
// shares cost too (4096 x 128: 128 of them 10.7, 64 10.0; 65536 x 64: 256 19.6, 128 20.4), and 1024
// logits to a gradient one (4096 x 60 8.5 us, with 2048 9.0, 512 8.6; 2000 x 60 8.5, 8.9, 8.5; others
// within 2%).  All of them with fp32 sums over tokens; 64-bit ones add 0 to 3% to each.
void balance_shares(int32_t T, int32_t E, int32_t* n_part, int32_t* n_grad) {
  const int64_t waves = ((int64_t)T * token_lanes(E) + 63) / 64, logits = (int64_t)T * E;
  *n_part = waves <= 64 ? 0 : (int32_t)std::max(std::min<int64_t>(64, (waves + 15) / 16), std::min<int64_t>(256, (waves + 31) / 32));
  *n_grad = (int32_t)std::min<int64_t>(512, (logits + 1023) / 1024);
}

hipError_t launch_balance_loss(const BalanceArgs& a, hipStream_t s) {
  if (a.E == 1) return go<1, 1, 1>(a, s);
  if (a.E <= 3) return go<2, 1, 2>(a, s);
  if (a.E <= 7) return go<4, 1, 2>(a, s);
  if (a.E == 8) return go<8, 1, 1>(a, s);
  if (a.E <= 16) return go<4, 4, 1>(a, s);
  if (a.E <= 32) return go<8, 4, 1>(a, s);
  if (a.E <= 64) return go<16, 4, 1>(a, s);
  if (a.E <= 128) return go<32, 4, 1>(a, s);
  if (a.E <= 256) return go<64, 4, 1>(a, s);
  if (a.E <= 512) return go<64, 4, 2>(a, s);
  return go<64, 4, 4>(a, s);
}

}  // namespace mxmoe
