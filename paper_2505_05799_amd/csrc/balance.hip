// Balance loss of the router, with per-expert counts, mean probabilities and the
// gradient of the logits.  Over the n tokens that the mask keeps:
//   c_e = number of (token, slot) pairs with expert e,  f_e = c_e / (k n)
//   P_e = 1/n sum_t p[t,e],  p[t] = softmax of the token's logits
//   L = alpha E sum_e f_e P_e
//   dL/dlogits[t,e] = alpha E / n * p[t,e] (f_e - sum_j f_j p[t,j])
// The counts are constants of the gradient (a choice of experts has none), so a
// token's gradient needs the counts and its own logits only: the ids are counted
// first, by a launch of their own, then one pass over the logits writes the gradient
// and sums the probabilities and the dots (L = alpha E / n sum_t sum_j f_j p[t,j]), and
// a last launch adds the workgroups' shares in their order.  Small batches take one
// workgroup and one launch.
//
// A token is held by LT lanes, V consecutive logits to a lane and chunk, so that a
// wavefront reads 64 / LT tokens side by side; sums over a token are butterflies
// over its lanes.
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
// the larger one; NaN where one is
BAL_INL float larger(float a, float b) { return (a > b || a != a) ? a : b; }
template <int L> BAL_INL float lanes_max(float v) { return lanes<L>(v, larger); }
// exp(d) for d <= 0 within 2 units in the last place: 2^(d log2 e) with the rounding error
// of the product put back (the library's expf takes three times the instructions; with it
// and a quotient a probability, one workgroup took 14.4 us for 512 tokens of 64 experts)
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
  BAL_INL void load(const float* row, int l, int E) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int e = expert(l, j);
      if (V == 4 && e + 4 <= E) {
        const f32x4 x = *reinterpret_cast<const f32x4_any*>(row + e);
#pragma unroll
        for (int i = 0; i < V; ++i) v[j][i] = x[i];
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[j][i] = e + i < E ? row[e + i] : -INFINITY;
      }
    }
  }
  BAL_INL void store(float* row, int l, int E) const {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int e = expert(l, j);
      if (V == 4 && e + 4 <= E) {
        f32x4 x;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = v[j][i];
        *reinterpret_cast<f32x4_any*>(row + e) = x;
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (e + i < E) row[e + i] = v[j][i];
      }
    }
  }
  // softmax in place; a token of nothing but -inf has probabilities 0
  BAL_INL void softmax() {
    float m = v[0][0];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) m = larger(m, v[j][i]);
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
    // a product with 1 / s where a lane holds many (one more rounding for ten fewer
    // instructions each), quotients where it holds one or two
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
      for (int i = 0; i < V; ++i) s += v[j][i] * f[j][i];
    return lanes_sum<LT>(s);
  }
};

// Shared memory of a workgroup of W wavefronts, for at most NE experts
template <int W, int NE> struct Lds {
  int32_t hist[NE + 1];  // counts; hist[E]: kept tokens
  float col[W][NE];      // sums of probabilities
  double loss[W];        // sums of dots
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

// The tokens of this workgroup's share, U of a lane at a time: gradients out;
// probabilities and dots summed into col[w] and loss[w] of every wavefront.  Counts and
// kept tokens are in hist.
template <int LT, int V, int J, int U, int W>
BAL_INL void tokens(Lds<W, LT * V * J>& L, const BalanceArgs& a, int64_t part, int64_t parts) {
  constexpr int G = 64 / LT;  // tokens of a wavefront
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, l = lane % LT, g = lane / LT;
  const int n = L.hist[a.E];
  const double per = n > 0 ? 1.0 / n : 0.0;
  const float gs = (float)((double)a.alpha * a.E * per);
  float f[J][V], sum[J][V];
  double dots = 0.0;
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = Tok<LT, V, J>::expert(l, j) + i;
      f[j][i] = e < a.E ? (float)((double)L.hist[e] * per / a.k) : 0.f;
      sum[j][i] = 0.f;
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
      const float fp = x[u].dot(f);
      dots += (double)fp;
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float q = x[u].v[j][i];
          sum[j][i] += q;
          x[u].v[j][i] = kept[u] ? gs * q * (f[j][i] - fp) : 0.f;
        }
      if (a.grad && t < a.T) x[u].store(a.grad + t * a.E, l, a.E);
    }
  }
  if (l != 0) dots = 0.0;  // (a token's lanes hold the same dot)
  dots = wave_sum(dots);
  if (lane == 0) L.loss[w] = dots;
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float s = sum[j][i];
      for (int d = LT; d < 64; d <<= 1) s += __shfl_xor(s, d, 64);
      const int e = Tok<LT, V, J>::expert(l, j) + i;
      if (g == 0 && e < a.E) L.col[w][e] = s;
    }
  __syncthreads();
}

// Small batches: everything by one workgroup.
template <int LT, int V, int J, int U>
__global__ void __launch_bounds__(1024) balance_small_kernel(BalanceArgs a) {
  constexpr int W = 16;
  __shared__ Lds<W, LT * V * J> L;
  count_pairs<W>(L.hist, a, 0, 1);
  tokens<LT, V, J, U, W>(L, a, 0, 1);
  const int n = L.hist[a.E];
  const double per = n > 0 ? 1.0 / n : 0.0;
  for (int e = threadIdx.x; e < a.E; e += 64 * W) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < W; ++i) s += (double)L.col[i][e];
    a.probs[e] = (float)(s * per);
    a.counts[e] = L.hist[e];
  }
  if (threadIdx.x == 0) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < W; ++i) s += L.loss[i];
    a.loss[0] = (float)((double)a.alpha * a.E * per * s);
  }
}

__global__ void __launch_bounds__(kThreads) balance_count_kernel(BalanceArgs a) {
  __shared__ int32_t hist[kMaxE + 1];
  count_pairs<kThreads / 64>(hist, a, blockIdx.x, gridDim.x);
  for (int e = threadIdx.x; e <= a.E; e += kThreads) a.part_counts[(int64_t)blockIdx.x * (a.E + 1) + e] = hist[e];
}

template <int LT, int V, int J, int U>
__global__ void __launch_bounds__(kThreads) balance_kernel(BalanceArgs a) {
  constexpr int W = kThreads / 64;
  __shared__ Lds<W, LT * V * J> L;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  // the counts: a wavefront adds up some of the shares, lanes along the experts
  for (int e = tid; e <= a.E; e += kThreads) L.hist[e] = 0;
  __syncthreads();
  for (int e = lane; e <= a.E; e += 64) {
    int32_t c = 0;
#pragma unroll 8
    for (int i = w; i < a.n_count; i += W) c += a.part_counts[(int64_t)i * (a.E + 1) + e];
    atomicAdd(&L.hist[e], c);
  }
  __syncthreads();
  tokens<LT, V, J, U, W>(L, a, blockIdx.x, gridDim.x);
  for (int e = tid; e < a.E; e += kThreads) {
    float s = L.col[0][e];
#pragma unroll
    for (int i = 1; i < W; ++i) s += L.col[i][e];
    a.part_probs[(int64_t)blockIdx.x * a.E + e] = s;
  }
  if (tid == 0) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < W; ++i) s += L.loss[i];
    a.part_loss[blockIdx.x] = s;
  }
}

// The shares of all workgroups, added in their order: 32 experts to a workgroup, 16
// threads each a run of the shares.  The first workgroup also adds the loss.
__global__ void __launch_bounds__(512) balance_sum_kernel(BalanceArgs a) {
  __shared__ double sum[16][32];
  __shared__ int32_t cnt[32], kept;
  __shared__ double loss[8];
  const int tid = threadIdx.x, c = tid & 31, r = tid >> 5, e = blockIdx.x * 32 + c;
  if (tid < 32) cnt[tid] = 0;
  if (tid == 0) kept = 0;
  __syncthreads();
  int32_t k = 0;
  for (int i = tid; i < a.n_count; i += 512) k += a.part_counts[(int64_t)i * (a.E + 1) + a.E];
  if (tid < a.n_count) atomicAdd(&kept, k);
  double s = 0.0;
  if (e < a.E) {
    int32_t n = 0;
#pragma unroll 8
    for (int i = r; i < a.n_count; i += 16) n += a.part_counts[(int64_t)i * (a.E + 1) + e];
    atomicAdd(&cnt[c], n);
#pragma unroll 8
    for (int i = r; i < a.n_part; i += 16) s += (double)a.part_probs[(int64_t)i * a.E + e];
  }
  sum[r][c] = s;
  if (blockIdx.x == 0) {
    double l = 0.0;
    for (int i = tid; i < a.n_part; i += 512) l += a.part_loss[i];
    l = wave_sum(l);
    if ((tid & 63) == 0) loss[tid >> 6] = l;
  }
  __syncthreads();
  const double per = kept > 0 ? 1.0 / kept : 0.0;
  if (tid < 32 && e < a.E) {
    s = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += sum[i][c];
    a.probs[e] = (float)(s * per);
    a.counts[e] = cnt[c];
  }
  if (blockIdx.x == 0 && tid == 0) {
    s = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += loss[i];
    a.loss[0] = (float)((double)a.alpha * a.E * per * s);
  }
}

template <int LT, int V, int J> hipError_t go(const BalanceArgs& a, hipStream_t s) {
  constexpr int U = V * J > 4 ? 1 : 4;  // tokens of a lane in flight
  if (a.n_part == 0) {
    hipLaunchKernelGGL((balance_small_kernel<LT, V, J, U>), dim3(1), dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(balance_count_kernel, dim3(a.n_count), dim3(kThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((balance_kernel<LT, V, J, U>), dim3(a.n_part), dim3(kThreads), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(balance_sum_kernel, dim3((a.E + 31) / 32), dim3(512), 0, s, a);
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
// more than they do: 64 tokens of 60 experts 5.7 us against 9.2 in three launches, 256 8.7 and
// 9.2, 512 of 64 12.0 and 10.2).  Otherwise 4096 pairs to a counting workgroup and 2048 logits
// to one of the tokens', at most 128 and 256: more of them bring the shares of the counts in more
// often than they save (65536 x 64: 128 / 256 21.4 us, 32 / 256 23.7, 64 / 512 23.6).
void balance_shares(int32_t T, int32_t E, int32_t k, int32_t* n_count, int32_t* n_part) {
  const int64_t pairs = (int64_t)T * k, logits = (int64_t)T * E;
  *n_part = (int64_t)T * token_lanes(E) <= 64 * 64 ? 0 : (int32_t)(logits >= kBalPart * 2048 ? kBalPart : (logits + 2047) / 2048);
  *n_count = *n_part == 0 ? 0 : (int32_t)(pairs >= kBalCount * 4096 ? kBalCount : (pairs + 4095) / 4096);
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
