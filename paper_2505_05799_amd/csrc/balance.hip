// Balance loss of the router, with per-expert counts, mean probabilities and the
// gradient of the logits.  Over the n tokens that the mask keeps:
//   c_e = number of (token, slot) pairs with expert e,  f_e = c_e / (k n)
//   P_e = 1/n sum_t p[t,e],  p[t] = softmax of the token's logits
//   L = alpha E sum_e f_e P_e
//   dL/dlogits[t,e] = alpha E / n * p[t,e] (f_e - sum_j f_j p[t,j])
// The counts are constants of the gradient (a choice of experts has none), so a
// token's gradient needs the counts and its own logits only: the ids are counted
// first, by a launch of their own, then one pass over the logits writes the gradient
// and sums the probabilities; the last workgroup to finish it adds up the shares of
// all, in their order, and forms the loss.  Small batches take one workgroup and one
// launch.
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
// the largest; NaN where one is
template <int L> BAL_INL float lanes_max(float v) {
  return lanes<L>(v, [](float a, float b) { return (a > b || a != a) ? a : b; });
}

// Logits of a token in a lane: chunk j holds experts V (LT j + l) .. + V - 1 (V = 1: LT j + l).
template <int LT, int V, int J> struct Tok {
  float v[J][V];
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
      for (int i = 0; i < V; ++i) m = (m > v[j][i] || m != m) ? m : v[j][i];
    m = lanes_max<LT>(m);
    const bool none = m == -INFINITY;
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[j][i] = none ? 0.f : expf(v[j][i] - m);
        s += v[j][i];
      }
    s = lanes_sum<LT>(s);
    if (none) s = 1.f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) v[j][i] = __fdiv_rn(v[j][i], s);
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

// Shared memory of a workgroup of W wavefronts
template <int W> struct Lds {
  int32_t hist[kMaxE + 1];  // counts, then kept tokens
  float f[kMaxE];
  float col[W][kMaxE];
  double red[W];
  int32_t flag;
};

BAL_INL double wave_sum(double v) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// Counts of the pairs first .. first + step, ... into L.hist (cleared here), and of the kept tokens
template <int W> BAL_INL void count_pairs(Lds<W>& L, const BalanceArgs& a, int64_t part, int64_t parts) {
  for (int e = threadIdx.x; e <= a.E; e += 64 * W) L.hist[e] = 0;
  __syncthreads();
  const int64_t P = (int64_t)a.T * a.k;
  if (!a.mask) {
    // four pairs to a load
    for (int64_t p = 4 * (part * (64 * W) + threadIdx.x); p < P; p += 4 * parts * (64 * W)) {
      i32x4 e = {-1, -1, -1, -1};
      if (p + 4 <= P) e = *reinterpret_cast<const i32x4_any*>(a.ids + p);
      else
        for (int i = 0; i < 3; ++i)
          if (p + i < P) e[i] = a.ids[p + i];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((uint32_t)e[i] < (uint32_t)a.E) atomicAdd(&L.hist[e[i]], 1);
    }
    if (part == 0 && threadIdx.x == 0) L.hist[a.E] = a.T;
  } else {
    for (int64_t t = part * (64 * W) + threadIdx.x; t < a.T; t += parts * (64 * W)) {
      if (!a.mask[t]) continue;
      atomicAdd(&L.hist[a.E], 1);
      for (int s = 0; s < a.k; ++s) {
        const int e = a.ids[t * a.k + s];
        if ((uint32_t)e < (uint32_t)a.E) atomicAdd(&L.hist[e], 1);
      }
    }
  }
  __syncthreads();
}

// The tokens of this workgroup's part: gradients out, probabilities summed into L.col[w].
// counts and kept tokens are in L.hist.
template <int LT, int V, int J, int U, int W>
BAL_INL void tokens(Lds<W>& L, const BalanceArgs& a, int64_t part, int64_t parts) {
  constexpr int G = 64 / LT;  // tokens of a wavefront
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, l = lane % LT, g = lane / LT;
  const int n = L.hist[a.E];
  const double per = n > 0 ? 1.0 / n : 0.0;
  const float gs = (float)((double)a.alpha * a.E * per);
  float f[J][V], sum[J][V];
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = Tok<LT, V, J>::expert(l, j) + i;
      f[j][i] = e < a.E ? (float)((double)L.hist[e] * per / a.k) : 0.f;
      sum[j][i] = 0.f;
    }
  const int64_t step = parts * (W * G);
  for (int64_t t0 = part * (W * G) + w * G + g; t0 - g < a.T; t0 += U * step) {
    Tok<LT, V, J> x[U];
    bool kept[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t t = t0 + u * step;
      kept[u] = t < a.T && (!a.mask || a.mask[t]);
      if (kept[u]) x[u].load(a.logits + t * a.E, l, a.E);
      else
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) x[u].v[j][i] = -INFINITY;  // probabilities 0, gradient 0
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t t = t0 + u * step;
      x[u].softmax();
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) sum[j][i] += x[u].v[j][i];
      if (a.grad) {
        const float fp = x[u].dot(f);
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) x[u].v[j][i] = kept[u] ? gs * x[u].v[j][i] * (f[j][i] - fp) : 0.f;
        if (t < a.T) x[u].store(a.grad + t * a.E, l, a.E);
      }
    }
  }
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

// The loss from the sums of probabilities: sum(e) by a lane each.
template <int W, typename F> BAL_INL void finish(Lds<W>& L, const BalanceArgs& a, F sum) {
  const int tid = threadIdx.x, n = L.hist[a.E];
  const double per = n > 0 ? 1.0 / n : 0.0;
  double s = 0.0;
  for (int e = tid; e < a.E; e += 64 * W) {
    const double p = sum(e) * per;
    a.probs[e] = (float)p;
    a.counts[e] = L.hist[e];
    s += (double)L.hist[e] * per / a.k * p;
  }
  s = wave_sum(s);
  if ((tid & 63) == 0) L.red[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) {
    s = 0.0;
    for (int i = 0; i < W; ++i) s += L.red[i];
    a.loss[0] = (float)((double)a.alpha * a.E * s);
  }
}

// Small batches: everything by one workgroup.
template <int LT, int V, int J>
__global__ void __launch_bounds__(1024) balance_small_kernel(BalanceArgs a) {
  __shared__ Lds<16> L;
  count_pairs<16>(L, a, 0, 1);
  tokens<LT, V, J, 1, 16>(L, a, 0, 1);
  finish<16>(L, a, [&](int e) {
    double s = 0.0;
    for (int i = 0; i < 16; ++i) s += (double)L.col[i][e];
    return s;
  });
}

__global__ void __launch_bounds__(kThreads) balance_count_kernel(BalanceArgs a) {
  __shared__ Lds<kThreads / 64> L;
  count_pairs<kThreads / 64>(L, a, blockIdx.x, gridDim.x);
  for (int e = threadIdx.x; e <= a.E; e += kThreads) a.part_counts[(int64_t)blockIdx.x * (a.E + 1) + e] = L.hist[e];
}

template <int LT, int V, int J, int U>
__global__ void __launch_bounds__(kThreads) balance_kernel(BalanceArgs a) {
  constexpr int W = kThreads / 64;
  __shared__ Lds<W> L;
  const int tid = threadIdx.x;
  for (int e = tid; e <= a.E; e += kThreads) {
    int32_t c = 0;
    for (int i = 0; i < a.n_count; ++i) c += a.part_counts[(int64_t)i * (a.E + 1) + e];
    L.hist[e] = c;
  }
  __syncthreads();
  tokens<LT, V, J, U, W>(L, a, blockIdx.x, gridDim.x);
  for (int e = tid; e < a.E; e += kThreads) {
    float s = L.col[0][e];
    for (int i = 1; i < W; ++i) s += L.col[i][e];
    a.part_probs[(int64_t)blockIdx.x * a.E + e] = s;
  }
}

__global__ void __launch_bounds__(1024) balance_loss_kernel(BalanceArgs a) {
  __shared__ Lds<16> L;
  __shared__ double part[1024];
  const int tid = threadIdx.x;
  for (int e = tid; e <= a.E; e += 1024) {
    int32_t c = 0;
    for (int i = 0; i < a.n_count; ++i) c += a.part_counts[(int64_t)i * (a.E + 1) + e];
    L.hist[e] = c;
  }
  // R threads to an expert, each a run of the shares
  int R = 1;
  while (2 * R * a.E <= 1024) R *= 2;
  const int e = tid % a.E, r = tid / a.E;
  double s = 0.0;
  if (r < R)
    for (int i = r; i < a.n_part; i += R) s += (double)a.part_probs[(int64_t)i * a.E + e];
  part[tid] = s;
  __syncthreads();
  finish<16>(L, a, [&](int c) {
    double t = 0.0;
    for (int i = 0; i < R; ++i) t += part[i * a.E + c];
    return t;
  });
}

template <int LT, int V, int J> hipError_t go(const BalanceArgs& a, hipStream_t s) {
  if (a.n_part == 0) {
    hipLaunchKernelGGL((balance_small_kernel<LT, V, J>), dim3(1), dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(balance_count_kernel, dim3(a.n_count), dim3(kThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr int U = V * J > 4 ? 1 : 4;
  hipLaunchKernelGGL((balance_kernel<LT, V, J, U>), dim3(a.n_part), dim3(kThreads), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(balance_loss_kernel, dim3(1), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_balance_loss(const BalanceArgs& a, hipStream_t s) {
  // few experts: a lane to an expert (or two), lanes a power of two
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
