// Balance loss of the router, with per-expert counts, mean probabilities and the
// gradient of the logits.  Over the n tokens that the mask keeps:
//   c_e = number of (token, slot) pairs with expert e,  f_e = c_e / (k n)
//   P_e = 1/n sum_t p[t,e],  p[t] = softmax of the token's logits
//   L = alpha E sum_e f_e P_e
//   dL/dlogits[t,e] = alpha E / n * p[t,e] (f_e - sum_j f_j p[t,j])
// The counts are constants of the gradient (a choice of experts has none), so a
// token's gradient needs the counts and its own logits only: one pass over the
// logits after one over the ids.
#include "mxmoe_internal.h"

namespace mxmoe {
namespace {

constexpr int kThreads = 256;

__device__ inline float wave_sum(float v) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}
__device__ inline float wave_max(float v) {
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
  return v;
}

// counts of a share of the tokens, and how many of them the mask keeps
__global__ void __launch_bounds__(kThreads) balance_count_kernel(BalanceArgs a) {
  __shared__ int32_t hist[kMaxE + 1];
  for (int e = threadIdx.x; e <= a.E; e += kThreads) hist[e] = 0;
  __syncthreads();
  for (int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x; p < (int64_t)a.T * a.k; p += (int64_t)gridDim.x * kThreads) {
    const int t = (int)(p / a.k);
    if (a.mask && !a.mask[t]) continue;
    const int e = a.ids[p];
    if (e >= 0 && e < a.E) atomicAdd(&hist[e], 1);
    if (p == (int64_t)t * a.k) atomicAdd(&hist[a.E], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e <= a.E; e += kThreads) a.part_counts[(int64_t)blockIdx.x * (a.E + 1) + e] = hist[e];
}

// one wavefront per token, strided over the tokens
__global__ void __launch_bounds__(kThreads) balance_grad_kernel(BalanceArgs a) {
  __shared__ float f[kMaxE];
  __shared__ float col[kMaxE];
  __shared__ float wcol[kThreads / 64][kMaxE];
  __shared__ int32_t kept;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  for (int e = tid; e <= a.E; e += kThreads) {
    int32_t c = 0;
    for (int g = 0; g < a.n_count; ++g) c += a.part_counts[(int64_t)g * (a.E + 1) + e];
    if (e < a.E) f[e] = (float)c;
    else kept = c;
    if (blockIdx.x == 0 && e < a.E) a.counts[e] = c;
  }
  __syncthreads();
  const int n = kept;
  const double per = n > 0 ? 1.0 / n : 0.0;
  for (int e = tid; e < a.E; e += kThreads) f[e] = (float)((double)f[e] * per / a.k);
  for (int e = lane; e < a.E; e += 64) wcol[w][e] = 0.f;
  __syncthreads();
  const float gs = (float)((double)a.alpha * a.E * per);
  for (int64_t t = (int64_t)blockIdx.x * (kThreads / 64) + w; t < a.T; t += (int64_t)gridDim.x * (kThreads / 64)) {
    const float* l = a.logits + t * a.E;
    float* g = a.grad ? a.grad + t * a.E : nullptr;
    if (a.mask && !a.mask[t]) {
      if (g)
        for (int e = lane; e < a.E; e += 64) g[e] = 0.f;
      continue;
    }
    float m = -INFINITY;
    bool nan = false;
    for (int e = lane; e < a.E; e += 64) {
      nan |= l[e] != l[e];
      m = fmaxf(m, l[e]);
    }
    m = wave_max(m);
    if (__ballot(nan)) m = __builtin_nanf("");
    const bool none = m == -INFINITY;
    float se = 0.f, fp = 0.f;
    for (int e = lane; e < a.E; e += 64) {
      const float x = none ? 0.f : expf(l[e] - m);
      se += x;
      fp += x * f[e];
    }
    se = wave_sum(se);
    fp = wave_sum(fp);
    const float inv = none ? 0.f : 1.f / se;
    for (int e = lane; e < a.E; e += 64) {
      const float p = none ? 0.f : expf(l[e] - m) * inv;
      wcol[w][e] += p;
      if (g) g[e] = gs * p * (f[e] - fp * inv);
    }
  }
  __syncthreads();
  for (int e = tid; e < a.E; e += kThreads) {
    float c = 0.f;
    for (int i = 0; i < kThreads / 64; ++i) c += wcol[i][e];
    a.part_probs[(int64_t)blockIdx.x * a.E + e] = c;
  }
}

__global__ void __launch_bounds__(kThreads) balance_loss_kernel(BalanceArgs a) {
  __shared__ double red[kThreads];
  int32_t n = 0;
  for (int g = 0; g < a.n_count; ++g) n += a.part_counts[(int64_t)g * (a.E + 1) + a.E];
  const double per = n > 0 ? 1.0 / n : 0.0;
  double s = 0.0;
  for (int e = threadIdx.x; e < a.E; e += kThreads) {
    double c = 0.0;
    for (int g = 0; g < a.n_part; ++g) c += (double)a.part_probs[(int64_t)g * a.E + e];
    int32_t cnt = 0;
    for (int g = 0; g < a.n_count; ++g) cnt += a.part_counts[(int64_t)g * (a.E + 1) + e];
    a.probs[e] = (float)(c * per);
    s += (double)cnt * per / a.k * c * per;
  }
  red[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int i = 0; i < kThreads; ++i) t += red[i];
    a.loss[0] = (float)((double)a.alpha * a.E * t);
  }
}

}  // namespace

hipError_t launch_balance_loss(const BalanceArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(balance_count_kernel, dim3(a.n_count), dim3(kThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(balance_grad_kernel, dim3(a.n_part), dim3(kThreads), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(balance_loss_kernel, dim3(1), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace mxmoe
