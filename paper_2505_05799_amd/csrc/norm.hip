// Residual addition, RMS norm and per-row 8-bit encoding in one launch.
//
//   z = round(x + residual)                         (the activation dtype)
//   r = fl32(1 / sqrt(mean(z^2) + eps))             (64-bit sum, root and quotient)
//   y = round(fl32(fl32(z r) weight))
//   codes, scale = the per-token recipe of rowquant.h on the rounded y
//
// The squares of 16-bit values are exact in 64 bits and their sum errs by some
// 2^-50, so r is the same whatever the order of the sum, and with it every bit
// of y, the codes and the scale: they equal act_quant of y, for any split of a
// row over lanes.
#include "mxmoe_internal.h"
#include "rowquant.h"

namespace mxmoe {
namespace {

constexpr int kThreads = 256;
// a row whose largest |y| is below this counts as zero: qmax / |y| would overflow
constexpr float kTinyAmax = 0x1p-118f;

template <int ACT> __device__ inline float norm_load(const uint16_t* p) {
  if constexpr (ACT == MXMOE_BF16) return __uint_as_float((uint32_t)*p << 16);
  else return (float)__builtin_bit_cast(_Float16, *p);
}
template <int ACT> __device__ inline uint16_t norm_round(float f) {
  // (the barrier keeps a product that was rounded to fp32 from being fused
  // with the conversion into one rounding)
  asm("" : "+v"(f));
  if constexpr (ACT == MXMOE_BF16) return __builtin_bit_cast(uint16_t, (__bf16)f);
  else return __builtin_bit_cast(uint16_t, (_Float16)f);
}

// One workgroup per row, one element per thread and step; the row is read once
// for the sum, once for the largest magnitude and once for the codes.
template <int ACT>
__global__ void __launch_bounds__(kThreads) norm_row_kernel(NormArgs a) {
  __shared__ double red[kThreads / 64];
  __shared__ uint32_t redm[kThreads / 64];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
  __syncthreads();  // (the last row's reductions are read)
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const uint16_t* x = reinterpret_cast<const uint16_t*>(a.x) + row * a.ldx;
  const uint16_t* res = a.res ? reinterpret_cast<const uint16_t*>(a.res) + row * a.ldr : nullptr;
  const uint16_t* g = reinterpret_cast<const uint16_t*>(a.weight);
  uint16_t* sum = a.sum ? reinterpret_cast<uint16_t*>(a.sum) + row * a.lds : nullptr;
  uint16_t* y = a.y ? reinterpret_cast<uint16_t*>(a.y) + row * a.ldy : nullptr;
  auto z_of = [&](int c) -> uint16_t {
    return res ? norm_round<ACT>(norm_load<ACT>(x + c) + norm_load<ACT>(res + c)) : x[c];
  };
  double ss = 0.0;
  for (int c = tid; c < a.cols; c += kThreads) {
    const uint16_t zb = z_of(c);
    const double z = (double)norm_load<ACT>(&zb);
    ss += z * z;
  }
  for (int d = 32; d > 0; d >>= 1) ss += __shfl_xor(ss, d, 64);
  if (lane == 0) red[w] = ss;
  __syncthreads();
  ss = (red[0] + red[1]) + (red[2] + red[3]);
  const float r = (float)(1.0 / sqrt(ss / (double)a.cols + a.eps));
  auto y_of = [&](int c) -> uint16_t {
    const uint16_t zb = z_of(c);
    return norm_round<ACT>(__fmul_rn(__fmul_rn(norm_load<ACT>(&zb), r), norm_load<ACT>(g + c)));
  };
  float inv = 0.f, scale = 0.f;
  if (a.qmax) {
    uint32_t mb = 0u;
    for (int c = tid; c < a.cols; c += kThreads) mb = max(mb, (uint32_t)y_of(c) & 0x7fffu);
    for (int d = 32; d > 0; d >>= 1) mb = max(mb, (uint32_t)__shfl_xor((int)mb, d, 64));
    if (lane == 0) redm[w] = mb;
    __syncthreads();
    mb = max(max(redm[0], redm[1]), max(redm[2], redm[3]));
    const float amax = bits_to_f32(mb, ACT), q = (float)a.qmax;
    if (mb >= (ACT == MXMOE_BF16 ? 0x7f80u : 0x7c00u)) {
      scale = __builtin_nanf("");
    } else if (amax >= kTinyAmax) {
      inv = __fdiv_rn(q, amax);
      scale = __fdiv_rn(amax, q);
    }
    if (tid == 0) a.scales[row] = scale;
  }
  for (int c = tid; c < a.cols; c += kThreads) {
    const uint16_t yb = y_of(c);
    if (sum) sum[c] = z_of(c);
    if (y) y[c] = yb;
    if (!a.qmax) continue;
    const float v = inv > 0.f ? __fmul_rn(norm_load<ACT>(&yb), inv) : 0.f;
    if (a.qmax == kQmaxF8) {
      a.codes[row * a.cols + c] = (int8_t)e4m3_byte(v);
    } else {
      const float q = (float)a.qmax;
      a.codes[row * a.cols + c] = (int8_t)(int)fminf(fmaxf(__builtin_rintf(v), -q), q);
    }
  }
  }
}

}  // namespace

hipError_t launch_add_rms_norm(const NormArgs& a, int act, hipStream_t s) {
  const unsigned grid = (unsigned)(a.rows < (1 << 20) ? a.rows : (1 << 20));
  if (act == MXMOE_BF16) hipLaunchKernelGGL(norm_row_kernel<MXMOE_BF16>, dim3(grid), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(norm_row_kernel<MXMOE_F16>, dim3(grid), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace mxmoe
