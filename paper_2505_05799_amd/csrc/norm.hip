// Residual addition, RMS norm and per-row 8-bit encoding in one launch.
//
//   z = round(x + residual)                         (the activation dtype)
//   r = fl32(1 / sqrt(mean(z^2) + eps))             (64-bit sum, root and quotient)
//   y = round(fl32(fl32(z r) weight))
//   codes, scale = the per-token recipe of rowquant.h on the rounded y
//
// The squares of 16-bit values are exact in 64 bits and their sum errs by some
// 2^-50 of it, so another split of a row over lanes gives another r, by one unit in its
// last place, for about one row in 2^25 only.  The codes and the scale equal act_quant of
// the rounded y for rows that are finite and whose largest |y| is 0 or at least 2^-118;
// others have scale NaN (act_quant passes over NaN) and 0.
//
// A row is read once: its elements stay in registers, 8 to a lane and chunk, and
// turn from x into z into y in place.  Rows whose pointers or strides are not
// 16-byte aligned take the same loads (global memory takes any alignment), and
// the last elements of a row of an odd length go one by one.
#include "mxmoe_internal.h"
#include "rowquant.h"

namespace mxmoe {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));

#define NORM_INL __device__ __attribute__((always_inline)) inline

// a row whose largest |y| is below this counts as zero: qmax / |y| would overflow
constexpr float kTinyAmax = 0x1p-118f;

template <int ACT> NORM_INL f32x2 unpack2(uint32_t w) {
  if constexpr (ACT == MXMOE_BF16) return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
  const f16x2 h = __builtin_bit_cast(f16x2, w);
  return f32x2{(float)h[0], (float)h[1]};
}
template <int ACT> NORM_INL uint32_t pack2(float lo, float hi) {
  if constexpr (ACT == MXMOE_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
  // (a product that was rounded to fp32 must not be fused with the conversion)
  asm("" : "+v"(lo), "+v"(hi));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, f16x2));
}

// Sum and packed 16-bit maxima over groups of L lanes (every lane ends with the
// result): DPP moves inside 16 lanes, cross-lane moves beyond.
template <int C> NORM_INL int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, C, 0xf, 0xf, true); }
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;
template <int C> NORM_INL double add_dpp(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)dpp<C>((int)(uint32_t)b), hi = (uint32_t)dpp<C>((int)(b >> 32));
  return v + __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
template <int L> NORM_INL double lanes_sum(double v) {
  if constexpr (L > 1) v = add_dpp<kXor1>(v);
  if constexpr (L > 2) v = add_dpp<kXor2>(v);
  if constexpr (L > 4) v = add_dpp<kHalfMirror>(v);
  if constexpr (L > 8) v = add_dpp<kMirror>(v);
  if constexpr (L > 16) v += __shfl_xor(v, 16, 64);
  if constexpr (L > 32) v += __shfl_xor(v, 32, 64);
  return v;
}
NORM_INL uint32_t max2(uint32_t a, uint32_t b) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int L> NORM_INL uint32_t lanes_max(uint32_t v) {
  if constexpr (L > 1) v = max2(v, (uint32_t)dpp<kXor1>((int)v));
  if constexpr (L > 2) v = max2(v, (uint32_t)dpp<kXor2>((int)v));
  if constexpr (L > 4) v = max2(v, (uint32_t)dpp<kHalfMirror>((int)v));
  if constexpr (L > 8) v = max2(v, (uint32_t)dpp<kMirror>((int)v));
  if constexpr (L > 16) v = max2(v, (uint32_t)__shfl_xor((int)v, 16, 64));
  if constexpr (L > 32) v = max2(v, (uint32_t)__shfl_xor((int)v, 32, 64));
  return v;
}

// Chunk c of a row of 16-bit values: elements 8 c .. 8 c + 7, zeros past the row.
NORM_INL u32x4 load_chunk(const uint16_t* p, int c, int cols) {
  u32x4 v = {0u, 0u, 0u, 0u};
  const int left = cols - 8 * c;
  if (left >= 8) {
    v = *reinterpret_cast<const u32x4_any*>(p + 8 * c);
  } else if (left > 0) {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < left) v[i >> 1] |= (uint32_t)p[8 * c + i] << (16 * (i & 1));
  }
  return v;
}
NORM_INL void store_chunk(uint16_t* p, int c, int cols, u32x4 v) {
  const int left = cols - 8 * c;
  if (left >= 8) {
    *reinterpret_cast<u32x4_any*>(p + 8 * c) = v;
  } else if (left > 0) {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < left) p[8 * c + i] = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
  }
}
NORM_INL void store_codes(int8_t* p, int c, int cols, u32x2 v) {
  const int left = cols - 8 * c;
  if (left >= 8) {
    *reinterpret_cast<u32x2_any*>(p + 8 * c) = v;
  } else if (left > 0) {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < left) p[8 * c + i] = (int8_t)(v[i >> 2] >> (8 * (i & 3)));
  }
}

// z of 8 elements, and the sum of their squares
template <int ACT> NORM_INL u32x4 add_chunk(u32x4 x, u32x4 r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 a = unpack2<ACT>(x[i]), b = unpack2<ACT>(r[i]);
    x[i] = pack2<ACT>(a[0] + b[0], a[1] + b[1]);
  }
  return x;
}
template <int ACT> NORM_INL double squares(u32x4 z, double ss) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 a = unpack2<ACT>(z[i]);
    ss = __builtin_fma((double)a[0], (double)a[0], ss);
    ss = __builtin_fma((double)a[1], (double)a[1], ss);
  }
  return ss;
}
template <int ACT> NORM_INL u32x4 norm_chunk(u32x4 z, u32x4 w, float r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 a = unpack2<ACT>(z[i]), g = unpack2<ACT>(w[i]);
    z[i] = pack2<ACT>(a[0] * r * g[0], a[1] * r * g[1]);
  }
  return z;
}
NORM_INL uint32_t chunk_max(u32x4 y, uint32_t mb) {
#pragma unroll
  for (int i = 0; i < 4; ++i) mb = max2(mb, y[i] & 0x7fff7fffu);
  return mb;
}
// Codes of 8 elements.  |y inv| <= qmax (1 + 2^-23) rounds to qmax at the most, so
// nothing is clamped.  int8: adding 1.5 2^23 leaves the integer nearest to the product
// (ties to even) in the low bits.  FP8: the conversion rounds to the nearest e4m3,
// ties to even; a zero loses its sign.
template <int ACT> NORM_INL u32x2 code_chunk(u32x4 y, float inv, bool f8) {
  u32x2 o;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x2 a = unpack2<ACT>(y[2 * h]), b = unpack2<ACT>(y[2 * h + 1]);
    float v[4] = {a[0] * inv, a[1] * inv, b[0] * inv, b[1] * inv};
    if (f8) {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
      const uint32_t u = (uint32_t)w;
      o[h] = u & (0x7f7f7f7fu | ((u & 0x7f7f7f7fu) + 0x7f7f7f7fu));
    } else {
      uint32_t q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        asm("" : "+v"(v[i]));  // the product is rounded before the addition
        q[i] = __float_as_uint(v[i] + 12582912.0f);
      }
      o[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[3], q[2], 0x0c0c0400u),
                                   __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u), 0x05040100u);
    }
  }
  return o;
}

struct RowScale { float inv, scale; };
// from the largest magnitude bits of y (packed pairs)
template <int ACT> NORM_INL RowScale row_scale(uint32_t mb2, int qmax) {
  const uint32_t mb = max(mb2 & 0xffffu, mb2 >> 16);
  const float amax = bits_to_f32(mb, ACT), q = (float)qmax;
  if (mb >= (ACT == MXMOE_BF16 ? 0x7f80u : 0x7c00u)) return {0.f, __builtin_nanf("")};
  if (amax < kTinyAmax) return {0.f, 0.f};
  return {__fdiv_rn(q, amax), __fdiv_rn(amax, q)};
}

// Row pointers of the call
struct RowPtrs {
  const uint16_t *x, *res;
  uint16_t *sum, *y;
  int8_t* codes;
  NORM_INL RowPtrs(const NormArgs& a, int64_t row) {
    x = reinterpret_cast<const uint16_t*>(a.x) + row * a.ldx;
    res = a.res ? reinterpret_cast<const uint16_t*>(a.res) + row * a.ldr : nullptr;
    sum = a.sum ? reinterpret_cast<uint16_t*>(a.sum) + row * a.lds : nullptr;
    y = a.y ? reinterpret_cast<uint16_t*>(a.y) + row * a.ldy : nullptr;
    codes = a.codes ? a.codes + row * (int64_t)a.cols : nullptr;
  }
};

NORM_INL float factor(double ss, const NormArgs& a) { return (float)(1.0 / __builtin_sqrt(ss / (double)a.cols + a.eps)); }

// Rows in registers.  L < 64 (NC = W = 1): a wavefront takes 64 / L rows of at most
// 8 L elements.  L = 64, W = 1: a wavefront per row; W > 1: a workgroup of W
// wavefronts per row.  NC: chunks of a lane.
template <int ACT, int L, int NC, int W>
__global__ void __launch_bounds__(W == 1 ? 256 : 64 * W) norm_kernel(NormArgs a) {
  __shared__ double red[W];
  __shared__ uint32_t redm[W];
  constexpr int kLanes = L * W;                              // lanes of a row
  constexpr int kRows = (W == 1 ? 256 : 64 * W) / kLanes;    // rows of a workgroup
  const int tid = threadIdx.x, idx = tid % kLanes, w = tid >> 6;
  const uint16_t* g = reinterpret_cast<const uint16_t*>(a.weight);
  for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < a.rows; r0 += (int64_t)gridDim.x * kRows) {
    const int64_t row = r0 + tid / kLanes;
    const bool live = row < a.rows;  // (lanes of no row go along: the cross-lane moves take whole groups)
    const int cols = live ? a.cols : 0;
    const RowPtrs p(a, live ? row : 0);
    u32x4 v[NC], gv[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) v[i] = load_chunk(p.x, idx + kLanes * i, cols);
    if (p.res) {
      u32x4 rv[NC];
#pragma unroll
      for (int i = 0; i < NC; ++i) rv[i] = load_chunk(p.res, idx + kLanes * i, cols);
#pragma unroll
      for (int i = 0; i < NC; ++i) gv[i] = load_chunk(g, idx + kLanes * i, cols);
#pragma unroll
      for (int i = 0; i < NC; ++i) v[i] = add_chunk<ACT>(v[i], rv[i]);
    } else {
#pragma unroll
      for (int i = 0; i < NC; ++i) gv[i] = load_chunk(g, idx + kLanes * i, cols);
    }
    double ss = 0.0;
#pragma unroll
    for (int i = 0; i < NC; ++i) ss = squares<ACT>(v[i], ss);
    ss = lanes_sum<L>(ss);
    if constexpr (W > 1) {
      if ((tid & 63) == 0) red[w] = ss;
      __syncthreads();
      ss = red[0];
#pragma unroll
      for (int i = 1; i < W; ++i) ss += red[i];
    }
    if (p.sum) {
#pragma unroll
      for (int i = 0; i < NC; ++i) store_chunk(p.sum, idx + kLanes * i, cols, v[i]);
    }
    const float r = factor(ss, a);
    uint32_t mb = 0u;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      v[i] = norm_chunk<ACT>(v[i], gv[i], r);
      mb = chunk_max(v[i], mb);
    }
    if (a.qmax) {
      // (a NaN factor makes NaN of the zeros past the row, too: then the row has NaN itself)
      mb = lanes_max<L>(mb);
      if constexpr (W > 1) {
        if ((tid & 63) == 0) redm[w] = mb;
        __syncthreads();
        mb = redm[0];
#pragma unroll
        for (int i = 1; i < W; ++i) mb = max2(mb, redm[i]);
      }
      const RowScale s = row_scale<ACT>(mb, a.qmax);
      if (idx == 0 && live) a.scales[row] = s.scale;
      const bool f8 = a.qmax == kQmaxF8;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const u32x2 q = s.inv > 0.f ? code_chunk<ACT>(v[i], s.inv, f8) : u32x2{0u, 0u};
        store_codes(p.codes, idx + kLanes * i, cols, q);
      }
    }
    if (p.y) {
#pragma unroll
      for (int i = 0; i < NC; ++i) store_chunk(p.y, idx + kLanes * i, cols, v[i]);
    }
    if constexpr (W > 1) __syncthreads();  // red and redm are read before the next row's
  }
}

// Rows beyond the registers: a workgroup of 16 wavefronts per row reads it for the
// sum, for the largest magnitude and for the codes.  Where the sum is stored it is
// what the later steps read (each thread its own elements), so that it may take
// the place of an input.
template <int ACT>
__global__ void __launch_bounds__(1024) norm_long_kernel(NormArgs a) {
  __shared__ double red[16];
  __shared__ uint32_t redm[16];
  const int tid = threadIdx.x, w = tid >> 6, cols = a.cols, nch = (cols + 7) / 8;
  const uint16_t* g = reinterpret_cast<const uint16_t*>(a.weight);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const RowPtrs p(a, row);
    auto z_of = [&](int c) {
      if (p.sum) return load_chunk(p.sum, c, cols);
      const u32x4 x = load_chunk(p.x, c, cols);
      return p.res ? add_chunk<ACT>(x, load_chunk(p.res, c, cols)) : x;
    };
    double ss = 0.0;
    for (int c = tid; c < nch; c += 1024) {
      u32x4 z = load_chunk(p.x, c, cols);
      if (p.res) z = add_chunk<ACT>(z, load_chunk(p.res, c, cols));
      if (p.sum) store_chunk(p.sum, c, cols, z);
      ss = squares<ACT>(z, ss);
    }
    ss = lanes_sum<64>(ss);
    if ((tid & 63) == 0) red[w] = ss;
    __syncthreads();
    ss = red[0];
    for (int i = 1; i < 16; ++i) ss += red[i];
    const float r = factor(ss, a);
    RowScale s{0.f, 0.f};
    if (a.qmax) {
      uint32_t mb = 0u;
      for (int c = tid; c < nch; c += 1024) mb = chunk_max(norm_chunk<ACT>(z_of(c), load_chunk(g, c, cols), r), mb);
      mb = lanes_max<64>(mb);
      if ((tid & 63) == 0) redm[w] = mb;
      __syncthreads();
      mb = redm[0];
      for (int i = 1; i < 16; ++i) mb = max2(mb, redm[i]);
      s = row_scale<ACT>(mb, a.qmax);
      if (tid == 0) a.scales[row] = s.scale;
    }
    for (int c = tid; c < nch; c += 1024) {
      const u32x4 y = norm_chunk<ACT>(z_of(c), load_chunk(g, c, cols), r);
      if (a.qmax) store_codes(p.codes, c, cols, s.inv > 0.f ? code_chunk<ACT>(y, s.inv, a.qmax == kQmaxF8) : u32x2{0u, 0u});
      if (p.y) store_chunk(p.y, c, cols, y);
    }
    __syncthreads();
  }
}

constexpr int64_t kMaxGrid = 1 << 20;

template <int ACT, int L, int NC, int W> hipError_t go(const NormArgs& a, hipStream_t s) {
  constexpr int threads = W == 1 ? 256 : 64 * W, rows = threads / (L * W);
  const int64_t grid = ((int64_t)a.rows + rows - 1) / rows;
  hipLaunchKernelGGL((norm_kernel<ACT, L, NC, W>), dim3((unsigned)(grid < kMaxGrid ? grid : kMaxGrid)), dim3(threads), 0, s, a);
  return hipGetLastError();
}

// Lanes of a row.  Few rows: a chunk to a lane, so that one trip to memory brings the
// row and the reductions end it (one row of 7168: 4.0 us a launch in a graph, 24.8 with
// an element to a thread and step).  Many: more chunks to a lane, fewer lanes that meet,
// up to 4096 elements without a barrier.  us few / many: 2048 elements, 2048 rows
// 9.0 / 9.5, 4096 14.4 / 12.6, 16384 54.0 / 50.7; 8192 elements, 256 rows 6.1 / 6.4,
// 512 10.8 / 9.7, 4096 75.0 / 51.5 (5.9 TB/s).  16384 x 3584 with FP8 rows: 100 us,
// 5.3 TB/s, against 4.7 of a copy of 4 GB: bound by memory.
template <int ACT> hipError_t launch(const NormArgs& a, hipStream_t s) {
  const int nch = (a.cols + 7) / 8, waves = (nch + 63) / 64;
  if (nch <= 8) return go<ACT, 8, 1, 1>(a, s);
  if (nch <= 16) return go<ACT, 16, 1, 1>(a, s);
  if (nch <= 32) return go<ACT, 32, 1, 1>(a, s);
  if (waves == 1) return go<ACT, 64, 1, 1>(a, s);
  if (a.rows >= 4096 && waves <= 8) {
    if (waves <= 2) return go<ACT, 64, 2, 1>(a, s);
    if (waves <= 4) return go<ACT, 64, 4, 1>(a, s);
    return go<ACT, 64, 8, 1>(a, s);
  }
  if (a.rows >= 512 && waves > 8 && waves <= 32) {
    if (waves <= 16) return go<ACT, 64, 4, 4>(a, s);
    return go<ACT, 64, 8, 4>(a, s);
  }
  if (waves <= 2) return go<ACT, 64, 1, 2>(a, s);
  if (waves <= 4) return go<ACT, 64, 1, 4>(a, s);
  if (waves <= 8) return go<ACT, 64, 1, 8>(a, s);
  if (waves <= 16) return go<ACT, 64, 1, 16>(a, s);
  if (waves <= 32) return go<ACT, 64, 2, 16>(a, s);
  if (waves <= 64) return go<ACT, 64, 4, 16>(a, s);
  const int64_t grid = a.rows;
  hipLaunchKernelGGL(norm_long_kernel<ACT>, dim3((unsigned)(grid < kMaxGrid ? grid : kMaxGrid)), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_add_rms_norm(const NormArgs& a, int act, hipStream_t s) {
  return act == MXMOE_BF16 ? launch<MXMOE_BF16>(a, s) : launch<MXMOE_F16>(a, s);
}

}  // namespace mxmoe
