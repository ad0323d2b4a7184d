// Quantisation to 8-bit floating point with a scale for each block of 128.
//
// For a block with largest finite magnitude a and the format's largest value
// t (448 or 57344):
//   scale S = 1 if a = 0, else max(fl32(a / t), 2^-126), or with scales in
//   powers of two the least 2^E >= a / t, E >= -126;
//   value Q = the format's nearest value to the exact quotient x / S, ties to
//   even. |x / S| <= t (1 + 2^-24), which rounds to t, so nothing saturates.
//   NaN stays NaN; an infinity is NaN in e4m3, which has none, and itself in
//   e5m2.
// One block of 256 threads takes 128 x 128 elements of X, held in registers
// from one read of X, whichever of the two directions are wanted. Memory
// bound: the bytes are X once and each output once.
#include "f8_round.hpp"

namespace ozfp4 {
namespace {

constexpr int kTLd = 128 + 8;   // bytes from column to column of the transposed tile in LDS

// Thread t holds columns 8 (t % 16) .. + 7 of rows 8 (t / 16) .. + 7: a row's
// 128 columns are 16 neighbouring lanes, a wave has 32 rows.
template <int kSrc, bool kPow2, int kFmt>
__global__ __launch_bounds__(256) void k_f8_quantize(F8Quantize p, unsigned tiles_c) {
  typedef typename Source<kSrc>::T T;
  __shared__ __align__(16) uint8_t turned[128 * kTLd];
  __shared__ float colmax[4][128];
  __shared__ float tilemax[4];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int cg = t & 15, rg = t >> 4;
  const unsigned tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
  const int64_t row0 = (int64_t)tr * 128 + rg * 8, col0 = (int64_t)tc * 128 + cg * 8;

  float x[8][8];
  const T* src = static_cast<const T*>(p.x) + row0 * p.ldx + col0;
  const bool whole = col0 + 8 <= p.cols;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool in = row0 + i < p.rows;
    if (in && whole) {
      T v[8];
      __builtin_memcpy(v, src + i * p.ldx, sizeof(v));
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = widen(v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = in && col0 + j < p.cols ? widen(src[i * p.ldx + j]) : 0.0f;
    }
  }

  float rowmax[8], cmax[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rowmax[i] = cmax[i] = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = finite_abs(x[i][j]);
      rowmax[i] = __builtin_fmaxf(rowmax[i], a);
      cmax[j] = __builtin_fmaxf(cmax[j], a);
    }
  if (p.tile) {
    float a = rowmax[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) a = __builtin_fmaxf(a, rowmax[i]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) a = __builtin_fmaxf(a, __shfl_xor(a, d));
    if (lane == 0) tilemax[wave] = a;
    __syncthreads();
    a = __builtin_fmaxf(__builtin_fmaxf(tilemax[0], tilemax[1]), __builtin_fmaxf(tilemax[2], tilemax[3]));
#pragma unroll
    for (int i = 0; i < 8; ++i) rowmax[i] = cmax[i] = a;
    if (t == 0) {
      if (p.q1) store_scale<kPow2, kFmt>(p.s1, tr * p.s1l + tc * p.s1k, a);
      if (p.q0) store_scale<kPow2, kFmt>(p.s0, tc * p.s0l + tr * p.s0k, a);
    }
  } else {
    if (p.q1) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int d = 1; d < 16; d *= 2) rowmax[i] = __builtin_fmaxf(rowmax[i], __shfl_xor(rowmax[i], d));
      if (cg < 8 && row0 + cg < p.rows) {   // lane cg of the row's sixteen stores row cg
        float a = rowmax[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) a = cg == i ? rowmax[i] : a;
        store_scale<kPow2, kFmt>(p.s1, (row0 + cg) * p.s1l + (int64_t)tc * p.s1k, a);
      }
    }
    if (p.q0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        cmax[j] = __builtin_fmaxf(cmax[j], __shfl_xor(cmax[j], 16));
        cmax[j] = __builtin_fmaxf(cmax[j], __shfl_xor(cmax[j], 32));
      }
      if (lane < 16)
#pragma unroll
        for (int j = 0; j < 8; ++j) colmax[wave][cg * 8 + j] = cmax[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = cg * 8 + j;
        cmax[j] = __builtin_fmaxf(__builtin_fmaxf(colmax[0][c], colmax[1][c]),
                                  __builtin_fmaxf(colmax[2][c], colmax[3][c]));
      }
      if (t < 128 && (int64_t)tc * 128 + t < p.cols) {
        const float a = __builtin_fmaxf(__builtin_fmaxf(colmax[0][t], colmax[1][t]),
                                        __builtin_fmaxf(colmax[2][t], colmax[3][t]));
        store_scale<kPow2, kFmt>(p.s0, ((int64_t)tc * 128 + t) * p.s0l + (int64_t)tr * p.s0k, a);
      }
    }
  }

  if (p.q1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Scale s = make_scale<kPow2, kFmt>(rowmax[i]);
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = quotient<kPow2>(x[i][j], s);
      const uint2 w = {pack4<kFmt>(v[0], v[1], v[2], v[3]), pack4<kFmt>(v[4], v[5], v[6], v[7])};
      if (row0 + i < p.rows && col0 < p.cols)   // the line's padding to 16 takes what is behind cols
        *reinterpret_cast<uint2*>(p.q1 + (row0 + i) * p.ld1 + col0) = w;
    }
  }
  if (p.q0) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const Scale s = make_scale<kPow2, kFmt>(cmax[j]);
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = quotient<kPow2>(x[i][j], s);
      const uint2 w = {pack4<kFmt>(v[0], v[1], v[2], v[3]), pack4<kFmt>(v[4], v[5], v[6], v[7])};
      *reinterpret_cast<uint2*>(turned + (cg * 8 + j) * kTLd + rg * 8) = w;
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int c = n * 32 + (t >> 3), piece = (t & 7) * 16;
      const int64_t col = (int64_t)tc * 128 + c, row = (int64_t)tr * 128 + piece;
      if (col < p.cols && row < p.rows) {
        const uint2 a = *reinterpret_cast<const uint2*>(turned + c * kTLd + piece);
        const uint2 b = *reinterpret_cast<const uint2*>(turned + c * kTLd + piece + 8);
        *reinterpret_cast<uint4*>(p.q0 + col * p.ld0 + row) = uint4{a.x, a.y, b.x, b.y};
      }
    }
  }
}

template <int kSrc, bool kPow2>
hipError_t launch(hipStream_t st, const F8Quantize& q, int64_t tr, int64_t tc) {
  const dim3 grid((unsigned)(tr * tc));
  if (q.fmt == OZFP4_E4M3)
    hipLaunchKernelGGL((k_f8_quantize<kSrc, kPow2, OZFP4_E4M3>), grid, dim3(256), 0, st, q, (unsigned)tc);
  else
    hipLaunchKernelGGL((k_f8_quantize<kSrc, kPow2, OZFP4_E5M2>), grid, dim3(256), 0, st, q, (unsigned)tc);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_f8_quantize(hipStream_t st, const F8Quantize& q) {
  const int64_t tr = (q.rows + 127) / 128, tc = (q.cols + 127) / 128;
  if (tr * tc == 0) return hipSuccess;
  switch (q.src) {
    case OZFP4_F32: return q.pow2 ? launch<OZFP4_F32, true>(st, q, tr, tc) : launch<OZFP4_F32, false>(st, q, tr, tc);
    case OZFP4_BF16:
      return q.pow2 ? launch<OZFP4_BF16, true>(st, q, tr, tc) : launch<OZFP4_BF16, false>(st, q, tr, tc);
    default: return q.pow2 ? launch<OZFP4_F16, true>(st, q, tr, tc) : launch<OZFP4_F16, false>(st, q, tr, tc);
  }
}

}  // namespace ozfp4
