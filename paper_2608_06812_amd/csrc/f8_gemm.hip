// Matrix product of block-scaled 8-bit operands:
//   C(p, q) = sum_b sP(p, b) sQ(q, b) sum_{k in b} P(p, k) Q(q, k)
// over blocks b of 128, in FP32 (see f8_device.hpp for the two ways to the inner sums).
// With scales in powers of two the whole sum stays in the matrix cores: an E8M0
// scale is an operand of the 8-bit instruction, or of the conversion to BF16.
// An FP32 scale multiplies a block's sum on its way into the FP32 accumulator.
#include "f8_device.hpp"

namespace ozfp4 {
namespace {

// Four adjacent elements of C from line p on; n of them exist.
__device__ __forceinline__ void store4(const F8Gemm& g, int64_t at, v4f v, int n) {
  if (g.type == OZFP4_F32) {
    float* c = static_cast<float*>(g.C) + at;
    if (n >= 4 && g.vec) {
      v4f* c4 = reinterpret_cast<v4f*>(c);
      *c4 = g.accumulate ? *c4 + v : v;
    } else {
      for (int e = 0; e < 4; ++e)
        if (e < n) c[e] = g.accumulate ? c[e] + v[e] : v[e];
    }
    return;
  }
  uint32_t w[2];
  if (g.type == OZFP4_BF16) {
    typedef __bf16 h4 __attribute__((ext_vector_type(4)));
    const h4 h = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    __builtin_memcpy(w, &h, 8);
  } else {
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    const h4 h = {(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
    __builtin_memcpy(w, &h, 8);
  }
  uint16_t* c = static_cast<uint16_t*>(g.C) + at;
  if (n >= 4 && g.vec)
    *reinterpret_cast<uint2*>(c) = uint2{w[0], w[1]};
  else
    for (int e = 0; e < 4; ++e)
      if (e < n) c[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
}

// Block tile (WP TP 16) lines of P x (WQ TQ 16) of Q, a wave TP x TQ MFMA
// tiles. A stage is one block of 128 of every line, 128 bytes a line, copied
// into LDS by buffer-form LDS DMA into kSlots slots, kSlots - 1 stages ahead. A
// copy is 8 lines; within a line the 16-byte piece c lies at c ^ (line % 8),
// which the copy's lanes arrange by the addresses they read, so that the lines
// of an operand read fall on different banks. The scales of a stage, one word a
// line, go through registers into LDS beside them.
template <bool kExact, int kMode, int FP, int FQ, int WP, int WQ, int TP, int TQ, int kSlots>
__global__ __launch_bounds__(WP * WQ * 64) void k_f8_gemm(F8Gemm g, unsigned tiles_p, unsigned tiles_q) {
  constexpr int kThreads = WP * WQ * 64, kWavesN = WP * WQ;
  constexpr int BP = WP * TP * 16, BQ = WQ * TQ * 16, kLines = BP + BQ;
  constexpr int kBytes = kLines * kF8Block;
  constexpr int CP = BP / 8 / kWavesN, CQ = BQ / 8 / kWavesN, kCopies = CP + CQ;   // per wave and stage
  static_assert(BP % (8 * kWavesN) == 0 && BQ % (8 * kWavesN) == 0, "whole copies a wave");
  static_assert(kLines <= kThreads, "a thread a line's scale");
  static_assert(kSlots == 2 || kSlots == 3, "the wait at a stage's top");
  __shared__ __align__(1024) uint8_t lds[kSlots * kBytes];
  __shared__ uint32_t scale[2][kLines];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wp = wave / WQ, wq = wave % WQ;
  int range;
  int64_t tp, tq;
  tile_coords(blockIdx.x, gridDim.x, tiles_p, tiles_q, &range, &tp, &tq);
  const int64_t p0 = tp * BP, q0 = tq * BQ;
  const int total = (int)((g.k + kF8Block - 1) / kF8Block);
  const int first = range * g.stages, nst = min(g.stages, total - first);
  const int tail = (int)(g.k - (int64_t)(total - 1) * kF8Block);   // k values of the last stage

  // this wave's copies: lines wave * C * 8 + 8 j + lane / 8 of each operand.
  // Lines behind the last are read as the last (their results are not stored),
  // pieces behind a line's end as its first, and cleared in LDS.
  const uint32_t piece = (uint32_t)((lane & 7) ^ (lane >> 3)) * 16;
  auto lines_from = [&](const F8Lines& l, int64_t line) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(l.x + line * l.ld), (short)0, -1, kBufferWord3);
  };
  const __amdgpu_buffer_rsrc_t from_p = lines_from(g.P, p0), from_q = lines_from(g.Q, q0);
  const uint32_t ldp = (uint32_t)g.P.ld, ldq = (uint32_t)g.Q.ld;
  const uint32_t last_p = (uint32_t)min(g.P.lines - 1 - p0, (int64_t)BP - 1) * ldp;
  const uint32_t last_q = (uint32_t)min(g.Q.lines - 1 - q0, (int64_t)BQ - 1) * ldq;
  const uint32_t own_p = (uint32_t)(wave * CP * 8 + (lane >> 3)) * ldp;
  const uint32_t own_q = (uint32_t)(wave * CQ * 8 + (lane >> 3)) * ldq;
  auto copy = [&](int s) {
    const int st = first + s;
    const uint32_t at = st == total - 1 && (int)piece >= tail ? 0 : piece;
    uint8_t* to = lds + (s % kSlots) * kBytes;
#pragma unroll
    for (int j = 0; j < CP; ++j)
      dma16_buf(from_p, min(own_p + j * 8 * ldp, last_p) + at, (uint32_t)st * kF8Block, to + (wave * CP + j) * 1024);
#pragma unroll
    for (int j = 0; j < CQ; ++j)
      dma16_buf(from_q, min(own_q + j * 8 * ldq, last_q) + at, (uint32_t)st * kF8Block,
                to + (BP / 8 + wave * CQ + j) * 1024);
  };

  // this thread's scale
  const bool scaling = tid < kLines;
  const bool sp_of = tid < BP;
  const F8Lines& sl = sp_of ? g.P : g.Q;
  const int64_t sline = min(sp_of ? p0 + tid : q0 + (tid - BP), sl.lines - 1) >> sl.shift;
  auto load_scale = [&](int s) -> uint32_t {
    if (!scaling || s >= nst) return 0;
    const int64_t at = sline * sl.sl + (int64_t)(first + s) * sl.sk;
    if constexpr (kMode == kPow2) return static_cast<const uint8_t*>(sl.s)[at];
    return static_cast<const uint32_t*>(sl.s)[at];
  };

  v4f acc[TP][TQ];
#pragma unroll
  for (int i = 0; i < TP; ++i)
#pragma unroll
    for (int j = 0; j < TQ; ++j) acc[i][j] = v4f{0, 0, 0, 0};

  uint32_t sc = load_scale(0);
  if (scaling) scale[0][tid] = sc;
  sc = load_scale(1);
  if (nst > 0) copy(0);
  if (kSlots == 3 && nst > 1) copy(1);

  // operand reads: line r = lane % 16 of a tile, pieces 2 (lane / 16) and the
  // next one (any order of k will do, as long as both operands have it)
  const int r = lane & 15, h = (lane >> 4) * 2;
  const int o0 = r * 128 + ((h ^ (r & 7)) * 16), o1 = r * 128 + (((h + 1) ^ (r & 7)) * 16);

  for (int s = 0; s < nst; ++s) {
    // stage s has landed (and the scales of stage s + 1), and every wave has
    // done with the slot that the next copies go to
    if (kSlots == 3 && s + 1 < nst)
      wait_vm_lgkm0<kCopies>();
    else
      wait_vm_lgkm0<0>();
    block_sync();
    if (scaling) scale[(s + 1) & 1][tid] = sc;
    if (s + 2 < nst) sc = load_scale(s + 2);
    if (s + kSlots - 1 < nst) copy(s + kSlots - 1);
    uint8_t* sb = lds + (s % kSlots) * kBytes;
    if (first + s == total - 1 && tail < kF8Block) {
      // zeros behind the end of the lines
      for (int l = tid; l < kLines; l += kThreads)
        for (int c = tail / 16; c < 8; ++c) {
          uint32_t* w = reinterpret_cast<uint32_t*>(sb + l * 128 + ((c ^ (l & 7)) * 16));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int keep = tail - (c * 16 + e * 4);
            w[e] = keep >= 4 ? w[e] : keep <= 0 ? 0 : w[e] & ((1u << (8 * keep)) - 1);
          }
        }
      wait_vm_lgkm0<0>();
      block_sync();
    }
    const uint32_t* ss = scale[s & 1];
    const uint8_t* pb = sb + wp * TP * 2048;
    const uint8_t* qb = sb + (BP + wq * TQ * 16) * 128;
    auto read = [&](const uint8_t* b) {
      const v4i x = *reinterpret_cast<const v4i*>(b + o0), y = *reinterpret_cast<const v4i*>(b + o1);
      return v8i{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    };
    constexpr uint32_t one = 127;   // E8M0 1
    Frag<kExact> q[TQ];
    uint32_t sq[TQ];
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
      sq[j] = ss[BP + (wq * TQ + j) * 16 + r];
      q[j] = Frag<kExact>::template make<FQ>(read(qb + j * 2048), kMode == kPow2 ? sq[j] : one);
    }
    if constexpr (kMode == kTileP) {
      const float a = __uint_as_float(ss[wp * TP * 16]);
#pragma unroll
      for (int j = 0; j < TQ; ++j) sq[j] = __float_as_uint(a * __uint_as_float(sq[j]));
    }
#pragma unroll
    for (int i = 0; i < TP; ++i) {
      uint32_t e8 = one;
      if constexpr (kMode == kPow2) e8 = ss[(wp * TP + i) * 16 + r];
      const auto p = Frag<kExact>::template make<FP>(read(pb + i * 2048), e8);
      v4f sp = {1, 1, 1, 1};
      if constexpr (kMode == kLineP)
        sp = *reinterpret_cast<const v4f*>(ss + (wp * TP + i) * 16 + (lane >> 4) * 4);
#pragma unroll
      for (int j = 0; j < TQ; ++j) {
        if constexpr (kMode == kPow2) {
          acc[i][j] = block_product<true, FP, FQ>(p, q[j], acc[i][j], e8, sq[j]);
        } else {
          const v4f c = block_product<false, FP, FQ>(p, q[j], v4f{0, 0, 0, 0}, 0, 0);
          const float f = __uint_as_float(sq[j]);
#pragma unroll
          for (int v = 0; v < 4; ++v)
            acc[i][j][v] = __builtin_fmaf(kMode == kLineP ? c[v] * sp[v] : c[v], f, acc[i][j][v]);
        }
      }
    }
  }

#pragma unroll
  for (int j = 0; j < TQ; ++j) {
    const int64_t q = q0 + (wq * TQ + j) * 16 + r;
    if (q >= g.Q.lines) continue;
#pragma unroll
    for (int i = 0; i < TP; ++i) {
      const int64_t p = p0 + (wp * TP + i) * 16 + (lane >> 4) * 4;
      const int64_t n = g.P.lines - p;
      if (n > 0) store4(g, (int64_t)range * g.part + q * g.ldc + p, acc[i][j], n < 4 ? (int)n : 4);
    }
  }
}

template <bool kExact, int kMode, int FP, int FQ, int WP, int WQ, int TP, int TQ, int kSlots>
hipError_t launch_tile(hipStream_t st, const F8Gemm& g) {
  const int64_t tiles_p = (g.P.lines + WP * TP * 16 - 1) / (WP * TP * 16);
  const int64_t tiles_q = (g.Q.lines + WQ * TQ * 16 - 1) / (WQ * TQ * 16);
  const int64_t total = (g.k + kF8Block - 1) / kF8Block,
                ranges = total > g.stages ? (total + g.stages - 1) / g.stages : 1;
  hipLaunchKernelGGL((k_f8_gemm<kExact, kMode, FP, FQ, WP, WQ, TP, TQ, kSlots>), dim3((unsigned)(tiles_p * tiles_q * ranges)),
                     dim3(WP * WQ * 64), 0, st, g, (unsigned)tiles_p, (unsigned)tiles_q);
  return hipGetLastError();
}

template <bool kExact, int kMode, int FP, int FQ>
hipError_t launch_size(hipStream_t st, const F8Gemm& g) {
  const int64_t big = ((g.P.lines + 255) / 256) * ((g.Q.lines + 255) / 256);
  if (big >= 192) {
    if constexpr (kExact) return launch_tile<kExact, kMode, FP, FQ, 4, 2, 4, 4, 3>(st, g);
    else return launch_tile<kExact, kMode, FP, FQ, 2, 4, 8, 4, 2>(st, g);
  }
  return launch_tile<kExact, kMode, FP, FQ, 2, 2, 4, 4, 2>(st, g);
}

template <bool kExact, int FP, int FQ>
hipError_t launch_mode(hipStream_t st, const F8Gemm& g) {
  if (g.pow2) return launch_size<kExact, kPow2, FP, FQ>(st, g);
  if (g.P.shift) return launch_size<kExact, kTileP, FP, FQ>(st, g);
  return launch_size<kExact, kLineP, FP, FQ>(st, g);
}

template <int FP, int FQ>
hipError_t launch_formats(hipStream_t st, const F8Gemm& g) {
  return g.type == OZFP4_F32 ? launch_mode<true, FP, FQ>(st, g) : launch_mode<false, FP, FQ>(st, g);
}

}  // namespace

hipError_t launch_f8_gemm(hipStream_t st, const F8Gemm& g) {
  switch (g.P.fmt * 2 + g.Q.fmt) {
    case 0: return launch_formats<0, 0>(st, g);
    case 1: return launch_formats<0, 1>(st, g);
    case 2: return launch_formats<1, 0>(st, g);
    default: return launch_formats<1, 1>(st, g);
  }
}

}  // namespace ozfp4
