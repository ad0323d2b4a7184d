// Product of block-scaled 8-bit operands where one has few lines (the tokens of
// a decoding step): memory bound, the bytes of the many lines (the weights)
// once. No LDS and no barrier between the weights and the matrix cores: a wave
// reads its operands straight into registers, with several blocks of 128 in
// flight, and the waves of a block take the blocks of 128 of the same 16 lines
// in turn, so that together they read up to 1 KiB of a line at a time and the
// chip has work from a few thousand lines on. Their sums meet in LDS at the end,
// in a fixed order.
//
// The values go to BF16 in registers whatever the output's type: the matrix
// cores have nothing to wait for here, and the formats need no variants.
//
// For up to 16 tokens of few values the product can take the tokens as they
// are (bfloat16, float16, float32): every block quantises all of them for
// itself, into LDS, while its first weights are on their way.
#include <type_traits>

#include "f8_device.hpp"
#include "f8_round.hpp"

namespace ozfp4 {
namespace {

constexpr int kTokWaves = 8;

// The 32 values of lane group g in a block: 16-byte pieces g and g + 4, from
// aligned lines (every line at a multiple of 4 bytes) or, kAny, any others.
template <bool kAny> struct Values;
template <> struct Values<false> {
  v4i v[2];
  __device__ __forceinline__ void load(int h, const uint8_t* p) {
    __builtin_memcpy(&v[h], __builtin_assume_aligned(p, 4), 16);
  }
  __device__ __forceinline__ void set(int h, v4i x) { v[h] = x; }
  __device__ __forceinline__ v8i get() const {
    return v8i{v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
  }
};
template <> struct Values<true> {
  Dwords v[2];
  __device__ __forceinline__ void load(int h, const uint8_t* p) { v[h] = load_dwords(p); }
  __device__ __forceinline__ void set(int h, v4i x) { v[h] = Dwords{x, 0, 0}; }
  __device__ __forceinline__ v8i get() const {
    const v4i a = v[0].bytes(), b = v[1].bytes();
    return v8i{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  }
};

// Those of the block that starts at byte `at` of a line, of which `left` bytes
// exist (kWhole: all).
template <bool kWhole, bool kAny>
__device__ __forceinline__ void load_block(Values<kAny>& v, const uint8_t* line, int64_t at, int g, int left) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int c = (g + 4 * h) * 16;
    const uint8_t* p = line + at + c;
    if (kWhole || c + 16 <= left)
      v.load(h, p);
    else
      v.set(h, load_end(line, p, left - c));
  }
}

template <bool kPow2>
__device__ __forceinline__ uint32_t load_scale(const F8Lines& l, int64_t line, int64_t block) {
  const int64_t at = (line >> l.shift) * l.sl + block * l.sk;
  if constexpr (kPow2) return static_cast<const uint8_t*>(l.s)[at];
  return static_cast<const uint32_t*>(l.s)[at];
}

__device__ __forceinline__ Frag<true> to_bf16(v8i w, uint32_t e8, int fmt) {
  return fmt == OZFP4_E4M3 ? Frag<true>::make<OZFP4_E4M3>(w, e8) : Frag<true>::make<OZFP4_E5M2>(w, e8);
}

// The tokens, quantised into LDS: block b of token i at u = b m + i, 128 bytes
// whose 16-byte piece c lies at c ^ (i % 8), and its scale behind them all.
// Sixteen lanes a block of 128, eight values a lane.
template <bool kPow, int kFmt, int kSrc>
__device__ __forceinline__ void quantize_tokens(const F8Token& t, int m, int total, uint8_t* lds, uint32_t* scales) {
  typedef typename Source<kSrc>::T T;
  const int tid = threadIdx.x, r = tid & 15, count = m * total;
  for (int u = tid >> 4; u < count; u += kTokWaves * 4) {
    const int b = u / m, i = u - b * m;
    const int64_t col = (int64_t)b * kF8Block + r * 8;
    const T* src = static_cast<const T*>(t.x) + i * t.ldx + col;
    float x[8], a = 0.0f;
    load8(src, t.k - col, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) a = __builtin_fmaxf(a, finite_abs(x[e]));
#pragma unroll
    for (int d = 1; d < 16; d *= 2) a = __builtin_fmaxf(a, __shfl_xor(a, d));
    const Scale s = make_scale<kPow, kFmt>(a);
    *reinterpret_cast<uint2*>(lds + u * 128 + (((r >> 1) ^ (i & 7)) * 16) + (r & 1) * 8) =
        pack8<kPow, true, kFmt>(x, s);
    if (r == 0) {
      if constexpr (kPow)
        scales[u] = (uint32_t)(scale_exp<kFmt>(a) + 127);
      else
        scales[u] = __float_as_uint(scale_f32<kFmt>(a));
    }
  }
}

// A block: 16 TP lines of P, all lines of Q (16 TQ at most). The tokens are
// the rows of the matrix instruction and the lines of P its columns, so that a
// lane needs one scale of P a tile, whether that is a line's or a tile's.
template <bool kPow, bool kAny, int TP, int TQ, int kSrc>
__global__ __launch_bounds__(kTokWaves * 64, TP + TQ == 2 ? 4 : 2) void k_f8_token(F8Token t) {
  constexpr bool kFused = kSrc >= 0;
  constexpr int kDeep = 2;              // blocks of 128 in flight in a wave
  constexpr int kOut = 256 * TP * TQ;
  constexpr int kSum = kTokWaves * kOut * 4, kHold = kFused ? kF8TokenBlocks * (128 + 4) : 0;
  __shared__ __align__(16) uint8_t lds[kSum > kHold ? kSum : kHold];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int64_t p0 = (int64_t)blockIdx.x * (16 * TP);
  const int total = (int)((t.k + kF8Block - 1) / kF8Block);
  const int tail = (int)(t.k - (int64_t)(total - 1) * kF8Block);
  const int m = (int)t.Q.lines;
  uint32_t* held = reinterpret_cast<uint32_t*>(lds + kF8TokenBlocks * 128);

  // this lane's lines; those behind the last are read as the last
  int64_t lp[TP];
  const uint8_t* px[TP];
#pragma unroll
  for (int i = 0; i < TP; ++i) {
    lp[i] = min(p0 + i * 16 + r, t.P.lines - 1);
    px[i] = t.P.x + lp[i] * t.P.ld;
  }
  int lq[TQ];
  const uint8_t* qx[TQ];
#pragma unroll
  for (int j = 0; j < TQ; ++j) {
    lq[j] = min(j * 16 + r, m - 1);
    qx[j] = t.Q.x + lq[j] * t.Q.ld;
  }

  struct Stage {
    Values<kAny> p[TP], q[TQ];
    uint32_t sp[TP], sq[TQ];
  };
  auto fetch = [&](int s, Stage& f) {
    const int64_t at = (int64_t)s * kF8Block;
    auto blocks = [&](auto whole, int left) {
#pragma unroll
      for (int i = 0; i < TP; ++i) load_block<decltype(whole)::value>(f.p[i], px[i], at, g, left);
      if constexpr (!kFused) {
#pragma unroll
        for (int j = 0; j < TQ; ++j) load_block<decltype(whole)::value>(f.q[j], qx[j], at, g, left);
      }
    };
    if (s == total - 1 && tail < kF8Block)
      blocks(std::false_type{}, tail);
    else
      blocks(std::true_type{}, kF8Block);
#pragma unroll
    for (int i = 0; i < TP; ++i) f.sp[i] = load_scale<kPow>(t.P, lp[i], s);
    if constexpr (!kFused) {
#pragma unroll
      for (int j = 0; j < TQ; ++j) f.sq[j] = load_scale<kPow>(t.Q, lq[j], s);
    }
  };

  Stage st[kDeep];
#pragma unroll
  for (int d = 0; d < kDeep; ++d)
    if (wave + d * kTokWaves < total) fetch(wave + d * kTokWaves, st[d]);

  if constexpr (kFused) {
    if (t.Q.fmt == OZFP4_E4M3)
      quantize_tokens<kPow, OZFP4_E4M3, kSrc>(t, m, total, lds, held);
    else
      quantize_tokens<kPow, OZFP4_E5M2, kSrc>(t, m, total, lds, held);
    __syncthreads();
  }

  v4f acc[TP][TQ];
#pragma unroll
  for (int i = 0; i < TP; ++i)
#pragma unroll
    for (int j = 0; j < TQ; ++j) acc[i][j] = v4f{0, 0, 0, 0};
  constexpr uint32_t one = 127;   // E8M0 1

  for (int s0 = wave; s0 < total; s0 += kTokWaves * kDeep) {
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      const int s = s0 + d * kTokWaves;
      if (s >= total) break;
      Stage& f = st[d];
      if constexpr (kFused) {
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
          const uint8_t* b = lds + (s * m + lq[j]) * 128;
          const v4i x = *reinterpret_cast<const v4i*>(b + ((g ^ (lq[j] & 7)) * 16));
          const v4i y = *reinterpret_cast<const v4i*>(b + (((g + 4) ^ (lq[j] & 7)) * 16));
          f.q[j].set(0, x);
          f.q[j].set(1, y);
          f.sq[j] = held[s * m + lq[j]];
        }
      }
      float sq[TQ][4];   // scales of this lane's rows, tokens 4 g .. + 3
      if constexpr (!kPow) {
#pragma unroll
        for (int j = 0; j < TQ; ++j)
#pragma unroll
          for (int v = 0; v < 4; ++v) sq[j][v] = __shfl(__uint_as_float(f.sq[j]), g * 4 + v);
      }
      auto as_p = [&](int i) { return to_bf16(f.p[i].get(), kPow ? f.sp[i] : one, t.P.fmt); };
      auto as_q = [&](int j) { return to_bf16(f.q[j].get(), kPow ? f.sq[j] : one, t.Q.fmt); };
      auto add = [&](int i, int j, const Frag<true>& p, const Frag<true>& q) {
        if constexpr (kPow) {
          acc[i][j] = block_product(q, p, acc[i][j]);
        } else {
          const v4f c = block_product(q, p, v4f{0, 0, 0, 0});
#pragma unroll
          for (int v = 0; v < 4; ++v)
            acc[i][j][v] = __builtin_fmaf(c[v], sq[j][v] * __uint_as_float(f.sp[i]), acc[i][j][v]);
        }
      };
      // the fewer operands stay converted, the others pass one by one
      if constexpr (TP <= TQ) {
        Frag<true> p[TP];
#pragma unroll
        for (int i = 0; i < TP; ++i) p[i] = as_p(i);
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
          const Frag<true> q = as_q(j);
#pragma unroll
          for (int i = 0; i < TP; ++i) add(i, j, p[i], q);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
        Frag<true> q[TQ];
#pragma unroll
        for (int j = 0; j < TQ; ++j) q[j] = as_q(j);
#pragma unroll
        for (int i = 0; i < TP; ++i) {
          const Frag<true> p = as_p(i);
#pragma unroll
          for (int j = 0; j < TQ; ++j) add(i, j, p, q[j]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (s + kTokWaves * kDeep < total) fetch(s + kTokWaves * kDeep, f);
    }
  }

  // the waves' sums, wave by wave: element (token, line) at token 16 TP + line
  if constexpr (kFused) __syncthreads();
  float* sum = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int j = 0; j < TQ; ++j)
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
      for (int i = 0; i < TP; ++i)
        sum[wave * kOut + (j * 16 + g * 4 + v) * (16 * TP) + i * 16 + r] = acc[i][j][v];
  __syncthreads();
  for (int e = tid; e < kOut; e += kTokWaves * 64) {
    const int64_t q = e / (16 * TP), p = p0 + e % (16 * TP);
    if (q >= m || p >= t.P.lines) continue;
    float v = sum[e];
#pragma unroll
    for (int w = 1; w < kTokWaves; ++w) v += sum[w * kOut + e];
    const int64_t at = p * t.cp + q * t.cq;
    if (t.type == OZFP4_F32) {
      float* c = static_cast<float*>(t.C) + at;
      *c = t.accumulate ? *c + v : v;
    } else if (t.type == OZFP4_BF16) {
      static_cast<__bf16*>(t.C)[at] = (__bf16)v;
    } else {
      static_cast<_Float16*>(t.C)[at] = (_Float16)v;
    }
  }
}

template <bool kPow, bool kAny, int TP, int TQ, int kSrc>
hipError_t launch(hipStream_t st, const F8Token& t) {
  hipLaunchKernelGGL((k_f8_token<kPow, kAny, TP, TQ, kSrc>), dim3((unsigned)((t.P.lines + 16 * TP - 1) / (16 * TP))),
                     dim3(kTokWaves * 64), 0, st, t);
  return hipGetLastError();
}

// Lines of P a block takes: for more than 16 tokens as many as leave about a
// block a CU, since every block reads all of the tokens; for fewer more blocks
// are better (one token, 8192 lines of 8192: 14.3 us with 16 lines, 19 with 32).
template <bool kPow, int TQ, int kSrc>
hipError_t launch_lines(hipStream_t st, const F8Token& t) {
  auto aligned = [](const F8Lines& l) {
    return (reinterpret_cast<uintptr_t>(l.x) | (l.lines > 1 ? l.ld : 0)) % 4 == 0;
  };
  const bool any = !aligned(t.P) || (kSrc < 0 && !aligned(t.Q));
  if constexpr (TQ == 2) {
    if (t.P.lines >= 2 * 16 * 256)
      return any ? launch<kPow, true, 2, TQ, kSrc>(st, t) : launch<kPow, false, 2, TQ, kSrc>(st, t);
  }
  return any ? launch<kPow, true, 1, TQ, kSrc>(st, t) : launch<kPow, false, 1, TQ, kSrc>(st, t);
}

template <bool kPow>
hipError_t launch_tokens(hipStream_t st, const F8Token& t) {
  if (t.x) {
    switch (t.src) {
      case OZFP4_F32: return launch_lines<kPow, 1, OZFP4_F32>(st, t);
      case OZFP4_BF16: return launch_lines<kPow, 1, OZFP4_BF16>(st, t);
      default: return launch_lines<kPow, 1, OZFP4_F16>(st, t);
    }
  }
  if (t.Q.lines <= 16) return launch_lines<kPow, 1, -1>(st, t);
  return launch_lines<kPow, 2, -1>(st, t);
}

}  // namespace

hipError_t launch_f8_token(hipStream_t st, const F8Token& t) {
  return t.pow2 ? launch_tokens<true>(st, t) : launch_tokens<false>(st, t);
}

}  // namespace ozfp4
