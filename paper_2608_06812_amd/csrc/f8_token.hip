// Product of block-scaled 8-bit operands where one has few lines (the tokens of
// a decoding step): memory bound, the bytes of the many lines (the weights)
// once. No LDS and no barrier between the weights and the matrix cores: a wave
// reads its operands straight into registers, with several blocks of 128 in
// flight, and the waves of a block take the blocks of 128 of the same 16 lines
// in turn, so that together they read up to 1 KiB of a line at a time and the
// chip has work from a few thousand lines on. Their sums meet in LDS at the end,
// in a fixed order.
//
// For up to 16 tokens of few values the product can take the tokens as they
// are (bfloat16, float16, float32): every block quantises all of them for
// itself, into LDS, while its first weights are on their way.
#include "f8_device.hpp"
#include "f8_round.hpp"

namespace ozfp4 {
namespace {

constexpr int kTokWaves = 8;

// n < 16 bytes, the rest zero
__device__ __forceinline__ v4i load_some(const uint8_t* p, int n) {
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 15; ++e)
    if (e < n) w[e >> 2] |= (uint32_t)p[e] << (8 * (e & 3));
  return v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
}

// The 16 bytes of piece c of a line's block, of which `left` bytes exist.
// Any alignment.
template <bool kWhole>
__device__ __forceinline__ v4i load_piece(const uint8_t* block, int c, int left) {
  const uint8_t* p = block + c * 16;
  if constexpr (!kWhole) {
    if (c * 16 + 16 > left) return load_some(p, left - c * 16);
  }
  v4i v;
  __builtin_memcpy(&v, p, 16);
  return v;
}

template <bool kWhole>
__device__ __forceinline__ v8i load_block(const uint8_t* block, int g, int left) {
  const v4i x = load_piece<kWhole>(block, g, left), y = load_piece<kWhole>(block, g + 4, left);
  return v8i{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
}

template <bool kPow2>
__device__ __forceinline__ uint32_t load_scale(const F8Lines& l, int64_t line, int64_t block) {
  const int64_t at = (line >> l.shift) * l.sl + block * l.sk;
  if constexpr (kPow2) return static_cast<const uint8_t*>(l.s)[at];
  return static_cast<const uint32_t*>(l.s)[at];
}

// Element (row, col) of the tokens as they come.
template <int kSrc>
__device__ __forceinline__ float source_at(const F8Token& t, int64_t row, int64_t col) {
  return widen(static_cast<const typename Source<kSrc>::T*>(t.x)[row * t.ldx + col]);
}

template <bool kExact, int kMode, int FP, int FQ, int TQ, int kSrc>
__global__ __launch_bounds__(kTokWaves * 64, 4) void k_f8_token(F8Token t) {
  constexpr bool kFused = kSrc >= 0, kPow = kMode == kPow2;
  constexpr int kDeep = TQ <= 2 ? 4 : 2;              // blocks of 128 in flight in a wave
  constexpr int kSum = kTokWaves * 256 * TQ * 4;
  constexpr int kHold = kFused ? kF8TokenBlocks * (128 + 4) : 0;
  __shared__ __align__(16) uint8_t lds[kSum > kHold ? kSum : kHold];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int64_t p0 = (int64_t)blockIdx.x * 16;
  const int total = (int)((t.k + kF8Block - 1) / kF8Block);
  const int tail = (int)(t.k - (int64_t)(total - 1) * kF8Block);
  const int m = (int)t.Q.lines;

  const uint8_t* px = t.P.x + min(p0 + r, t.P.lines - 1) * t.P.ld;
  const uint8_t* qx[TQ];
#pragma unroll
  for (int j = 0; j < TQ; ++j) qx[j] = t.Q.x + (int64_t)min(j * 16 + r, m - 1) * t.Q.ld;

  struct Stage {
    v8i p;
    uint32_t sp[kMode == kLineP ? 4 : 1];
  };
  auto fetch = [&](int s) {
    Stage f;
    const uint8_t* at = px + (int64_t)s * kF8Block;
    if (s == total - 1 && tail < kF8Block)
      f.p = load_block<false>(at, g, tail);
    else
      f.p = load_block<true>(at, g, kF8Block);
    if constexpr (kMode == kLineP) {
#pragma unroll
      for (int v = 0; v < 4; ++v) f.sp[v] = load_scale<false>(t.P, min(p0 + g * 4 + v, t.P.lines - 1), s);
    } else {
      f.sp[0] = load_scale<kPow>(t.P, min(p0 + (kPow ? r : 0), t.P.lines - 1), s);
    }
    return f;
  };

  Stage st[kDeep];
#pragma unroll
  for (int d = 0; d < kDeep; ++d)
    if (wave + d * kTokWaves < total) st[d] = fetch(wave + d * kTokWaves);

  float* held_scale = reinterpret_cast<float*>(lds + kF8TokenBlocks * 128);
  if constexpr (kFused) {
    // sixteen lanes a block of 128, eight values a lane; block b of token i at
    // (b m + i), its piece c at c ^ (i % 8)
    const int count = m * total;
    for (int u = tid >> 4; u < count; u += kTokWaves * 4) {
      const int b = u / m, i = u - b * m, c0 = r * 8;
      const int64_t col = (int64_t)b * kF8Block + c0;
      float x[8], a = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = col + e < t.k ? source_at<kSrc>(t, i, col + e) : 0.0f;
        a = __builtin_fmaxf(a, finite_abs(x[e]));
      }
#pragma unroll
      for (int d = 1; d < 16; d *= 2) a = __builtin_fmaxf(a, __shfl_xor(a, d));
      const Scale s = make_scale<kPow, FQ>(a);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = quotient<kPow>(x[e], s);
      *reinterpret_cast<uint2*>(lds + u * 128 + (((r >> 1) ^ (i & 7)) * 16) + (r & 1) * 8) =
          uint2{pack4<FQ>(x[0], x[1], x[2], x[3]), pack4<FQ>(x[4], x[5], x[6], x[7])};
      if (r == 0) {
        if constexpr (kPow)
          reinterpret_cast<uint32_t*>(held_scale)[u] = (uint32_t)(scale_exp<FQ>(a) + 127);
        else
          held_scale[u] = scale_f32<FQ>(a);
      }
    }
    __syncthreads();
  }

  v4f acc[TQ];
#pragma unroll
  for (int j = 0; j < TQ; ++j) acc[j] = v4f{0, 0, 0, 0};
  constexpr uint32_t one = 127;

  for (int s0 = wave; s0 < total; s0 += kTokWaves * kDeep) {
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      const int s = s0 + d * kTokWaves;
      if (s >= total) break;
      const Stage f = st[d];
      v8i q[TQ];
      uint32_t sq[TQ];
#pragma unroll
      for (int j = 0; j < TQ; ++j) {
        const int i = min(j * 16 + r, m - 1);
        if constexpr (kFused) {
          const uint8_t* b = lds + (s * m + i) * 128;
          const v4i x = *reinterpret_cast<const v4i*>(b + ((g ^ (i & 7)) * 16));
          const v4i y = *reinterpret_cast<const v4i*>(b + (((g + 4) ^ (i & 7)) * 16));
          q[j] = v8i{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
          sq[j] = reinterpret_cast<const uint32_t*>(held_scale)[s * m + i];
        } else {
          const uint8_t* at = qx[j] + (int64_t)s * kF8Block;
          if (s == total - 1 && tail < kF8Block)
            q[j] = load_block<false>(at, g, tail);
          else
            q[j] = load_block<true>(at, g, kF8Block);
          sq[j] = load_scale<kPow>(t.Q, i, s);
        }
      }
      if (s + kTokWaves * kDeep < total) st[d] = fetch(s + kTokWaves * kDeep);
      const auto p = Frag<kExact>::template make<FP>(f.p, kPow ? f.sp[0] : one);
#pragma unroll
      for (int j = 0; j < TQ; ++j) {
        const auto qf = Frag<kExact>::template make<FQ>(q[j], kPow ? sq[j] : one);
        if constexpr (kPow) {
          acc[j] = block_product<true, FP, FQ>(p, qf, acc[j], f.sp[0], sq[j]);
        } else {
          const v4f c = block_product<false, FP, FQ>(p, qf, v4f{0, 0, 0, 0}, 0, 0);
          const float b = __uint_as_float(sq[j]);
#pragma unroll
          for (int v = 0; v < 4; ++v)
            acc[j][v] = __builtin_fmaf(c[v], __uint_as_float(f.sp[kMode == kLineP ? v : 0]) * b, acc[j][v]);
        }
      }
    }
  }

  // the waves' sums, wave by wave: element (token, line) at token 16 + line
  if constexpr (kFused) __syncthreads();
  float* sum = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int j = 0; j < TQ; ++j)
    *reinterpret_cast<v4f*>(sum + wave * 256 * TQ + (j * 16 + r) * 16 + g * 4) = acc[j];
  __syncthreads();
  for (int e = tid; e < 256 * TQ; e += kTokWaves * 64) {
    const int64_t q = e >> 4, p = p0 + (e & 15);
    if (q >= m || p >= t.P.lines) continue;
    float v = sum[e];
#pragma unroll
    for (int w = 1; w < kTokWaves; ++w) v += sum[w * 256 * TQ + e];
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

template <bool kExact, int kMode, int FP, int FQ, int TQ, int kSrc>
hipError_t launch(hipStream_t st, const F8Token& t) {
  hipLaunchKernelGGL((k_f8_token<kExact, kMode, FP, FQ, TQ, kSrc>), dim3((unsigned)((t.P.lines + 15) / 16)),
                     dim3(kTokWaves * 64), 0, st, t);
  return hipGetLastError();
}

template <bool kExact, int kMode, int FP, int FQ>
hipError_t launch_lines(hipStream_t st, const F8Token& t) {
  if (t.x) {
    switch (t.src) {
      case OZFP4_F32: return launch<kExact, kMode, FP, FQ, 1, OZFP4_F32>(st, t);
      case OZFP4_BF16: return launch<kExact, kMode, FP, FQ, 1, OZFP4_BF16>(st, t);
      default: return launch<kExact, kMode, FP, FQ, 1, OZFP4_F16>(st, t);
    }
  }
  if (t.Q.lines <= 16) return launch<kExact, kMode, FP, FQ, 1, -1>(st, t);
  if (t.Q.lines <= 32) return launch<kExact, kMode, FP, FQ, 2, -1>(st, t);
  return launch<kExact, kMode, FP, FQ, 4, -1>(st, t);
}

template <bool kExact, int FP, int FQ>
hipError_t launch_mode(hipStream_t st, const F8Token& t) {
  if (t.pow2) return launch_lines<kExact, kPow2, FP, FQ>(st, t);
  if (t.P.shift) return launch_lines<kExact, kTileP, FP, FQ>(st, t);
  return launch_lines<kExact, kLineP, FP, FQ>(st, t);
}

template <int FP, int FQ>
hipError_t launch_formats(hipStream_t st, const F8Token& t) {
  return t.type == OZFP4_F32 ? launch_mode<true, FP, FQ>(st, t) : launch_mode<false, FP, FQ>(st, t);
}

}  // namespace

hipError_t launch_f8_token(hipStream_t st, const F8Token& t) {
  switch (t.P.fmt * 2 + t.Q.fmt) {
    case 0: return launch_formats<0, 0>(st, t);
    case 1: return launch_formats<0, 1>(st, t);
    case 2: return launch_formats<1, 0>(st, t);
    default: return launch_formats<1, 1>(st, t);
  }
}

}  // namespace ozfp4
