// Relayout of 8-bit operands: lines of adjacent values, 16-byte aligned, as
// the products read them (f8_gemm.hip), from any storage order and alignment.
// Memory bound: the operand's bytes once in and once out.
#include "f8_device.hpp"

namespace ozfp4 {
namespace {

constexpr int kPackTile = 128;
constexpr int kPackLd = kPackTile + 4;

struct F8PackPair {
  F8Pack p[2];
  unsigned first;     // blocks of p[0]
  unsigned tiles[2];  // 128-line tiles of each
};

// One 128 x 128 tile of bytes: 16-byte pieces of a line straight from where they
// lie if k is adjacent, else through LDS, read along the lines and written along
// k.
__global__ __launch_bounds__(256) void k_f8_pack(F8PackPair two) {
  __shared__ __align__(16) uint8_t tile[kPackTile * kPackLd];
  const int which = blockIdx.x >= two.first;
  const F8Pack p = which ? two.p[1] : two.p[0];
  const unsigned b = blockIdx.x - (which ? two.first : 0), nl = two.tiles[which];
  const int64_t l0 = (int64_t)(b % nl) * kPackTile, k0 = (int64_t)(b / nl) * kPackTile;
  const int t = threadIdx.x, sub = t & 31, row = t >> 5;   // 4 bytes of a row of the tile, 8 rows a pass
  if (p.ks == 1) {
    // all loads before the first use, those of a line's end too: the 16 bytes
    // that end with it
    Dwords d[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int64_t line = l0 + n * 32 + (t >> 3), kk = k0 + (t & 7) * 16;
      if (line < p.lines && kk < p.k && p.k >= 16) d[n] = load_dwords(p.x + line * p.ls + min(kk, p.k - 16));
    }
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int64_t line = l0 + n * 32 + (t >> 3), kk = k0 + (t & 7) * 16;
      if (line >= p.lines || kk >= p.k) continue;
      v4i v;
      if (p.k >= 16) {
        v = d[n].bytes();
        if (kk + 16 > p.k) v = last_bytes(v, (int)(p.k - kk));
      } else {
        const uint8_t* from = p.x + line * p.ls;
        v = load_end(from, from + kk, (int)(p.k - kk));
      }
      *reinterpret_cast<v4i*>(p.out + line * p.ld + kk) = v;
    }
    return;
  }
#pragma unroll
  for (int n = 0; n < 16; ++n) {
    const int r = n * 8 + row;
    const int64_t a = k0 + r, u = l0 + sub * 4;
    uint32_t w = 0;
    if (a < p.k) {
      const uint8_t* src = p.x + a * p.ks + u;
      if (u + 4 <= p.lines)
        __builtin_memcpy(&w, src, 4);
      else
        for (int e = 0; e < 4; ++e)
          if (u + e < p.lines) w |= (uint32_t)src[e] << (8 * e);
    }
    *reinterpret_cast<uint32_t*>(tile + r * kPackLd + sub * 4) = w;
  }
  __syncthreads();
  // four k values of a line a thread
#pragma unroll
  for (int n = 0; n < 16; ++n) {
    const int l = n * 8 + row;
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= (uint32_t)tile[(sub * 4 + e) * kPackLd + l] << (8 * e);
    // the rest of a line's last 16 bytes is written with zeros
    const int64_t line = l0 + l, kk = k0 + sub * 4;
    if (line < p.lines && kk < p.ld && kk < ((p.k + 15) & ~int64_t(15)))
      *reinterpret_cast<uint32_t*>(p.out + line * p.ld + kk) = w;
  }
}

}  // namespace

hipError_t launch_f8_pack(hipStream_t st, const F8Pack* p, int count) {
  F8PackPair two = {};
  int64_t blocks = 0;
  for (int i = 0; i < count; ++i) {
    two.p[i] = p[i];
    two.tiles[i] = (unsigned)((p[i].lines + kPackTile - 1) / kPackTile);
    const int64_t n = two.tiles[i] * ((p[i].k + kPackTile - 1) / kPackTile);
    if (i == 0) two.first = (unsigned)n;
    blocks += n;
  }
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(k_f8_pack, dim3((unsigned)blocks), dim3(256), 0, st, two);
  return hipGetLastError();
}

}  // namespace ozfp4
