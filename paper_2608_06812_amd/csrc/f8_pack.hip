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
  const int t = threadIdx.x, sub = t & 31, row = t >> 5;
  // rows along the unit stride: of k values, or of lines
  const bool along_k = p.ks == 1;
  const int64_t a0 = along_k ? l0 : k0, as = along_k ? p.ls : p.ks, an = along_k ? p.lines : p.k;
  const int64_t u0 = (along_k ? k0 : l0) + (t & 7) * 16, un = along_k ? p.k : p.lines;
  // all loads before the first use, those of a row's end too: the 16 bytes that
  // end with it
  Dwords d[4];
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const int64_t a = a0 + n * 32 + (t >> 3);
    if (a < an && u0 < un && un >= 16) d[n] = load_dwords(p.x + a * as + min(u0, un - 16));
  }
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const int r = n * 32 + (t >> 3);
    const int64_t a = a0 + r;
    v4i v = {0, 0, 0, 0};
    if (a < an && u0 < un) {
      if (un >= 16) {
        v = d[n].bytes();
        if (u0 + 16 > un) v = last_bytes(v, (int)(un - u0));
      } else {
        const uint8_t* from = p.x + a * as;
        v = load_end(from, from + u0, (int)(un - u0));
      }
      if (along_k) *reinterpret_cast<v4i*>(p.out + a * p.ld + u0) = v;
    }
    if (!along_k)
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<int*>(tile + r * kPackLd + (t & 7) * 16 + e * 4) = v[e];
  }
  if (along_k) return;
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
