// The products of operands whose k values are adjacent (f8_gemm.hpp), and the
// sum of k ranges.
#include "f8_gemm.hpp"

namespace ozfp4 {
namespace {

// Memory bound: the partial sums once in, C once out.
__global__ __launch_bounds__(256) void k_f8_sum(F8Sum s, bool vec) {
  const int64_t fours = s.ldp / 4, count = fours * s.lines_q;
  for (int64_t u = blockIdx.x * 256ll + threadIdx.x; u < count; u += gridDim.x * 256ll) {
    const int64_t q = u / fours, p = (u - q * fours) * 4;
    const float* x = s.x + q * s.ldp + p;
    v4f v = *reinterpret_cast<const v4f*>(x);
    for (int r = 1; r < s.ranges; ++r) v += *reinterpret_cast<const v4f*>(x + r * s.part);
    const int64_t n = s.lines_p - p;
    store4(s.C, s.type, s.accumulate, vec, q * s.ldc + p, v, n < 4 ? (int)n : 4);
  }
}

}  // namespace

hipError_t launch_f8_gemm_turned(hipStream_t st, const F8Gemm& g);   // f8_gemm_turned.hip

hipError_t launch_f8_gemm(hipStream_t st, const F8Gemm& g) {
  return g.turned ? launch_f8_gemm_turned(st, g) : launch_gemm<false>(st, g);
}

hipError_t launch_f8_sum(hipStream_t st, const F8Sum& s) {
  const int64_t size = s.type == OZFP4_F32 ? 4 : 2;
  const bool vec = reinterpret_cast<uintptr_t>(s.C) % (4 * size) == 0 && s.ldc % 4 == 0;
  hipLaunchKernelGGL(k_f8_sum, dim3(stride_blocks(s.ldp / 4 * s.lines_q, 256)), dim3(256), 0, st, s, vec);
  return hipGetLastError();
}

}  // namespace ozfp4
