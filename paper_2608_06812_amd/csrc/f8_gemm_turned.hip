// The products whose P has its lines adjacent (f8_gemm.hpp, kTurned).
#include "f8_gemm.hpp"

namespace ozfp4 {

hipError_t launch_f8_gemm_turned(hipStream_t st, const F8Gemm& g) { return launch_gemm<true>(st, g); }

}  // namespace ozfp4
