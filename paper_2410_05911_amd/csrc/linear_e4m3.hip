// The products of gemm.h for factors of one type.
#include "gemm.h"

namespace aecct {
hipError_t launch_gemm_e4m3(const Gemm *g, const GemmPlan *plan, int count, hipStream_t s) { return launch_type<f16_t, e4m3_t>(g, plan, count, s); }
}  // namespace aecct
