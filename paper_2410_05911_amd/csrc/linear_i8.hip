// The products of gemm.h for factors of one type.
#include "gemm.h"

namespace aecct {
hipError_t launch_gemm_i8(const Gemm *g, const GemmPlan *plan, int count, hipStream_t s) { return launch_type<int8_t>(g, plan, count, s); }
}  // namespace aecct
