// Cross attention (gspn_attend_impl.hpp): bf16 storage.
#include "gspn_attend_impl.hpp"

namespace gspn {
hipError_t launch_attend_bf16(const AttendParams& p, const AttendPlan& plan, hipStream_t s) { return launch_attend_type<bf16_t>(p, plan, s); }
hipError_t launch_attend_bwd_bf16(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s) { return launch_attend_bwd_type<bf16_t>(p, plan, s); }
}  // namespace gspn
