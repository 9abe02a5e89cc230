// Cross attention (gspn_attend_impl.hpp): f16 storage.
#include "gspn_attend_impl.hpp"

namespace gspn {
hipError_t launch_attend_f16(const AttendParams& p, const AttendPlan& plan, hipStream_t s) { return launch_attend_type<f16_t>(p, plan, s); }
hipError_t launch_attend_bwd_f16(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s) { return launch_attend_bwd_type<f16_t>(p, plan, s); }
}  // namespace gspn
