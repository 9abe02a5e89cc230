// Cross attention (gspn_attend_impl.hpp): f32 storage.
#include "gspn_attend_impl.hpp"

namespace gspn {
hipError_t launch_attend_f32(const AttendParams& p, const AttendPlan& plan, hipStream_t s) { return launch_attend_type<float>(p, plan, s); }
hipError_t launch_attend_bwd_f32(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s) { return launch_attend_bwd_type<float>(p, plan, s); }
}  // namespace gspn
