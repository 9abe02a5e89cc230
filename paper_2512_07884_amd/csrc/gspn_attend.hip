// Host side of the cross attention (gspn_attend_impl.hpp): how a call is cut, its workspace, its launches.
#include "gspn_attend_impl.hpp"

namespace gspn {

namespace {
size_t rounded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
}

// 64 positions per wave where that leaves two workgroups for every CU, else 32; where that leaves less than one, the waves of a workgroup share
// 32 positions and take the tokens apart.  Few of those workgroups and many tokens: stretches of the tokens, joined by a launch of their own.
AttendPlan attend_plan(const AttendParams& p, int dtype) {
    AttendPlan a = {};
    const size_t groups = (size_t)p.B * p.kv, columns = (size_t)p.per * p.N;
    a.splits = 1;
    if (groups * ((columns + 255) / 256) >= 512) a.wide = 1;
    else if (groups * ((columns + 127) / 128) < 256) {
        a.by_token = 1;
        const size_t items = groups * ((columns + 31) / 32), stages = ((size_t)p.L + 127) / 128;
        if (items < 256 && stages > 1) {
            size_t n = (512 + items - 1) / items;
            if (n > (stages + 1) / 2) n = (stages + 1) / 2;
            a.splits = (int)n;
        }
    }
    if (a.splits > 1) a.bytes = rounded((size_t)a.splits * groups * (p.D + 2) * columns * sizeof(float));
    return a;
}

AttendBackPlan attend_back_plan(const AttendParams& p, int dtype) {
    AttendBackPlan a = {};
    a.token_waves = p.L > 64 || (dtype == 0 && p.D > 96) ? 4 : (p.L > 32 ? 2 : 1);
    const int px = a.token_waves == 1 ? 128 : 64;
    const size_t items = (size_t)p.B * p.kv * ((p.L + 32 * a.token_waves - 1) / (32 * a.token_waves));
    const size_t stages = (size_t)((p.N + px - 1) / px) * p.per;
    size_t n = (512 + items - 1) / items;
    if (n > stages / 2) n = stages / 2;
    a.splits = n < 1 ? 1 : (int)n;
    a.parts = a.splits * (4 / a.token_waves);
    a.delta_bytes = rounded((size_t)p.B * p.heads * p.N * sizeof(float));
    a.bytes = a.delta_bytes + (a.parts > 1 ? rounded(2 * (size_t)a.parts * p.B * p.L * p.kv * p.D * sizeof(float)) : 0);
    return a;
}

hipError_t launch_attend(const AttendParams& p, const AttendPlan& plan, int dtype, hipStream_t s) {
    return dtype == 0 ? launch_attend_f32(p, plan, s) : dtype == 1 ? launch_attend_bf16(p, plan, s) : launch_attend_f16(p, plan, s);
}

hipError_t launch_attend_bwd(const AttendParams& p, const AttendBackPlan& plan, int dtype, hipStream_t s) {
    hipError_t e = dtype == 0 ? launch_attend_bwd_f32(p, plan, s) : dtype == 1 ? launch_attend_bwd_bf16(p, plan, s) : launch_attend_bwd_f16(p, plan, s);
    if (e != hipSuccess || plan.parts == 1) return e;
    const size_t n = (size_t)p.B * p.L * p.kv * p.D;
    if (p.gk && (e = launch_sum_parts(p.parts, p.gk, plan.parts, n, dtype, s)) != hipSuccess) return e;
    return p.gv ? launch_sum_parts(p.parts + (size_t)plan.parts * n, p.gv, plan.parts, n, dtype, s) : e;
}

}  // namespace gspn
