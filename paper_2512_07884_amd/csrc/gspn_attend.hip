// Host side of the cross attention (gspn_attend_impl.hpp): how a call is cut, its workspace, its launches.
#include "gspn_attend_impl.hpp"

namespace gspn {

namespace {
size_t rounded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

int steps_of(const AttendParams& p) { return (p.D + 15) / 16; }
// The launch over the positions, 32 per wave.  A head's tokens stay in LDS where all of them fit; four waves share up to a third of a CU's LDS, eight (where
// there is a kernel of eight) what is more; as many workgroups per head as fill the chip (by LDS, and by `simd` waves per SIMD), each with equal shares of the head's tiles.
void plan_positions(AttendPlan& a, const AttendParams& p, int row_bytes, int simd, bool eight, int dtype) {
    const size_t groups = (size_t)p.B * p.kv, tiles = (size_t)((p.N + 31) / 32) * p.per;
    const int map = steps_of(p) * 16 * (dtype == 0 ? 144 : 64);
    size_t bytes = resident_bytes(p.L, row_bytes, 4, map);
    a.waves = 4;
    if (bytes > (size_t)RESIDENT_MOST / 3 && eight && resident_bytes(p.L, row_bytes, 8, map) <= (size_t)RESIDENT_MOST) {
        a.waves = 8;
        bytes = resident_bytes(p.L, row_bytes, 8, map);
    }
    a.resident = bytes <= (size_t)RESIDENT_MOST;
    if (!a.resident) { a.workers = (int)((tiles + 3) / 4); return; }
    a.lds = (int)bytes;
    size_t fit = RESIDENT_MOST / bytes;
    if (fit > (size_t)simd * 4 / a.waves) fit = (size_t)simd * 4 / a.waves;
    if (fit < 1) fit = 1;
    const size_t share = (256 * fit + groups - 1) / groups, turns = (tiles + share * a.waves - 1) / (share * a.waves);
    a.workers = (int)((tiles + turns * a.waves - 1) / (turns * a.waves));
}

}  // namespace

// Where the positions are less than three waves for every CU, the waves of a workgroup share 32 positions and take the tokens apart -- from more than 128 tokens
// on, or on maps of less than a tile (6 heads of 64 channels, 14x14, 77 tokens: 7.1 us so, 5.5 a wave per tile; 20 positions of 12 fp32 heads,
// 60 tokens: 7.6, 10.9).  Few of those workgroups and many tokens: stretches of the tokens, joined by a launch of their own.
AttendPlan attend_plan(const AttendParams& p, int dtype) {
    AttendPlan a = {};
    const int ks = steps_of(p), es = dtype == 0 ? 4 : 2;
    const size_t groups = (size_t)p.B * p.kv, columns = (size_t)p.per * p.N;
    a.splits = 1;
    if ((size_t)p.B * p.heads * ((p.N + 31) / 32) >= 768 || (p.L <= 128 && p.N >= 32)) {
        const int dt = (ks + 1) / 2, across = es == 4 ? dt * 128 + 32 : (dt % 2 ? dt * 64 : dt * 64 + 64);
        const bool both = es == 2 && p.L <= SPLIT_MOST;
        plan_positions(a, p, ks * 16 * es + 16 + across, both ? (ks <= 4 ? 3 : 2) : attend_waves(dtype == 0, ks), !both, dtype);
        return a;
    }
    a.few = 1;
    const size_t items = groups * ((columns + 31) / 32), stages = ((size_t)p.L + 127) / 128;
    if (items < 256 && stages > 1) {
        size_t n = (512 + items - 1) / items;
        if (n > (stages + 1) / 2) n = (stages + 1) / 2;
        a.splits = (int)n;
    }
    if (a.splits > 1) a.bytes = rounded((size_t)a.splits * groups * (p.D + 2) * columns * sizeof(float));
    return a;
}

AttendBackPlan attend_back_plan(const AttendParams& p, int dtype) {
    AttendBackPlan a = {};
    const int ks = steps_of(p);
    plan_positions(a.q, p, 2 * (ks * 16 * (dtype == 0 ? 4 : 2) + 16), attend_grad_waves(dtype == 0, ks), attend_grad_waves(dtype == 0, ks) > 1, dtype);
    // waves along the tokens: as few idle ones as may be, a stage's way into LDS counted like one more
    size_t least = ~(size_t)0;
    for (int w = dtype == 0 && ks >= 7 ? 4 : 1; w <= 4; w *= 2) {
        const size_t cost = (size_t)((p.L + 32 * w - 1) / (32 * w)) * (w + 1);
        if (cost <= least) { least = cost; a.token_waves = w; }
    }
    const int px = a.token_waves == 1 ? 128 : 64;
    const size_t items = (size_t)p.B * p.kv * ((p.L + 32 * a.token_waves - 1) / (32 * a.token_waves));
    const size_t stages = (size_t)((p.N + px - 1) / px) * p.per, room = 256 * (size_t)attend_token_groups(dtype == 0, ks, a.token_waves);
    // Stretches of the positions: the chip's rounds of workgroups times the stages of one and two more for its start and end, at the least.  Stretches of fewer than
    // four stages only while there are CUs without a workgroup (the sums of their results cost more than they gain).  The backward call with 512 workgroups
    // or a few more, and by this rule: 16 heads of 72, two 64x64 maps, 300 tokens, f16 128 and 111 us, fp32 653 and 572; 8 heads of 128, 450 tokens, f16
    // 145 and 134, fp32 703 and 671; 8 heads of 40, eight 32x32, 77 tokens, f16 29 and 26; 16 heads of 64, 77 tokens, f16 49 and 50, fp32 162 and 151.
    const size_t idle = 256 / items < stages / 2 ? 256 / items : stages / 2;
    size_t fewest = ~(size_t)0;
    for (size_t rounds = 1; rounds <= 4; ++rounds) {
        size_t n = rounds * room / items;
        if (n > stages / 4) n = stages / 4;
        if (n < idle) n = idle;
        if (n < 1) n = 1;
        const size_t cost = (items * n + room - 1) / room * ((stages + n - 1) / n + 2);
        if (cost < fewest) { fewest = cost; a.splits = (int)n; }
    }
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
    if (e != hipSuccess || plan.parts == 1 || (!p.gk && !p.gv)) return e;
    const size_t n = (size_t)p.B * p.L * p.kv * p.D;
    const float* const gv = p.parts + (size_t)plan.parts * n;
    if (!p.gk) return launch_sum_parts(gv, p.gv, plan.parts, n, dtype, s);
    return launch_sum_parts(p.parts, p.gk, plan.parts, n, dtype, s, p.gv ? gv : nullptr, p.gv);
}

}  // namespace gspn
