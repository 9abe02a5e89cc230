// C entry points of the operators around the scan: argument checks, the layout of the workspaces, the launches of a call.
#include "../../include/gspn.h"
#include "gspn_block.hpp"

using namespace gspn;

namespace {

bool off16(const void* p) { return ((uintptr_t)p & 15u) != 0; }
bool known_type(int dtype) { return dtype == GSPN_F32 || dtype == GSPN_BF16 || dtype == GSPN_F16; }
bool known_act(int act) { return act == GSPN_ACT_NONE || act == GSPN_ACT_SILU || act == GSPN_ACT_GELU || act == GSPN_ACT_SIGMOID; }
size_t storage(int dtype) { return dtype == GSPN_F32 ? 4 : 2; }
size_t rounded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
constexpr long long TOP = 1ll << 31;

// A launch counts the workgroups of a result of `rows` rows and N pixels: 32 pixels of short rows each at least, 128 of others (narrower ones are taken where they are few)
bool counted(long long B, long long rows, long long N) {
    const long long columns = N < 128 ? N / 32 + 1 : N / 128 + 1;
    return columns * B < TOP / 128 && columns * B * (rows / 32 + 1) < TOP / 128;
}

// rows: rows of P (M, or 2 F of the gated pair)
int check_product(int B, int K, int M, int rows_per, int H, int W, int act, int dtype) {
    if (B < 1 || K < 1 || M < 1 || H < 1 || W < 1) return GSPN_ERR_SHAPE;
    if (!known_type(dtype)) return GSPN_ERR_DTYPE;
    if (!known_act(act)) return GSPN_ERR_UNSUPPORTED;
    if (H > GSPN_MAX_LINE || W > GSPN_MAX_LINE) return GSPN_ERR_UNSUPPORTED;
    const long long rows = (long long)M * rows_per, N = (long long)H * W;
    // maps and matrices of less than 2^31 values a side
    if (rows >= TOP || N >= TOP || K >= TOP / 2 || rows * K >= TOP || !counted(B, rows, N)) return GSPN_ERR_UNSUPPORTED;
    return GSPN_OK;
}

// The workspace of a backward call: the gradient at the product's result (with an activation), partial sums of the bias's gradient and of
// the matrix's
struct ProductBack {
    size_t grad, sums, parts, bytes;
    int sum_parts, splits;
};
ProductParams forward_params(int B, int K, int M, int N, int act) {
    ProductParams p = {};
    p.M = M; p.N = N; p.K = K; p.images = B; p.act = act; p.splits = 1;
    return p;
}
ProductParams matrix_params(int B, int K, int rows, int N) {
    ProductParams p = {};
    p.M = rows; p.N = K; p.K = N; p.images = B; p.splits = 1;
    return p;
}
// What the backward call launches besides: results of K rows, of rows x K, and the sums over rows
int check_product_back(int B, int K, int M, int rows_per, int H, int W, int act, int dtype) {
    const int st = check_product(B, K, M, rows_per, H, W, act, dtype);
    if (st != GSPN_OK) return st;
    const long long rows = (long long)M * rows_per, N = (long long)H * W;
    if (!counted(B, K, N) || (rows / 64 + 1) * (K / 64 + 1) >= TOP / 512 || (N / 4096 + 1) * B * M >= TOP / 32) return GSPN_ERR_UNSUPPORTED;
    return GSPN_OK;
}
ProductBack back_layout(int B, int K, int M, bool gated, int N, int act, int dtype) {
    ProductBack w = {};
    const int rows = gated ? 2 * M : M;
    const bool direct = !gated && act == GSPN_ACT_NONE;
    w.sum_parts = direct ? row_sum_parts(B, M, N) : product_sum_parts(forward_params(B, K, M, N, act), gated ? OUT_GATED_GRAD : OUT_PROJECT_GRAD, dtype);
    w.splits = product_splits(matrix_params(B, K, rows, N), dtype);
    w.grad = 0;
    w.sums = direct ? 0 : rounded((size_t)B * rows * N * storage(dtype));
    w.parts = w.sums + rounded((size_t)w.sum_parts * rows * sizeof(float));
    w.bytes = w.parts + (w.splits > 1 ? rounded((size_t)w.splits * rows * K * sizeof(float)) : 0);
    return w;
}

int product_backward(const void* gout, const void* in, const void* P, const void* bias, void* gin, void* gP, void* gbias, void* workspace,
                     unsigned long long workspace_bytes, int B, int K, int M, bool gated, int H, int W, int act, int dtype, void* stream) {
    if (!gout || !in || !P || (!gin && !gP && !gbias)) return GSPN_ERR_NULL;
    const int st = check_product_back(B, K, M, gated ? 2 : 1, H, W, act, dtype);
    if (st != GSPN_OK) return st;
    if (!workspace) return GSPN_ERR_NULL;
    if (off16(gout) || off16(in) || off16(P) || off16(bias) || off16(gin) || off16(gP) || off16(gbias) || off16(workspace)) return GSPN_ERR_ALIGN;
    const int N = H * W, rows = gated ? 2 * M : M;
    const ProductBack w = back_layout(B, K, M, gated, N, act, dtype);
    if (workspace_bytes < w.bytes) return GSPN_ERR_SHAPE;
    hipStream_t s = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    float* const sums = (float*)(ws + w.sums);
    const void* g = gout;
    hipError_t e;
    if (gated || act != GSPN_ACT_NONE) {
        ProductParams p = forward_params(B, K, M, N, act);
        p.a = P; p.b = in; p.bias = bias; p.extra = gout; p.out = ws + w.grad; p.sums = gbias ? sums : nullptr;
        if ((e = launch_product(p, PRODUCT_FORWARD, gated ? OUT_GATED_GRAD : OUT_PROJECT_GRAD, dtype, s)) != hipSuccess) return GSPN_ERR_HIP;
        if (gbias && (e = launch_sum_parts(sums, gbias, w.sum_parts, (size_t)rows, dtype, s)) != hipSuccess) return GSPN_ERR_HIP;
        g = ws + w.grad;
    } else if (gbias) {
        if ((e = launch_row_sums(gout, gbias, sums, B, M, N, dtype, s)) != hipSuccess) return GSPN_ERR_HIP;
    }
    if (gin) {
        ProductParams p = {};
        p.a = P; p.b = g; p.out = gin; p.M = K; p.N = N; p.K = rows; p.images = B; p.splits = 1;
        if ((e = launch_product(p, PRODUCT_GRAD_INPUT, OUT_PLAIN, dtype, s)) != hipSuccess) return GSPN_ERR_HIP;
    }
    if (gP) {
        ProductParams p = matrix_params(B, K, rows, N);
        p.a = g; p.b = in; p.out = gP; p.splits = w.splits; p.parts = w.splits > 1 ? (float*)(ws + w.parts) : nullptr;
        if ((e = launch_product(p, PRODUCT_GRAD_MATRIX, OUT_PLAIN, dtype, s)) != hipSuccess) return GSPN_ERR_HIP;
        if (w.splits > 1 && (e = launch_sum_parts(p.parts, gP, w.splits, (size_t)rows * K, dtype, s)) != hipSuccess) return GSPN_ERR_HIP;
    }
    return GSPN_OK;
}

int check_attend(int B, int heads, int kv_heads, int D, int H, int W, int L, float scale, int dtype) {
    if (B < 1 || heads < 1 || kv_heads < 1 || D < 1 || H < 1 || W < 1 || L < 1 || heads % kv_heads != 0) return GSPN_ERR_SHAPE;
    if (!(scale > 0.f) || scale > 3.4e38f) return GSPN_ERR_SHAPE;
    if (!known_type(dtype)) return GSPN_ERR_DTYPE;
    if (H > GSPN_MAX_LINE || W > GSPN_MAX_LINE || D % 8 != 0 || D > GSPN_MAX_HEAD || L > GSPN_MAX_TOKENS) return GSPN_ERR_UNSUPPORTED;
    // workgroups of a launch: 32 positions each at least
    const long long N = (long long)H * W, per = heads / kv_heads;
    if (N >= TOP / 32 || per * N >= TOP / 4 || (long long)B * kv_heads >= TOP / 1024 || (long long)B * kv_heads * (per * N / 32 + 1) >= TOP / 128 || (long long)B * heads * N >= TOP / 16 ||
        (long long)B * kv_heads * (L / 32 + 1) >= TOP / 128)
        return GSPN_ERR_UNSUPPORTED;
    return GSPN_OK;
}
AttendParams attend_params(int B, int heads, int kv_heads, int D, int H, int W, int L, float scale) {
    AttendParams p = {};
    p.B = B; p.heads = heads; p.kv = kv_heads; p.per = heads / kv_heads; p.D = D; p.N = H * W; p.L = L; p.scale = scale; p.splits = 1;
    return p;
}

}  // namespace

extern "C" {

unsigned long long gspn_cross_attention_bytes(int B, int heads, int kv_heads, int D, int H, int W, int L, int dtype) {
    if (check_attend(B, heads, kv_heads, D, H, W, L, 1.f, dtype) != GSPN_OK) return 0;
    return attend_plan(attend_params(B, heads, kv_heads, D, H, W, L, 1.f), dtype).bytes;
}

unsigned long long gspn_cross_attention_bwd_bytes(int B, int heads, int kv_heads, int D, int H, int W, int L, int dtype) {
    if (check_attend(B, heads, kv_heads, D, H, W, L, 1.f, dtype) != GSPN_OK) return 0;
    return attend_back_plan(attend_params(B, heads, kv_heads, D, H, W, L, 1.f), dtype).bytes;
}

int gspn_cross_attention(const void* q, const void* k, const void* v, const unsigned char* mask, void* out, float* lse,
                         void* workspace, unsigned long long workspace_bytes,
                         int B, int heads, int kv_heads, int D, int H, int W, int L, float scale, int dtype, void* stream) {
    if (!q || !k || !v || !out) return GSPN_ERR_NULL;
    const int st = check_attend(B, heads, kv_heads, D, H, W, L, scale, dtype);
    if (st != GSPN_OK) return st;
    if (off16(q) || off16(k) || off16(v) || off16(out) || off16(lse) || off16(workspace)) return GSPN_ERR_ALIGN;
    AttendParams p = attend_params(B, heads, kv_heads, D, H, W, L, scale);
    p.q = q; p.k = k; p.v = v; p.mask = mask; p.out = out; p.lse = lse;
    AttendPlan plan = attend_plan(p, dtype);
    if (workspace && workspace_bytes < plan.bytes) return GSPN_ERR_SHAPE;
    if (!workspace) plan.splits = 1;
    p.splits = plan.splits;
    p.workers = plan.workers;
    p.parts = (float*)workspace;
    return launch_attend(p, plan, dtype, (hipStream_t)stream) == hipSuccess ? GSPN_OK : GSPN_ERR_HIP;
}

int gspn_cross_attention_bwd(const void* gout, const void* q, const void* k, const void* v, const unsigned char* mask, const void* out, const float* lse,
                             void* gq, void* gk, void* gv, void* workspace, unsigned long long workspace_bytes,
                             int B, int heads, int kv_heads, int D, int H, int W, int L, float scale, int dtype, void* stream) {
    if (!gout || !q || !k || !v || !out || !lse || (!gq && !gk && !gv)) return GSPN_ERR_NULL;
    const int st = check_attend(B, heads, kv_heads, D, H, W, L, scale, dtype);
    if (st != GSPN_OK) return st;
    if (!workspace) return GSPN_ERR_NULL;
    if (off16(gout) || off16(q) || off16(k) || off16(v) || off16(out) || off16(lse) || off16(gq) || off16(gk) || off16(gv) || off16(workspace))
        return GSPN_ERR_ALIGN;
    AttendParams p = attend_params(B, heads, kv_heads, D, H, W, L, scale);
    p.gout = gout; p.q = q; p.k = k; p.v = v; p.mask = mask; p.out = (void*)out; p.lse = (float*)lse;
    p.gq = gq; p.gk = gk; p.gv = gv;
    const AttendBackPlan plan = attend_back_plan(p, dtype);
    if (workspace_bytes < plan.bytes) return GSPN_ERR_SHAPE;
    p.splits = plan.splits;
    p.delta = (float*)workspace;
    p.parts = (float*)((char*)workspace + plan.delta_bytes);
    return launch_attend_bwd(p, plan, dtype, (hipStream_t)stream) == hipSuccess ? GSPN_OK : GSPN_ERR_HIP;
}

int gspn_proxy_project_fused(const void* in, const void* P, const void* bias, const void* residual, void* out,
                             int B, int K, int M, int H, int W, int act, int dtype, void* stream) {
    if (!in || !P || !out) return GSPN_ERR_NULL;
    const int st = check_product(B, K, M, 1, H, W, act, dtype);
    if (st != GSPN_OK) return st;
    if (off16(in) || off16(P) || off16(bias) || off16(residual) || off16(out)) return GSPN_ERR_ALIGN;
    ProductParams p = forward_params(B, K, M, H * W, act);
    p.a = P; p.b = in; p.bias = bias; p.extra = residual; p.out = out;
    return launch_product(p, PRODUCT_FORWARD, OUT_PROJECT, dtype, (hipStream_t)stream) == hipSuccess ? GSPN_OK : GSPN_ERR_HIP;
}

int gspn_gated_project(const void* in, const void* P, const void* bias, void* out,
                       int B, int K, int F, int H, int W, int act, int dtype, void* stream) {
    if (!in || !P || !out) return GSPN_ERR_NULL;
    const int st = check_product(B, K, F, 2, H, W, act, dtype);
    if (st != GSPN_OK) return st;
    if (off16(in) || off16(P) || off16(bias) || off16(out)) return GSPN_ERR_ALIGN;
    ProductParams p = forward_params(B, K, F, H * W, act);
    p.a = P; p.b = in; p.bias = bias; p.out = out;
    return launch_product(p, PRODUCT_FORWARD, OUT_GATED, dtype, (hipStream_t)stream) == hipSuccess ? GSPN_OK : GSPN_ERR_HIP;
}

unsigned long long gspn_proxy_project_fused_bwd_bytes(int B, int K, int M, int H, int W, int act, int dtype) {
    if (check_product_back(B, K, M, 1, H, W, act, dtype) != GSPN_OK) return 0;
    return back_layout(B, K, M, false, H * W, act, dtype).bytes;
}

unsigned long long gspn_gated_project_bwd_bytes(int B, int K, int F, int H, int W, int act, int dtype) {
    if (check_product_back(B, K, F, 2, H, W, act, dtype) != GSPN_OK) return 0;
    return back_layout(B, K, F, true, H * W, act, dtype).bytes;
}

int gspn_proxy_project_fused_bwd(const void* gout, const void* in, const void* P, const void* bias, void* gin, void* gP, void* gbias,
                                 void* workspace, unsigned long long workspace_bytes,
                                 int B, int K, int M, int H, int W, int act, int dtype, void* stream) {
    return product_backward(gout, in, P, bias, gin, gP, gbias, workspace, workspace_bytes, B, K, M, false, H, W, act, dtype, stream);
}

int gspn_gated_project_bwd(const void* gout, const void* in, const void* P, const void* bias, void* gin, void* gP, void* gbias,
                           void* workspace, unsigned long long workspace_bytes,
                           int B, int K, int F, int H, int W, int act, int dtype, void* stream) {
    return product_backward(gout, in, P, bias, gin, gP, gbias, workspace, workspace_bytes, B, K, F, true, H, W, act, dtype, stream);
}

}  // extern "C"
