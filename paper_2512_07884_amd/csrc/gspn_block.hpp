// Launch parameters of the operators around the scan: products with an epilogue (gspn_product*.hip) and cross attention (gspn_attend*.hip).
#pragma once
#include "gspn_common.hpp"

namespace gspn {

// One product over the channels, or over the pixels, of [image][channel][pixel] maps:
//     R[m][n] = sum_k A[m][k] B[k][n],  per image (images > 1) or summed over images (PRODUCT_GRAD_MATRIX)
// forms, by how the operands are stored:
//   PRODUCT_FORWARD      A = P [M][K] (k contiguous), B = in [K][N] (n contiguous)
//   PRODUCT_GRAD_INPUT   A = P^T, stored [K][M] (m contiguous), B = gout [K][N]
//   PRODUCT_GRAD_MATRIX  A = gout [M][K], B = in^T, stored [N][K] (k, the pixels, contiguous in both); K pixels of each of `images`
enum { PRODUCT_FORWARD = 0, PRODUCT_GRAD_INPUT = 1, PRODUCT_GRAD_MATRIX = 2 };
enum { ACT_NONE = 0, ACT_SILU = 1, ACT_GELU = 2, ACT_SIGMOID = 3 };
// what becomes of R: stored as it is; act(R + bias) + residual; gout * act'(R + bias); the gated pair, forward and backward
enum { OUT_PLAIN = 0, OUT_PROJECT = 1, OUT_PROJECT_GRAD = 2, OUT_GATED = 3, OUT_GATED_GRAD = 4 };

struct ProductParams {
    const void* a; const void* b;
    const void* bias;          // [rows of P], storage type, or null
    const void* extra;         // residual (OUT_PROJECT, or null) or gout (OUT_*_GRAD), [images][rows of R][N]
    void* out;
    float* sums;               // OUT_*_GRAD: partial sums of the rows of the result, [images * column tiles][rows of P], or null
    float* parts;              // PRODUCT_GRAD_MATRIX: [splits][M][N], or null (one split: stored to out)
    int M, N, K, images;       // OUT_GATED*: M = hidden channels F, P has 2 F rows
    int act;
    int splits;                // PRODUCT_GRAD_MATRIX: stretches of the contracted axis
};
// number of partial sums per row that an OUT_*_GRAD launch writes
int product_sum_parts(const ProductParams& p, int outcome, int dtype);
int product_splits(const ProductParams& p, int dtype);            // PRODUCT_GRAD_MATRIX: stretches that such a call is cut into
hipError_t launch_product(const ProductParams& p, int form, int outcome, int dtype, hipStream_t s);
// out[i] = sum over `parts` of in[part][i], in order, rounded to the storage type; and a second sum of the same size in the same launch
hipError_t launch_sum_parts(const float* in, void* out, int parts, size_t n, int dtype, hipStream_t s, const float* in2 = nullptr, void* out2 = nullptr);
// out[m] = sum over images and pixels of g[image][m][n]
hipError_t launch_row_sums(const void* g, void* out, float* parts, int images, int M, int N, int dtype, hipStream_t s);
int row_sum_parts(int images, int M, int N);

// Attention of the positions of [image][head][channel][position] maps to [image][token][head][channel] states.  `per` heads of the map share
// a head of the tokens; the columns of such a group are its heads' positions, one head after the other (per * N of them).
struct AttendParams {
    const void* q; const void* k; const void* v;
    const unsigned char* mask;       // [B][L], 0: the token takes no part; or null
    void* out;                       // forward: out; backward: the forward call's out, read
    float* lse;                      // [B][heads][N], or null in the forward call
    const void* gout;
    void* gq; void* gk; void* gv;
    float* delta;                    // backward: [B][heads][N]
    float* parts;                    // forward: states of the stretches of the tokens; backward: partial sums of gk and gv
    int B, heads, kv, per, D, N, L;
    float scale;
    int splits;                      // stretches of the tokens (forward), of the positions (backward)
    int workers;                     // workgroups per head of the tokens
};
// How a call runs.  few: the waves of a workgroup on the tokens instead of the positions, in `splits` stretches; else
// resident: a head's tokens all in LDS (`lds` bytes); waves of a workgroup; workgroups per head of the tokens.
struct AttendPlan { int few, resident, waves, workers, splits, lds; size_t bytes; };
AttendPlan attend_plan(const AttendParams& p, int dtype);
// backward: the launch of gq; for gk and gv waves along the tokens (4, 2 or 1; the others along the positions) and stretches of the positions
struct AttendBackPlan { AttendPlan q; int token_waves, splits, parts; size_t delta_bytes, bytes; };
AttendBackPlan attend_back_plan(const AttendParams& p, int dtype);
hipError_t launch_attend(const AttendParams& p, const AttendPlan& plan, int dtype, hipStream_t s);
hipError_t launch_attend_bwd(const AttendParams& p, const AttendBackPlan& plan, int dtype, hipStream_t s);

}  // namespace gspn
