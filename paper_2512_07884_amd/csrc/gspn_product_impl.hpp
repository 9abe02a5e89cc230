// Products over channels or pixels of [image][channel][pixel] maps on the matrix cores, with what follows them in the same launch:
// the projections with bias, activation and residual, the gated pair, and the three products of their gradients.
//
//     R[m][n] = sum_k A[m][k] B[k][n]
//
// A workgroup owns a tile of BM x BN results and walks the contracted axis in stages of WK times 128 bytes.  Both operands of a stage
// go through LDS: requests of 16 bytes that run along the rows as they are stored, two stages of LDS, the stage after them on its way in
// registers while the waves multiply.  An operand whose contracted axis is contiguous is read from LDS 16 bytes per lane; one whose rows run
// across it (the pixels of the maps) is turned on the way out of LDS (ds_read_b64_tr_b16; fp32: single words).  Both are stored with the
// 16-byte pieces of a row exchanged by the row's number, so that neither the rows nor the columns that a request touches share banks.
// The waves stand WM x WN over the tile and WK over the stage (small results, where tiles are few: the sums of the WK waves meet in LDS).
// What follows the product is done on rows of the result that passed through LDS in fp32, eight neighbouring pixels per lane: bias,
// activation, residual or the gradient's factor, one rounding, 16-byte stores.
// Rows that end inside a tile: the last tile of a row starts where it is whole (its first columns are computed twice, the same bits are
// stored twice); rows shorter than a tile are requested piece by piece.  Rows of A past the end are read as the last one, not stored.
#pragma once
#include "gspn_matrix.hpp"
#include "gspn_block.hpp"

namespace gspn {

// the activation of z, and its derivative
template <bool GRAD> __device__ __forceinline__ float activation(float z, int act, float* slope) {
    if (act == ACT_NONE) { if (GRAD) *slope = 1.f; return z; }
    if (act == ACT_GELU) {
        const float phi = fmaf(0.5f, erff(z * 0.70710678118654752f), 0.5f);
        if (GRAD) *slope = fmaf(z * 0.39894228040143268f, __expf(-0.5f * z * z), phi);
        return z * phi;
    }
    const float g = 1.0f / (1.0f + __expf(-z));
    if (act == ACT_SIGMOID) { if (GRAD) *slope = g * (1.f - g); return g; }
    if (GRAD) *slope = fmaf(z * g, 1.f - g, g);
    return z * g;
}

// where the 16-byte piece c of row r goes in LDS: contracted axis along the row (rows of 128 bytes) ...
__device__ __forceinline__ int along_swap(int r, int c) { return c ^ ((r >> 1) & 7); }
// ... and across the rows (rows of COLS values)
template <typename T, int COLS> __device__ __forceinline__ int across_swap(int r, int c) {
    if constexpr (sizeof(T) == 4) return COLS >= 64 ? c ^ (((r >> 3) & 1) << 3) : c;
    else return COLS >= 128 ? c ^ ((r & 3) << 2) : (COLS == 64 ? c ^ (((r >> 1) & 1) << 2) : c);
}

template <typename T> __device__ __forceinline__ MatFrag<T> along_operand(const char* tile, int r, int s, int half) {
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const u32x4 a = *(const u32x4*)(tile + r * 128 + along_swap(r, 4 * s + 2 * half + j) * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) f.v[4 * j + i] = __uint_as_float(a[i]);
        }
    } else {
        f.w = *(const u32x4*)(tile + r * 128 + along_swap(r, 2 * s + half) * 16);
    }
    return f;
}
template <typename T, int COLS> __device__ __forceinline__ MatFrag<T> across_operand(const char* tile, int col0, int s, int lane) {
    const int half = lane >> 5;
    constexpr int PITCH = COLS * (int)sizeof(T);
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
        const int col = col0 + (lane & 31);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 16 * s + 8 * half + i;
            f.v[i] = *(const float*)(tile + r * PITCH + across_swap<T, COLS>(r, col >> 2) * 16 + (col & 3) * 4);
        }
    } else {
        const int j = lane & 15, col = col0 + (lane & 16) + (j & 3) * 4;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = 16 * s + 8 * half + 4 * i + (j >> 2);
            const u32x2 v = lds_turned(tile + r * PITCH + across_swap<T, COLS>(r, col >> 3) * 16 + (col & 7) * 2);
            f.w[2 * i] = v.x; f.w[2 * i + 1] = v.y;
        }
    }
    return f;
}

template <typename T, int FORM, int OUTC, int MT, int NT, int WM, int WN, int WK>
struct ProductShape {
    static constexpr int BM = 32 * MT * WM, BN = 32 * NT * WN, THREADS = 64 * WM * WN * WK;
    static constexpr int BK = 128 / (int)sizeof(T), E = 16 / (int)sizeof(T);
    static constexpr int A_BYTES = WK * BM * 128, B_BYTES = WK * BN * 128, STAGE = A_BYTES + B_BYTES;
    static constexpr bool GATED = OUTC == OUT_GATED || OUTC == OUT_GATED_GRAD;
    static constexpr int PAIR = GATED ? 2 : 1;                       // row tiles that are finished together
    static constexpr int PITCH = 32 * NT + 4;                        // floats of a row of the result in LDS
    static constexpr int FINISH = WM * WN * WK * PAIR * 32 * PITCH * 4;
    static constexpr int LDS = 2 * STAGE > FINISH ? 2 * STAGE : FINISH;
    static constexpr int ROWS = GATED ? BM / 2 : BM;                 // rows of the result
};

template <typename T, int FORM, int OUTC, int MT, int NT, int WM, int WN, int WK>
__global__ void __launch_bounds__(64 * WM * WN * WK) product_kernel(const ProductParams p) {
    using S = ProductShape<T, FORM, OUTC, MT, NT, WM, WN, WK>;
    constexpr int BM = S::BM, BN = S::BN, BK = S::BK, E = S::E, THREADS = S::THREADS;
    constexpr bool A_ACROSS = FORM == PRODUCT_GRAD_INPUT, B_ACROSS = FORM != PRODUCT_GRAD_MATRIX;
    constexpr int CA = WK * BM * 8 / THREADS, CB = WK * BN * 8 / THREADS;        // 16-byte pieces of a stage per thread
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wk = wave % WK, wn = (wave / WK) % WN, wm = wave / (WK * WN);
    const int M = p.M, N = p.N, K = p.K;

    // work item -> tile.  An XCD (an L2 of its own) takes neighbouring items; eight column tiles pass over the row tiles together, so
    // that what the items in flight read again of either operand is still there.
    const int mtiles = (M + S::ROWS - 1) / S::ROWS, ntiles = (N + BN - 1) / BN;
    unsigned item = xcd_contiguous_item(blockIdx.x, gridDim.x);
    int split = 0, image = 0, mt, nt;
    if constexpr (FORM == PRODUCT_GRAD_MATRIX) {
        const unsigned tiles = (unsigned)mtiles * ntiles;
        split = item / tiles;
        item -= split * tiles;
        mt = item / ntiles; nt = item % ntiles;
    } else {
        const unsigned cols = (unsigned)ntiles * p.images, group = item / (8u * mtiles), rest = item - group * 8u * mtiles;
        const unsigned wide = min(8u, cols - group * 8u), col = group * 8u + rest % wide;
        mt = rest / wide;
        image = col / ntiles; nt = col - image * ntiles;
    }
    const int m0 = A_ACROSS && M >= BM ? min(mt * BM, M - BM) : mt * S::ROWS;
    const int n0 = B_ACROSS && N >= BN ? min(nt * BN, N - BN) : nt * BN;

    // stages of the contracted axis: [first, last)
    constexpr int STEP = WK * BK;
    const int stages = (K + STEP - 1) / STEP;                        // of an image
    int first = 0, last = stages;
    if constexpr (FORM == PRODUCT_GRAD_MATRIX) {
        const long all = (long)stages * p.images;
        first = (int)(all * split / p.splits);
        last = (int)(all * (split + 1) / p.splits);
    }

    const T* const A = (const T*)p.a;
    const T* const B = (const T*)p.b + (FORM == PRODUCT_GRAD_MATRIX ? 0 : (size_t)image * K * N);
    const bool a_narrow = A_ACROSS && M < BM, b_narrow = B_ACROSS && N < BN;

    u32x4 ra[CA], rb[CB];
    // row of A (stored along the contracted axis) that row r of the tile stands for
    auto a_row = [&](int r) {
        if constexpr (S::GATED) return ((r >> 5) & 1) * M + min(m0 + (r >> 6) * 32 + (r & 31), M - 1);
        else return min(m0 + r, M - 1);
    };
    auto fetch = [&](int st) {
        int k0 = st * STEP;
        const T *a = A, *b = B;
        if constexpr (FORM == PRODUCT_GRAD_MATRIX) {
            const int im = st / stages;
            k0 = (st - im * stages) * STEP;
            a += (size_t)im * M * K;
            b += (size_t)im * N * K;
        }
        const bool ends = k0 + STEP > K;
#pragma unroll
        for (int i = 0; i < CA; ++i) {
            const int c = tid + i * THREADS;
            if constexpr (A_ACROSS) {
                const int kk = c / (BM / E), col = m0 + (c % (BM / E)) * E;
                if (ends || a_narrow) ra[i] = k0 + kk < K ? row_chunk(a + (size_t)(k0 + kk) * M, col, M) : u32x4{0, 0, 0, 0};
                else ra[i] = rg_load(a + (size_t)(k0 + kk) * M + col);
            } else {
                const int r = a_row(c / (8 * WK)), k = k0 + (c % (8 * WK)) * E;
                if (ends) ra[i] = row_chunk(a + (size_t)r * K, k, K);
                else ra[i] = rg_load(a + (size_t)r * K + k);
            }
        }
#pragma unroll
        for (int i = 0; i < CB; ++i) {
            const int c = tid + i * THREADS;
            if constexpr (B_ACROSS) {
                const int kk = c / (BN / E), col = n0 + (c % (BN / E)) * E;
                if (ends || b_narrow) rb[i] = k0 + kk < K ? row_chunk(b + (size_t)(k0 + kk) * N, col, N) : u32x4{0, 0, 0, 0};
                else rb[i] = rg_load(b + (size_t)(k0 + kk) * N + col);
            } else {
                const int r = min(n0 + c / (8 * WK), N - 1), k = k0 + (c % (8 * WK)) * E;
                if (ends) rb[i] = row_chunk(b + (size_t)r * K, k, K);
                else rb[i] = rg_load(b + (size_t)r * K + k);
            }
        }
    };
    auto put = [&](int buf) {
        char* const ta = lds + buf * S::STAGE;
        char* const tb = ta + S::A_BYTES;
#pragma unroll
        for (int i = 0; i < CA; ++i) {
            const int c = tid + i * THREADS;
            if constexpr (A_ACROSS) {
                const int kk = c / (BM / E), ch = c % (BM / E);
                *(u32x4*)(ta + (size_t)kk * BM * sizeof(T) + across_swap<T, BM>(kk, ch) * 16) = ra[i];
            } else {
                const int r = c / (8 * WK), ch = c % (8 * WK);
                *(u32x4*)(ta + (ch >> 3) * BM * 128 + r * 128 + along_swap(r, ch & 7) * 16) = ra[i];
            }
        }
#pragma unroll
        for (int i = 0; i < CB; ++i) {
            const int c = tid + i * THREADS;
            if constexpr (B_ACROSS) {
                const int kk = c / (BN / E), ch = c % (BN / E);
                *(u32x4*)(tb + (size_t)kk * BN * sizeof(T) + across_swap<T, BN>(kk, ch) * 16) = rb[i];
            } else {
                const int r = c / (8 * WK), ch = c % (8 * WK);
                *(u32x4*)(tb + (ch >> 3) * BN * 128 + r * 128 + along_swap(r, ch & 7) * 16) = rb[i];
            }
        }
    };

    f32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) mat_zero(acc[i][j]);
    auto multiply = [&](int buf) {
        const char* const ta = lds + buf * S::STAGE + wk * BM * 128;
        const char* const tb = lds + buf * S::STAGE + S::A_BYTES + wk * BN * 128;
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
            MatFrag<T> fa[MT], fb[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if constexpr (A_ACROSS) fa[i] = across_operand<T, BM>(ta, (wm * MT + i) * 32, s, lane);
                else fa[i] = along_operand<T>(ta, (wm * MT + i) * 32 + (lane & 31), s, half);
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if constexpr (B_ACROSS) fb[j] = across_operand<T, BN>(tb, (wn * NT + j) * 32, s, lane);
                else fb[j] = along_operand<T>(tb, (wn * NT + j) * 32 + (lane & 31), s, half);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) mat_mul<T>(acc[i][j], fa[i], fb[j]);
        }
    };

    if (first < last) {                                              // (a split may be empty: it stores zeros)
        fetch(first);
        put(0);
        if (first + 1 < last) fetch(first + 1);
        lds_barrier();
        for (int st = first; st < last; ++st) {
            const int buf = (st - first) & 1;
            multiply(buf);
            if (st + 1 < last) {
                put(buf ^ 1);
                if (st + 2 < last) fetch(st + 2);
                lds_barrier();
            }
        }
    }

    // the result through LDS, PAIR row tiles at a time; of the WK waves that hold sums of the same results each finishes its share of the rows
    constexpr int LANES = 4 * NT, SHARE = 32 / WK, AT_ONCE = 64 / LANES;
    static_assert(SHARE % AT_ONCE == 0 || AT_ONCE > SHARE, "rows of a share");
    float* const mine = (float*)lds + (size_t)wave * S::PAIR * 32 * S::PITCH;
    const float* const from = (const float*)lds + (size_t)(wave - wk) * S::PAIR * 32 * S::PITCH;
    const int c8 = (lane % LANES) * 8, n = n0 + wn * NT * 32 + c8, have = min(8, N - n);
    const int fresh = nt * BN - n;                                   // the first of the eight pixels that no tile before this one has
#pragma unroll
    for (int i0 = 0; i0 < MT; i0 += S::PAIR) {
        lds_barrier();
#pragma unroll
        for (int i = 0; i < S::PAIR; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) mine[(i * 32 + acc_row(r, half)) * S::PITCH + j * 32 + (lane & 31)] = acc[i0 + i][j][r];
        lds_barrier();
        for (int r0 = 0; r0 < SHARE; r0 += AT_ONCE) {
            const int rr = r0 + lane / LANES, row = wk * SHARE + rr;
            const int m = m0 + (S::GATED ? (wm * MT + i0) / 2 * 32 : (wm * MT + i0) * 32) + row;
            const bool ok = rr < SHARE && m < M && have > 0;
            float v[S::PAIR][8];
#pragma unroll
            for (int i = 0; i < S::PAIR; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
                if (rr < SHARE) {
#pragma unroll
                    for (int w = 0; w < WK; ++w) {
                        const float* f = from + ((size_t)w * S::PAIR * 32 + i * 32 + row) * S::PITCH + c8;
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[i][e] += f[e];
                    }
                }
            }
            if constexpr (FORM == PRODUCT_GRAD_MATRIX) {
                if (ok) {
                    if (p.parts) row_store(p.parts + ((size_t)split * M + m) * N + n, have, v[0]);
                    else row_store((T*)p.out + (size_t)m * N + n, have, v[0]);
                }
            } else if constexpr (OUTC == OUT_PLAIN) {
                if (ok) row_store((T*)p.out + ((size_t)image * M + m) * N + n, have, v[0]);
            } else {
                const size_t at = ((size_t)image * M + m) * N + n;
                float bias[S::PAIR], x[8];
#pragma unroll
                for (int i = 0; i < S::PAIR; ++i) bias[i] = p.bias && ok ? ldf((const T*)p.bias + (size_t)i * M + m) : 0.f;
                if (p.extra && ok) row_values((const T*)p.extra + at, have, x);
                else
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = 0.f;
                if constexpr (OUTC == OUT_PROJECT) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[0][e] = activation<false>(v[0][e] + bias[0], p.act, nullptr) + x[e];
                    if (ok) row_store((T*)p.out + at, have, v[0]);
                } else if constexpr (OUTC == OUT_GATED) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[0][e] = activation<false>(v[0][e] + bias[0], p.act, nullptr) * (v[1][e] + bias[1]);
                    if (ok) row_store((T*)p.out + at, have, v[0]);
                } else {
                    const size_t rows = (size_t)S::PAIR * M;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float slope;
                        const float a = activation<true>(v[0][e] + bias[0], p.act, &slope);
                        if constexpr (S::GATED) {
                            const float u = v[1][e] + bias[1];
                            v[1][e] = x[e] * a;
                            v[0][e] = x[e] * u * slope;
                        } else {
                            v[0][e] = x[e] * slope;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < S::PAIR; ++i) {
                        if (ok) row_store((T*)p.out + ((size_t)image * rows + (size_t)i * M + m) * N + n, have, v[i]);
                        if (p.sums) {
                            float sum = 0.f;
#pragma unroll
                            for (int e = 0; e < 8; ++e) sum += ok && e >= fresh && e < have ? v[i][e] : 0.f;
#pragma unroll
                            for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
                            if (rr < SHARE && m < M && lane % LANES == 0)        // (columns past the end: 0)
                                p.sums[((size_t)(image * ntiles + nt) * WN + wn) * rows + (size_t)i * M + m] = sum;
                        }
                    }
                }
            }
        }
    }
}

// tiles: 0: 128 x 128 (2 x 2 waves of 64 x 64); 1: 64 x 64 (two waves along the pixels, two along the stage); 2: 64 x 32 (four along the
// stage); 3: 32 x 128 (few rows)
enum { TILE_LARGE = 0, TILE_MEDIUM = 1, TILE_SMALL = 2, TILE_FLAT = 3 };

template <typename T, int FORM, int OUTC, int MT, int NT, int WM, int WN, int WK>
hipError_t launch_product_tile(const ProductParams& p, hipStream_t s) {
    using S = ProductShape<T, FORM, OUTC, MT, NT, WM, WN, WK>;
    auto kernel = product_kernel<T, FORM, OUTC, MT, NT, WM, WN, WK>;
    hipError_t e = allow_dynamic_lds((const void*)kernel, S::LDS);
    if (e != hipSuccess) return e;
    const size_t tiles = (size_t)((p.M + S::ROWS - 1) / S::ROWS) * ((p.N + S::BN - 1) / S::BN) * (FORM == PRODUCT_GRAD_MATRIX ? p.splits : p.images);
    if (tiles * S::THREADS >= ((size_t)1 << 32)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(S::THREADS), S::LDS, s, p);
    return hipGetLastError();
}

template <typename T, int FORM, int OUTC> hipError_t launch_product_as(const ProductParams& p, int tile, hipStream_t s) {
    switch (tile) {
        case TILE_LARGE: return launch_product_tile<T, FORM, OUTC, 2, 2, 2, 2, 1>(p, s);
        case TILE_MEDIUM: return launch_product_tile<T, FORM, OUTC, 2, 1, 1, 2, 2>(p, s);
        case TILE_SMALL: return launch_product_tile<T, FORM, OUTC, 2, 1, 1, 1, 4>(p, s);
        default:
            if constexpr (OUTC == OUT_GATED || OUTC == OUT_GATED_GRAD) return launch_product_tile<T, FORM, OUTC, 2, 1, 1, 4, 1>(p, s);
            else return launch_product_tile<T, FORM, OUTC, 1, 1, 1, 4, 1>(p, s);
    }
}
template <typename T> hipError_t launch_product_type(const ProductParams& p, int form, int outcome, int tile, hipStream_t s) {
    if (form == PRODUCT_GRAD_INPUT) return launch_product_as<T, PRODUCT_GRAD_INPUT, OUT_PLAIN>(p, tile, s);
    if (form == PRODUCT_GRAD_MATRIX) return launch_product_as<T, PRODUCT_GRAD_MATRIX, OUT_PLAIN>(p, tile, s);
    switch (outcome) {
        case OUT_PROJECT: return launch_product_as<T, PRODUCT_FORWARD, OUT_PROJECT>(p, tile, s);
        case OUT_PROJECT_GRAD: return launch_product_as<T, PRODUCT_FORWARD, OUT_PROJECT_GRAD>(p, tile, s);
        case OUT_GATED: return launch_product_as<T, PRODUCT_FORWARD, OUT_GATED>(p, tile, s);
        default: return launch_product_as<T, PRODUCT_FORWARD, OUT_GATED_GRAD>(p, tile, s);
    }
}
// instantiated in a translation unit per storage type
hipError_t launch_product_f32(const ProductParams& p, int form, int outcome, int tile, hipStream_t s);
hipError_t launch_product_bf16(const ProductParams& p, int form, int outcome, int tile, hipStream_t s);
hipError_t launch_product_f16(const ProductParams& p, int form, int outcome, int tile, hipStream_t s);

}  // namespace gspn
