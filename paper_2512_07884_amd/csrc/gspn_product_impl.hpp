// Products over channels or pixels of [image][channel][pixel] maps on the matrix cores, with what follows them in the same launch:
// the projections with bias, activation and residual, the gated pair, and the three products of their gradients.
//
//     R[m][n] = sum_k A[m][k] B[k][n]
//
// A workgroup owns a tile of BM x BN results and walks the contracted axis in stages of WK times 64 or 128 bytes.  Both operands of a stage
// go through LDS in requests of 16 bytes that run along the rows as they are stored, into NBUF stages of LDS: straight from memory where the rows are whole
// 16-byte pieces and at least a tile long, else through registers, the next stage on its way while the waves multiply (1024 x 1024 channels on 64x64 maps and on
// 63x65 ones, bf16: 26.3 and 30.6 us).  An operand whose contracted axis is contiguous is read from LDS 16 bytes per lane; one whose rows run
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

// Activations of eight values, and their derivatives (one branch for all eight).
// gelu: the normal distribution's tail 1 - Phi(a) = exp(-a^2/2) R(a) for a = |z|, where R(a) = erfcx(a / sqrt 2) / 2 falls slowly: a polynomial of degree 8 in
// t = 1 / (1 + 0.3 a), fitted on [0, 14] for the least relative error (5.8e-8; 3.4e-7 as evaluated in fp32).  The exponential is also what
// the derivative wants.  (With the library's erff a product of 1152 x 1152 channels on two 64x64 maps took 4 us longer.)
template <bool GRAD> __device__ __forceinline__ float gelu(float z, float* slope) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, fabsf(z), 1.f)), e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
    float r = 0.0383786329f;
    r = fmaf(r, t, -0.169167699f);
    r = fmaf(r, t, 0.228663176f);
    r = fmaf(r, t, -0.0765097901f);
    r = fmaf(r, t, 0.142537644f);
    r = fmaf(r, t, 0.094682696f);
    r = fmaf(r, t, 0.121920534f);
    r = fmaf(r, t, 0.119487665f);
    r = fmaf(r, t, 7.17011553e-06f);
    const float tail = r * e, phi = z > 0.f ? 1.f - tail : tail;
    if (GRAD) *slope = fmaf(z * 0.39894228f, e, phi);
    return z * phi;
}
// (the hardware's reciprocal: within one unit of the quotient)
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f)); }
template <bool GRAD> __device__ __forceinline__ void activate(float* z, int act, float* slope) {
    if (act == ACT_NONE) {
        if (GRAD)
#pragma unroll
            for (int e = 0; e < 8; ++e) slope[e] = 1.f;
    } else if (act == ACT_GELU) {
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = gelu<GRAD>(z[e], slope + e);
    } else if (act == ACT_SILU) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float g = logistic(z[e]);
            z[e] *= g;
            if (GRAD) slope[e] = fmaf(z[e], 1.f - g, g);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            z[e] = logistic(z[e]);
            if (GRAD) slope[e] = z[e] * (1.f - z[e]);
        }
    }
}

// where the 16-byte piece c of row r goes in LDS: contracted axis along the row (rows of RB = 128 or 64 bytes) ...
template <int RB> __device__ __forceinline__ int along_swap(int r, int c) { return RB == 128 ? c ^ ((r >> 1) & 7) : c ^ ((r >> 2) & 3); }
// ... and across the rows (rows of COLS values)
template <typename T, int COLS> __device__ __forceinline__ int across_swap(int r, int c) {
    if constexpr (sizeof(T) == 4) return COLS >= 64 ? c ^ (((r >> 3) & 1) << 3) : c;
    else return COLS >= 128 ? c ^ ((r & 3) << 2) : (COLS == 64 ? c ^ (((r >> 1) & 1) << 2) : c);
}

template <typename T, int RB> __device__ __forceinline__ MatFrag<T> along_operand(const char* tile, int r, int s, int half) {
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const u32x4 a = *(const u32x4*)(tile + r * RB + along_swap<RB>(r, 4 * s + 2 * half + j) * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) f.v[4 * j + i] = __uint_as_float(a[i]);
        }
    } else {
        f.w = *(const u32x4*)(tile + r * RB + along_swap<RB>(r, 2 * s + half) * 16);
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

// 16 bytes per lane from memory to LDS without registers in between: lane l's go to `to` + 16 * l.  The request is counted like a load (vmcnt) and
// is not known to the compiler: it writes no register, and what it writes in LDS is read behind stage_arrived() alone.
__device__ __forceinline__ void lds_request(const void* base, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void lds_request_at(const void* at, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(to), "v"(at) : "memory", "m0");
}
// all but the `later` youngest requests of the wave have arrived, and those of the workgroup's other waves
template <int LATER> __device__ __forceinline__ void stage_arrived() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(LATER) : "memory");
}
__device__ const uint32_t zero_piece[4] = {0, 0, 0, 0};              // what is requested in place of positions past the end

template <typename T, int FORM, int OUTC, int MT, int NT, int WM, int WN, int WK, int RB = 128, int NBUF = 2>
struct ProductShape {
    static constexpr int BM = 32 * MT * WM, BN = 32 * NT * WN, THREADS = 64 * WM * WN * WK;
    static constexpr int BK = RB / (int)sizeof(T), E = 16 / (int)sizeof(T);
    static constexpr int A_BYTES = WK * BM * RB, B_BYTES = WK * BN * RB, STAGE = A_BYTES + B_BYTES;
    static constexpr bool GATED = OUTC == OUT_GATED || OUTC == OUT_GATED_GRAD;
    static constexpr int PAIR = GATED ? 2 : 1;                       // row tiles that are finished together
    static constexpr int PITCH = 32 * NT + 4;                        // floats of a row of the result in LDS
    static constexpr int HROWS = WK == 1 ? 16 : 32;                  // rows of a row tile that are finished together
    static constexpr int FINISH = WM * WN * WK * PAIR * HROWS * PITCH * 4;
    static constexpr int BUFFERS = NBUF;
    static constexpr int LDS = BUFFERS * STAGE > FINISH ? BUFFERS * STAGE : FINISH;
    static constexpr int ROWS = GATED ? BM / 2 : BM;                 // rows of the result
};

template <typename T, int FORM, int OUTC, int MT, int NT, int WM, int WN, int WK, bool DIRECT, int RB, int NBUF>
__global__ void __launch_bounds__(64 * WM * WN * WK) product_kernel(const ProductParams p) {
    using S = ProductShape<T, FORM, OUTC, MT, NT, WM, WN, WK, RB, NBUF>;
    constexpr int BM = S::BM, BN = S::BN, BK = S::BK, E = S::E, THREADS = S::THREADS;
    constexpr bool A_ACROSS = FORM == PRODUCT_GRAD_INPUT, B_ACROSS = FORM != PRODUCT_GRAD_MATRIX;
    constexpr int PR = RB / 16, CA = WK * BM * PR / THREADS, CB = WK * BN * PR / THREADS;        // 16-byte pieces of a row; of a stage per thread
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
                const int r = a_row(c / (PR * WK)), k = k0 + (c % (PR * WK)) * E;
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
                const int r = min(n0 + c / (PR * WK), N - 1), k = k0 + (c % (PR * WK)) * E;
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
                const int r = c / (PR * WK), ch = c % (PR * WK);
                *(u32x4*)(ta + ch / PR * BM * RB + r * RB + along_swap<RB>(r, ch % PR) * 16) = ra[i];
            }
        }
#pragma unroll
        for (int i = 0; i < CB; ++i) {
            const int c = tid + i * THREADS;
            if constexpr (B_ACROSS) {
                const int kk = c / (BN / E), ch = c % (BN / E);
                *(u32x4*)(tb + (size_t)kk * BN * sizeof(T) + across_swap<T, BN>(kk, ch) * 16) = rb[i];
            } else {
                const int r = c / (PR * WK), ch = c % (PR * WK);
                *(u32x4*)(tb + ch / PR * BN * RB + r * RB + along_swap<RB>(r, ch % PR) * 16) = rb[i];
            }
        }
    };

    f32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) mat_zero(acc[i][j]);
    auto multiply = [&](int buf) {
        const char* const ta = lds + buf * S::STAGE + wk * BM * RB;
        const char* const tb = lds + buf * S::STAGE + S::A_BYTES + wk * BN * RB;
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
            MatFrag<T> fa[MT], fb[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if constexpr (A_ACROSS) fa[i] = across_operand<T, BM>(ta, (wm * MT + i) * 32, s, lane);
                else fa[i] = along_operand<T, RB>(ta, (wm * MT + i) * 32 + (lane & 31), s, half);
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if constexpr (B_ACROSS) fb[j] = across_operand<T, BN>(tb, (wn * NT + j) * 32, s, lane);
                else fb[j] = along_operand<T, RB>(tb, (wn * NT + j) * 32 + (lane & 31), s, half);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) mat_mul<T>(acc[i][j], fa[i], fb[j]);
        }
    };

    if constexpr (DIRECT) {
        // a wave requests CA (CB) kilobytes of the stage's tiles, in the order of LDS; the exchange of a row's pieces is in the addresses
        uint32_t oa[CA], ob[CB];
#pragma unroll
        for (int i = 0; i < CA; ++i) {
            const int c = (wave * CA + i) * 64 + lane;
            if constexpr (A_ACROSS) {
                const int kk = c / (BM / E), ch = across_swap<T, BM>(kk, c % (BM / E));
                oa[i] = (uint32_t)(((size_t)kk * M + m0 + ch * E) * sizeof(T));
            } else {
                const int g = c / (BM * PR), r = c / PR % BM, ch = along_swap<RB>(r, c % PR);
                oa[i] = (uint32_t)(((size_t)a_row(r) * K + g * BK + ch * E) * sizeof(T));
            }
        }
#pragma unroll
        for (int i = 0; i < CB; ++i) {
            const int c = (wave * CB + i) * 64 + lane;
            if constexpr (B_ACROSS) {
                const int kk = c / (BN / E), ch = across_swap<T, BN>(kk, c % (BN / E));
                ob[i] = (uint32_t)(((size_t)kk * N + n0 + ch * E) * sizeof(T));
            } else {
                const int g = c / (BN * PR), r = c / PR % BN, ch = along_swap<RB>(r, c % PR);
                ob[i] = (uint32_t)(((size_t)min(n0 + r, N - 1) * K + g * BK + ch * E) * sizeof(T));
            }
        }
        const uint32_t at = (uint32_t)(uintptr_t)lds_ptr(lds);
        auto request = [&](int st, int buf) {
            int k0 = st * STEP;
            const T *a = A, *b = B;
            if constexpr (FORM == PRODUCT_GRAD_MATRIX) {
                const int im = st / stages;
                k0 = (st - im * stages) * STEP;
                a += (size_t)im * M * K;
                b += (size_t)im * N * K;
            }
            a += A_ACROSS ? (size_t)k0 * M : (size_t)k0;
            b += B_ACROSS ? (size_t)k0 * N : (size_t)k0;
            const uint32_t ta = at + buf * S::STAGE + wave * CA * 1024, tb = at + buf * S::STAGE + S::A_BYTES + wave * CB * 1024;
            if (k0 + STEP <= K) {
#pragma unroll
                for (int i = 0; i < CA; ++i) lds_request(a, oa[i], ta + i * 1024);
#pragma unroll
                for (int i = 0; i < CB; ++i) lds_request(b, ob[i], tb + i * 1024);
            } else {
                const int rest = K - k0;                             // positions of the stage that exist
#pragma unroll
                for (int i = 0; i < CA; ++i) {
                    const int c = (wave * CA + i) * 64 + lane;
                    const int k = A_ACROSS ? c / (BM / E) : c / (BM * PR) * BK + along_swap<RB>(c / PR % BM, c % PR) * E;
                    lds_request_at(k < rest ? (const void*)((const char*)a + oa[i]) : zero_piece, ta + i * 1024);
                }
#pragma unroll
                for (int i = 0; i < CB; ++i) {
                    const int c = (wave * CB + i) * 64 + lane;
                    const int k = B_ACROSS ? c / (BN / E) : c / (BN * PR) * BK + along_swap<RB>(c / PR % BN, c % PR) * E;
                    lds_request_at(k < rest ? (const void*)((const char*)b + ob[i]) : zero_piece, tb + i * 1024);
                }
            }
        };
        if (first < last) {
            constexpr int AHEAD = NBUF - 1;                          // stages on their way
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (first + i < last) request(first + i, i);
            int buf = 0;
            for (int st = first; st < last; ++st) {
                // this stage is here, and every wave has read the one before
                if (st + AHEAD <= last) stage_arrived<(AHEAD - 1) * (CA + CB)>();
                else stage_arrived<0>();
                if (st + AHEAD < last) request(st + AHEAD, buf == 0 ? NBUF - 1 : buf - 1);
                multiply(buf);
                buf = buf + 1 == NBUF ? 0 : buf + 1;
            }
        }
    } else if (first < last) {                                       // (a split may be empty: it stores zeros)
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
    constexpr int HR = S::HROWS, HALVES = 32 / HR, LANES = 4 * NT, SHARE = HR / WK, AT_ONCE = 64 / LANES, TURNS = SHARE > AT_ONCE ? SHARE / AT_ONCE : 1;
    constexpr int BLOCKS = MT / S::PAIR * HALVES;
    float* const mine = (float*)lds + (size_t)wave * S::PAIR * HR * S::PITCH;
    const float* const from = (const float*)lds + (size_t)(wave - wk) * S::PAIR * HR * S::PITCH;
    const int c8 = (lane % LANES) * 8, n = n0 + wn * NT * 32 + c8, have = min(8, N - n);
    const int fresh = nt * BN - n;                                   // the first of the eight pixels that no tile before this one has
    auto row_of = [&](int block, int turn) { return m0 + (wm * BLOCKS + block) * HR + wk * SHARE + turn * AT_ONCE + lane / LANES; };
    const bool rows_here = AT_ONCE <= SHARE || lane / LANES < SHARE;
    // What a row of the result is joined with is requested for all rows at once, one wait where the rows one by one would take eight
    // (a workgroup of sixteen waves has registers for one step of the loop below at a time).
    constexpr bool JOINS = OUTC != OUT_PLAIN;
    constexpr int W = (int)sizeof(T) / 2;                            // 16-byte pieces of eight values
    constexpr int HELD = !JOINS || THREADS >= 1024 ? 1 : BLOCKS;
    u32x4 other[HELD][TURNS][W];
    float bias[HELD][TURNS][S::PAIR];
    const bool whole = n0 + BN <= N;                                 // (uniform) all columns of the tile exist
    auto join = [&](int block, int to) {
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const int m = min(row_of(block, t), M - 1);              // (rows past the end: the last one, nothing is stored)
#pragma unroll
            for (int w = 0; w < W; ++w) {
                other[to][t][w] = u32x4{0, 0, 0, 0};
                if (p.extra && whole) other[to][t][w] = rg_load((const T*)p.extra + ((size_t)image * M + m) * N + n + w * E);
            }
#pragma unroll
            for (int j = 0; j < S::PAIR; ++j) bias[to][t][j] = p.bias ? ldf((const T*)p.bias + (size_t)j * M + m) : 0.f;
        }
    };
    if constexpr (JOINS && HELD == BLOCKS) {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) join(i, i);
    }
#pragma unroll
    for (int block = 0; block < BLOCKS; ++block) {
        constexpr bool ONE = HELD == 1;
        if constexpr (JOINS && HELD != BLOCKS) join(block, 0);
        lds_barrier();
#pragma unroll
        for (int i = 0; i < S::PAIR; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int r = 0; r < 16 / HALVES; ++r)
                    mine[(i * HR + acc_row(r, half)) * S::PITCH + j * 32 + (lane & 31)] = acc[block / HALVES * S::PAIR + i][j][block % HALVES * 8 + r];
        lds_barrier();
#pragma unroll
        for (int turn = 0; turn < TURNS; ++turn) {
            const int row = wk * SHARE + turn * AT_ONCE + lane / LANES, m = row_of(block, turn);
            const bool ok = rows_here && m < M && have > 0;
            float v[S::PAIR][8];
#pragma unroll
            for (int i = 0; i < S::PAIR; ++i) {
                const float* f = from + ((size_t)i * HR + (rows_here ? row : 0)) * S::PITCH + c8;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = f[e];
#pragma unroll
                for (int w = 1; w < WK; ++w)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[i][e] += f[(size_t)w * S::PAIR * HR * S::PITCH + e];
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
#pragma unroll
                for (int i = 0; i < S::PAIR; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[i][e] += bias[ONE ? 0 : block][turn][i];
                float x[8];
                if (p.extra && !whole) {
                    if (ok) row_values_slow((const T*)p.extra + at, have, x);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = rg_elem<T>(other[ONE ? 0 : block][turn][e / E], e % E);
                }
                if constexpr (OUTC == OUT_PROJECT) {
                    activate<false>(v[0], p.act, nullptr);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[0][e] += x[e];
                    if (ok) row_store((T*)p.out + at, have, v[0]);
                } else if constexpr (OUTC == OUT_GATED) {
                    activate<false>(v[0], p.act, nullptr);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[0][e] *= v[1][e];
                    if (ok) row_store((T*)p.out + at, have, v[0]);
                } else {
                    const size_t rows = (size_t)S::PAIR * M;
                    float slope[8];
                    activate<true>(v[0], p.act, slope);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if constexpr (S::GATED) {
                            const float a = v[0][e];
                            v[0][e] = x[e] * v[1][e] * slope[e];
                            v[1][e] = x[e] * a;
                        } else {
                            v[0][e] = x[e] * slope[e];
                        }
                    }
#pragma unroll
                    for (int i = 0; i < S::PAIR; ++i) {
                        if (ok) row_store((T*)p.out + ((size_t)image * rows + (size_t)i * M + m) * N + n, have, v[i]);
                        if (p.sums) {
                            float sum = 0.f;
                            if (whole && fresh <= 0) {
#pragma unroll
                                for (int e = 0; e < 8; ++e) sum += v[i][e];
                            } else {
#pragma unroll
                                for (int e = 0; e < 8; ++e) sum += ok && e >= fresh && e < have ? v[i][e] : 0.f;
                            }
#pragma unroll
                            for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
                            if (rows_here && m < M && lane % LANES == 0)         // (columns past the end: 0)
                                p.sums[((size_t)(image * ntiles + nt) * WN + wn) * rows + (size_t)i * M + m] = sum;
                        }
                    }
                }
            }
        }
    }
}

// tiles: 0: 128 x 128 (2 x 2 waves of 64 x 64); 1: 64 x 64 (two waves along the pixels, two along the stage); 2: 64 x 32 (four along the
// stage); 3: 32 x 128 (four waves along the pixels; gated: 64 rows of P); 4: 256 x 256 (4 x 4 waves)
enum { TILE_LARGE = 0, TILE_MEDIUM = 1, TILE_SMALL = 2, TILE_FLAT = 3, TILE_HUGE = 4 };

// Requests straight to LDS: whole rows of 16-byte pieces, and offsets of 32 bits
template <typename S> bool product_direct(const ProductParams& p, int form, int e, int width) {
    const size_t rows = (S::GATED ? 2 : 1) * (size_t)p.M;
    const bool a_across = form == PRODUCT_GRAD_INPUT, b_across = form != PRODUCT_GRAD_MATRIX;
    if ((a_across && (p.M % e || p.M < S::BM)) || (b_across && (p.N % e || p.N < S::BN)) || ((!a_across || !b_across) && p.K % e)) return false;
    const size_t step = (size_t)S::A_BYTES / (S::BM * width);        // positions of a stage
    return (a_across ? step * p.M : rows * p.K) * width < ((size_t)1 << 32) && (b_across ? step * p.N : (size_t)p.N * p.K) * width < ((size_t)1 << 32);
}

template <typename T, int FORM, int OUTC, int MT, int NT, int WM, int WN, int WK, int RB = 128, int NBUF = 2, bool ONLY_DIRECT = false>
hipError_t launch_product_tile(const ProductParams& p, hipStream_t s) {
    using S = ProductShape<T, FORM, OUTC, MT, NT, WM, WN, WK, RB, NBUF>;
    using R = ProductShape<T, FORM, OUTC, MT, NT, WM, WN, WK, RB, 2>;       // through registers: two buffers
    const bool direct = product_direct<S>(p, FORM, S::E, sizeof(T));
    auto kernel = product_kernel<T, FORM, OUTC, MT, NT, WM, WN, WK, true, RB, NBUF>;
    if constexpr (ONLY_DIRECT) { if (!direct) return hipErrorInvalidValue; }         // (product_tile does not choose it then)
    else if (!direct) kernel = product_kernel<T, FORM, OUTC, MT, NT, WM, WN, WK, false, RB, 2>;
    const int lds = direct ? S::LDS : R::LDS;
    hipError_t e = allow_dynamic_lds((const void*)kernel, lds);
    if (e != hipSuccess) return e;
    const size_t tiles = (size_t)((p.M + S::ROWS - 1) / S::ROWS) * ((p.N + S::BN - 1) / S::BN) * (FORM == PRODUCT_GRAD_MATRIX ? p.splits : p.images);
    if (tiles * S::THREADS >= ((size_t)1 << 32)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(S::THREADS), lds, s, p);
    return hipGetLastError();
}

// Bytes of a row in a stage: 64, which leaves room for more workgroups on a CU, but 128 for flat tiles of one row block (fewer turns; 64 is less than a request per
// thread) and 256 x 256, and for the 64 x 64 tiles of the matrix's gradient, which read both operands along their rows (512 x 512 on two 64x64 maps in
// bf16, at the best number of stretches: 18 us, with 64 bytes 21).
template <typename T, int FORM, int OUTC> hipError_t launch_product_as(const ProductParams& p, int tile, hipStream_t s) {
    if (tile == TILE_HUGE) {
        if constexpr (sizeof(T) == 2) return launch_product_tile<T, FORM, OUTC, 2, 2, 4, 4, 1, 128, 2, true>(p, s);
        else return hipErrorInvalidValue;               // (product_tile does not choose it)
    }
    if (tile == TILE_LARGE) return launch_product_tile<T, FORM, OUTC, 2, 2, 2, 2, 1, 64, 2>(p, s);
    if constexpr (FORM == PRODUCT_GRAD_MATRIX) return launch_product_tile<T, FORM, OUTC, 2, 1, 1, 2, 2>(p, s);
    else {
        if (tile == TILE_MEDIUM) return launch_product_tile<T, FORM, OUTC, 2, 1, 1, 2, 2, 64, 2>(p, s);
        if (tile == TILE_SMALL) return launch_product_tile<T, FORM, OUTC, 2, 1, 1, 1, 4, 64, 2>(p, s);
        if constexpr (OUTC == OUT_GATED || OUTC == OUT_GATED_GRAD) return launch_product_tile<T, FORM, OUTC, 2, 1, 1, 4, 1, 64, 2>(p, s);
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
