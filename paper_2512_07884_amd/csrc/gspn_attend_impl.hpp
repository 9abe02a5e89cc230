// Cross attention of feature maps to an encoder's states, forward and backward, on the matrix cores.
//
//     s[t][n] = scale * sum_d k[t][d] q[d][n] ,   p = softmax over the tokens t that take part ,   out[d][n] = sum_t p[t][n] v[t][d]
//
// The maps are channel-first, so a lane is a position n throughout the forward call: scores are computed as [token][position] (the
// positions are the columns of the result), the softmax of a position stays within two lanes, and its weights are already the operand that the
// product with v wants (out as [channel][position], which is how the maps are stored).  Nothing of the scores leaves the registers:
// one pass over the tokens with the running maximum and sum of each position, both in fp32.  The weights are rounded to the storage type for
// the product with v (the sum is of the unrounded ones); the error is that of one more rounding of out.
// Tokens that take no part are stored as zeros on the way into LDS and their scores are replaced by -inf: whatever they hold is never used.
// A position without any token gets 0 and lse = -inf.
#pragma once
#include "gspn_matrix.hpp"
#include "gspn_block.hpp"

namespace gspn {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// the value of the lane 32 away as well: both halves of the wave
__device__ __forceinline__ float other_half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// rows of tokens in LDS: read along the row (16 bytes per lane; an odd number of 16-byte pieces: 16 rows on all banks) ...
template <typename T, int DT> constexpr int along_pitch() { return DT * 32 * (int)sizeof(T) + 16; }
// ... and across the rows, turned (four rows of 64 bytes on all banks; fp32: rows four apart on both halves of the banks)
template <typename T, int DT> constexpr int across_pitch() {
    return sizeof(T) == 4 ? DT * 128 + 32 : (DT % 2 ? DT * 64 : DT * 64 + 64);
}

// operand A from rows of tokens: the channels contracted (step s), row r
template <typename T, int DT> __device__ __forceinline__ MatFrag<T> token_rows(const char* tile, int r, int s, int half) {
    return mat_contiguous<T>(tile + r * along_pitch<T, DT>() + (16 * s + 8 * half) * (int)sizeof(T));
}
// ... and the tokens contracted, in the order of an accumulator's rows (16 * s ...), channels dt * 32 ...
template <typename T, int DT> __device__ __forceinline__ MatFrag<T> token_columns(const char* tile, int dt, int s, int lane) {
    constexpr int PITCH = across_pitch<T, DT>();
    const int half = lane >> 5;
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f.v[i] = *(const float*)(tile + acc_row(8 * s + i, half) * PITCH + (dt * 32 + (lane & 31)) * 4);
    } else {
        const int j = lane & 15, col = dt * 32 + (lane & 16) + (j & 3) * 4;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x2 v = lds_turned(tile + (16 * s + 8 * i + 4 * half + (j >> 2)) * PITCH + col * 2);
            f.w[2 * i] = v.x; f.w[2 * i + 1] = v.y;
        }
    }
    return f;
}

// eight channels of a position, rows N apart, as an operand: channels d .. d + 7 at p, all of them or none
template <typename T> __device__ __forceinline__ MatFrag<T> position_channels(const T* p, size_t N, bool have) {
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f.v[i] = have ? p[i * N] : 0.f;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t lo = 0, hi = 0;
            if (have) { lo = *(const uint16_t*)(p + (2 * i) * N); hi = *(const uint16_t*)(p + (2 * i + 1) * N); }
            f.w[i] = lo | hi << 16;
        }
    }
    return f;
}
template <typename T> __device__ __forceinline__ float frag_value(const MatFrag<T>& f, int i) {
    if constexpr (sizeof(T) == 4) return f.v[i];
    else return rg_elem<T>(f.w, i);
}

// A stage of TB tokens on its way to LDS: keys and values of one head, and which of the tokens take part
template <typename T, int DT, int TB> struct TokenStage {
    static constexpr int E = 16 / (int)sizeof(T), PIECES = DT * 32 / E;            // 16-byte pieces of a token's row
    static constexpr int COUNT = TB * PIECES / 256;                                // per thread
    static_assert(TB * PIECES % 256 == 0, "pieces per thread");
    u32x4 k[COUNT], v[COUNT];
    uint32_t here[(TB + 63) / 64];

    __device__ __forceinline__ void fetch(const AttendParams& p, int b, int head, int t0, int tid) {
#pragma unroll
        for (int i = 0; i < (TB + 63) / 64; ++i) {
            const int t = t0 + 64 * i + (tid & 63);
            here[i] = t < p.L && t < t0 + TB ? (p.mask ? p.mask[(size_t)b * p.L + t] : 1) : 0;
        }
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = tid + i * 256, t = min(t0 + c / PIECES, p.L - 1), d = c % PIECES * E;
            k[i] = v[i] = u32x4{0, 0, 0, 0};
            if (d < p.D) {
                const size_t at = (((size_t)b * p.L + t) * p.kv + head) * p.D + d;
                k[i] = *(const u32x4*)((const T*)p.k + at);
                v[i] = *(const u32x4*)((const T*)p.v + at);
            }
        }
    }
    // bits of the tokens that take part, 64 of them
    __device__ __forceinline__ uint64_t bits(int i) const { return __ballot(here[i] != 0); }
    // ROWS of k and v into LDS at two pitches: to k_at, v_at (and k a second time to k2_at)
    __device__ __forceinline__ void put(char* k_at, int k_pitch, char* v_at, int v_pitch, char* k2_at, int k2_pitch, int tid) const {
        uint64_t w[(TB + 63) / 64];
#pragma unroll
        for (int i = 0; i < (TB + 63) / 64; ++i) w[i] = bits(i);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = tid + i * 256, r = c / PIECES, o = c % PIECES * 16;
            const bool in = (w[TB > 64 ? r >> 6 : 0] >> (r & 63)) & 1;
            const u32x4 zero = {0, 0, 0, 0};
            *(u32x4*)(k_at + r * k_pitch + o) = in ? k[i] : zero;
            *(u32x4*)(v_at + r * v_pitch + o) = in ? v[i] : zero;
            if (k2_at) *(u32x4*)(k2_at + r * k2_pitch + o) = in ? k[i] : zero;
        }
    }
};

// BY_TOKEN: the four waves of a workgroup hold the same 32 positions and take 32 of the 128 tokens of a stage each (few positions); else
// each holds 32 * PT positions of its own and all take the 64 tokens of a stage.
template <typename T, int DT, int PT, bool BY_TOKEN> struct AttendShape {
    static constexpr int TB = BY_TOKEN ? 128 : 64;
    static constexpr int K_BYTES = TB * along_pitch<T, DT>(), V_BYTES = TB * across_pitch<T, DT>(), STAGE = K_BYTES + V_BYTES;
    static constexpr int BUFFERS = 2 * STAGE <= 160 * 1024 ? 2 : 1;
    static constexpr int JOIN = BY_TOKEN ? 4 * (DT * 32 + 2) * 32 * 4 : 0;
    static constexpr int LDS = BUFFERS * STAGE > JOIN ? BUFFERS * STAGE : JOIN;
    static constexpr int COLUMNS = BY_TOKEN ? 32 : 128 * PT;
};

template <typename T, int DT, int PT, bool BY_TOKEN>
__global__ void __launch_bounds__(256) attend_kernel(const AttendParams p) {
    using S = AttendShape<T, DT, PT, BY_TOKEN>;
    constexpr int TB = S::TB, KS = DT * 2, TILES = BY_TOKEN ? 1 : TB / 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int columns = p.per * p.N, tiles = (columns + S::COLUMNS - 1) / S::COLUMNS;
    unsigned item = xcd_contiguous_item(blockIdx.x, gridDim.x);
    const int split = item % p.splits;
    item /= p.splits;
    const int tile = item % tiles, group = item / tiles, head = group % p.kv, b = group / p.kv;
    const int stages = (p.L + TB - 1) / TB;
    const int first = (int)((long)stages * split / p.splits), last = (int)((long)stages * (split + 1) / p.splits);

    // the lane's positions
    size_t base[PT];                                                // of the position's first channel
    MatFrag<T> q[PT][KS];
    int col[PT];
#pragma unroll
    for (int t = 0; t < PT; ++t) {
        col[t] = tile * S::COLUMNS + (BY_TOKEN ? 0 : wave * 32 * PT) + t * 32 + (lane & 31);
        const int c = min(col[t], columns - 1), g = c / p.N;
        base[t] = ((size_t)b * p.heads + head * p.per + g) * p.D * p.N + (c - g * p.N);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int d = 16 * s + 8 * half;
            q[t][s] = position_channels<T>((const T*)p.q + base[t] + (size_t)d * p.N, p.N, d < p.D);
        }
    }
    f32x16 o[PT][DT];
    float top[PT], sum[PT];                                         // running maximum (in powers of two) and sum of the lane's half
#pragma unroll
    for (int t = 0; t < PT; ++t) {
        top[t] = -__builtin_huge_valf(); sum[t] = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) mat_zero(o[t][i]);
    }
    const float c2 = p.scale * LOG2E;

    auto tokens = [&](const char* kt, const char* vt, uint32_t word) {
        // word: bit r = token r of the 32 takes part
        const uint32_t w = word >> (4 * half);
#pragma unroll
        for (int t = 0; t < PT; ++t) {
            f32x16 s;
            mat_zero(s);
#pragma unroll
            for (int i = 0; i < KS; ++i) mat_mul<T>(s, token_rows<T, DT>(kt, lane & 31, i, half), q[t][i]);
            if (word != 0xffffffffu) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = (w >> (8 * (r >> 2) + (r & 3))) & 1 ? s[r] : -__builtin_huge_valf();
            }
            float m = s[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) m = fmaxf(m, s[r]);
            m = other_half_max(m) * c2;
            // The maximum is a reference that keeps the powers in range: it is moved only where it has grown by more than 2^8
            if (__ballot(m > top[t] + 8.f)) {
                const float next = fmaxf(top[t], m), shrink = next == -__builtin_huge_valf() ? 1.f : __builtin_amdgcn_exp2f(top[t] - next);
                top[t] = next;
                sum[t] *= shrink;
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[t][i][r] *= shrink;
            }
            const float ref = top[t] == -__builtin_huge_valf() ? 0.f : top[t];
            float e[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) { e[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c2, -ref)); sum[t] += e[r]; }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const MatFrag<T> w8 = mat_from_acc<T>(e + 8 * j);
#pragma unroll
                for (int i = 0; i < DT; ++i) mat_mul<T>(o[t][i], token_columns<T, DT>(vt, i, j, lane), w8);
            }
        }
    };

    TokenStage<T, DT, TB> next;
    if (first < last) {
        next.fetch(p, b, head, first * TB, tid);
        for (int st = first; st < last; ++st) {
            const int buf = S::BUFFERS == 2 ? (st - first) & 1 : 0;
            char* const kt = lds + buf * S::STAGE;
            char* const vt = kt + S::K_BYTES;
            if (S::BUFFERS == 1 && st > first) lds_barrier();       // (the stage before has been read)
            next.put(kt, along_pitch<T, DT>(), vt, across_pitch<T, DT>(), nullptr, 0, tid);
            uint64_t in = next.bits(0);
            if (BY_TOKEN && wave >= 2) in = next.bits((TB + 63) / 64 - 1);
            if (st + 1 < last) next.fetch(p, b, head, (st + 1) * TB, tid);
            lds_barrier();
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                const int r = BY_TOKEN ? wave * 32 : i * 32;
                const uint32_t word = (uint32_t)(in >> (r & 32));
                if (word) tokens(kt + r * along_pitch<T, DT>(), vt + r * across_pitch<T, DT>(), word);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < PT; ++t) sum[t] = other_half_sum(sum[t]);

    if constexpr (BY_TOKEN) {
        // the four waves' states meet in LDS: [wave][channel][position], then maximum and sum
        float* const join = (float*)lds;
        float* const tops = join + 4 * DT * 32 * 32;
        lds_barrier();
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) join[(wave * DT * 32 + i * 32 + acc_row(r, half)) * 32 + (lane & 31)] = o[0][i][r];
        if (half == 0) { tops[wave * 32 + lane] = top[0]; tops[128 + wave * 32 + lane] = sum[0]; }
        lds_barrier();
        const int n = tid & 31;                                     // a thread finishes every eighth channel of a position
        float m = tops[n], f[4], l = 0.f;
#pragma unroll
        for (int w = 1; w < 4; ++w) m = fmaxf(m, tops[w * 32 + n]);
        const float ref = m == -__builtin_huge_valf() ? 0.f : m;
#pragma unroll
        for (int w = 0; w < 4; ++w) { f[w] = __builtin_amdgcn_exp2f(tops[w * 32 + n] - ref); l += f[w] * tops[128 + w * 32 + n]; }
        const int column = tile * 32 + n;
        if (column >= columns) return;
        const int g = column / p.N;
        const size_t at = ((size_t)b * p.heads + head * p.per + g) * p.D * p.N + (column - g * p.N);
        if (p.splits > 1) {
            // [split][group][channel, then maximum and sum][column]
            float* const state = p.parts + ((size_t)split * p.B * p.kv + group) * (p.D + 2) * columns + column;
            for (int d = tid >> 5; d < p.D; d += 8) {
                float v = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) v += f[w] * join[(w * DT * 32 + d) * 32 + n];
                state[(size_t)d * columns] = v;
            }
            if (tid < 32) { state[(size_t)p.D * columns] = m; state[(size_t)(p.D + 1) * columns] = l; }
            return;
        }
        const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);         // (NaN stays NaN)
        for (int d = tid >> 5; d < p.D; d += 8) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) v += f[w] * join[(w * DT * 32 + d) * 32 + n];
            stf((T*)p.out + at + (size_t)d * p.N, v * inv);
        }
        if (p.lse && tid < 32) p.lse[((size_t)b * p.heads + head * p.per + g) * p.N + (column - g * p.N)] = (m + __builtin_amdgcn_logf(l)) * LN2;
    } else {
#pragma unroll
        for (int t = 0; t < PT; ++t) {
            if (col[t] >= columns) continue;
            const float l = sum[t], inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int d = i * 32 + acc_row(r, half);
                    if (d < p.D) stf((T*)p.out + base[t] + (size_t)d * p.N, o[t][i][r] * inv);
                }
            if (p.lse && half == 0) {
                const int g = col[t] / p.N;
                p.lse[((size_t)b * p.heads + head * p.per + g) * p.N + (col[t] - g * p.N)] = (top[t] + __builtin_amdgcn_logf(l)) * LN2;
            }
        }
    }
}

// joins the stretches of the tokens: a thread per channel of a column
template <typename T> __global__ void __launch_bounds__(256) attend_join_kernel(const AttendParams p) {
    const int columns = p.per * p.N;
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, groups = (size_t)p.B * p.kv;
    if (i >= groups * p.D * columns) return;
    const int column = i % columns, d = (i / columns) % p.D;
    const size_t group = i / columns / p.D, step = groups * (p.D + 2) * columns;
    const float* state = p.parts + group * (p.D + 2) * columns + column;
    float m = -__builtin_huge_valf(), l = 0.f, v = 0.f;
    for (int s = 0; s < p.splits; ++s) m = fmaxf(m, state[s * step + (size_t)p.D * columns]);
    const float ref = m == -__builtin_huge_valf() ? 0.f : m;
    for (int s = 0; s < p.splits; ++s) {
        const float f = __builtin_amdgcn_exp2f(state[s * step + (size_t)p.D * columns] - ref);
        l += f * state[s * step + (size_t)(p.D + 1) * columns];
        v += f * state[s * step + (size_t)d * columns];
    }
    const int head = group % p.kv, b = group / p.kv, g = column / p.N;
    const size_t plane = (size_t)b * p.heads + head * p.per + g;
    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
    stf((T*)p.out + (plane * p.D + d) * p.N + (column - g * p.N), v * inv);
    if (p.lse && d == 0) p.lse[plane * p.N + (column - g * p.N)] = (m + __builtin_amdgcn_logf(l)) * LN2;
}

// ---- backward -----------------------------------------------------------------------------------------------------------------------
//     p = exp(s - lse) ,  dp[t][n] = sum_d v[t][d] gout[d][n] ,  ds = p (dp - delta[n]) ,  delta[n] = sum_t p dp = sum_d gout out
//     gq[d][n] = scale sum_t ds k[t][d] ,   gk[t][d] = scale sum_n ds q[d][n] ,   gv[t][d] = sum_n p gout[d][n]
// Two launches: gq (and delta) with a lane per position as in the forward call, then gk and gv with a lane per token and the positions
// walked in stages.  p and ds are rounded to the storage type for the products, everything else is fp32.

template <typename T, int DT> struct AttendGradShape {
    static constexpr int TB = 64;
    static constexpr int K_BYTES = TB * along_pitch<T, DT>(), K2_BYTES = TB * across_pitch<T, DT>(), STAGE = 2 * K_BYTES + K2_BYTES;
    static constexpr int BUFFERS = 2 * STAGE <= 160 * 1024 ? 2 : 1;
    static constexpr int LDS = BUFFERS * STAGE;
};

// gq, and delta for the launch after it.  Up to 64 tokens (one stage) delta is the sum over the tokens, in a pass of its own over what LDS holds;
// else gout * out.
template <typename T, int DT>
__global__ void __launch_bounds__(256) attend_grad_q_kernel(const AttendParams p) {
    using S = AttendGradShape<T, DT>;
    constexpr int TB = S::TB, KS = DT * 2;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int columns = p.per * p.N, tiles = (columns + 127) / 128;
    const unsigned item = xcd_contiguous_item(blockIdx.x, gridDim.x);
    const int tile = item % tiles, group = item / tiles, head = group % p.kv, b = group / p.kv;
    const int stages = (p.L + TB - 1) / TB;

    const int col = tile * 128 + wave * 32 + (lane & 31), c = min(col, columns - 1), g = c / p.N;
    const size_t plane = (size_t)b * p.heads + head * p.per + g, pos = plane * p.N + (c - g * p.N);
    const size_t base = plane * p.D * p.N + (c - g * p.N);
    MatFrag<T> q[KS], go[KS];
    float delta = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int d = 16 * s + 8 * half;
        q[s] = position_channels<T>((const T*)p.q + base + (size_t)d * p.N, p.N, d < p.D);
        go[s] = position_channels<T>((const T*)p.gout + base + (size_t)d * p.N, p.N, d < p.D);
        if (stages > 1) {
            const MatFrag<T> out = position_channels<T>((const T*)p.out + base + (size_t)d * p.N, p.N, d < p.D);
#pragma unroll
            for (int i = 0; i < 8; ++i) delta = fmaf(frag_value<T>(go[s], i), frag_value<T>(out, i), delta);
        }
    }
    delta = other_half_sum(delta);
    const float lse = p.lse[pos], c2 = p.scale * LOG2E;
    const float ref = lse == -__builtin_huge_valf() ? __builtin_huge_valf() : lse * LOG2E;      // (no token: all weights 0)

    f32x16 acc[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) mat_zero(acc[i]);
    // weights and dp of 32 tokens
    auto weights = [&](const char* kt, const char* vt, uint32_t word, float* e, f32x16& dp) {
        const uint32_t w = word >> (4 * half);
        f32x16 s;
        mat_zero(s);
        mat_zero(dp);
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            mat_mul<T>(s, token_rows<T, DT>(kt, lane & 31, i, half), q[i]);
            mat_mul<T>(dp, token_rows<T, DT>(vt, lane & 31, i, half), go[i]);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) e[r] = (w >> (8 * (r >> 2) + (r & 3))) & 1 ? __builtin_amdgcn_exp2f(fmaf(s[r], c2, -ref)) : 0.f;
    };

    TokenStage<T, DT, TB> next;
    next.fetch(p, b, head, 0, tid);
    for (int st = 0; st < stages; ++st) {
        const int buf = S::BUFFERS == 2 ? st & 1 : 0;
        char* const kt = lds + buf * S::STAGE;
        char* const vt = kt + S::K_BYTES;
        char* const k2 = vt + S::K_BYTES;
        if (S::BUFFERS == 1 && st) lds_barrier();
        next.put(kt, along_pitch<T, DT>(), vt, along_pitch<T, DT>(), k2, across_pitch<T, DT>(), tid);
        const uint64_t in = next.bits(0);
        if (st + 1 < stages) next.fetch(p, b, head, (st + 1) * TB, tid);
        lds_barrier();
        if (stages == 1) {
            float sum = 0.f;
            for (int i = 0; i < TB / 32; ++i) {
                const uint32_t word = (uint32_t)(in >> (32 * i));
                if (!word) continue;
                float e[16];
                f32x16 dp;
                weights(kt + 32 * i * along_pitch<T, DT>(), vt + 32 * i * along_pitch<T, DT>(), word, e, dp);
#pragma unroll
                for (int r = 0; r < 16; ++r) sum = fmaf(e[r], dp[r], sum);
            }
            delta = other_half_sum(sum);
        }
        for (int i = 0; i < TB / 32; ++i) {
            const uint32_t word = (uint32_t)(in >> (32 * i));
            if (!word) continue;
            float e[16];
            f32x16 dp;
            weights(kt + 32 * i * along_pitch<T, DT>(), vt + 32 * i * along_pitch<T, DT>(), word, e, dp);
#pragma unroll
            for (int r = 0; r < 16; ++r) e[r] *= dp[r] - delta;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const MatFrag<T> ds = mat_from_acc<T>(e + 8 * j);
#pragma unroll
                for (int a = 0; a < DT; ++a) mat_mul<T>(acc[a], token_columns<T, DT>(k2 + 32 * i * across_pitch<T, DT>(), a, j, lane), ds);
            }
        }
    }
    if (col >= columns) return;
    if (half == 0) p.delta[pos] = delta;
    if (p.gq)
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int d = i * 32 + acc_row(r, half);
                if (d < p.D) stf((T*)p.gq + base + (size_t)d * p.N, acc[i][r] * p.scale);
            }
}

// gk and gv.  A lane is a token: WT waves of a workgroup hold 32 tokens each, 4 / WT waves the same tokens on other positions.  A stage is
// PX positions of a head: q and gout as they are stored, [channel][position]; the scores as [position][token], so that the weights are
// the operand of the products over the positions.
template <typename T, int DT, int WT> struct AttendTokenShape {
    static constexpr int WP = 4 / WT, PX = WP == 4 ? 128 : 64, PITCH = PX * (int)sizeof(T) + 16;
    static constexpr int TILE = DT * 32 * PITCH, STAGE = 2 * TILE + 2 * PX * 4;
    static constexpr int BUFFERS = 2 * STAGE <= 160 * 1024 ? 2 : 1;
    static constexpr int LDS = BUFFERS * STAGE;
};

// operand A from [channel][position] in LDS: the positions as rows (from p0), channels contracted (step s)
template <typename T, int PITCH> __device__ __forceinline__ MatFrag<T> map_turned(const char* tile, int p0, int s, int lane) {
    const int half = lane >> 5;
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f.v[i] = *(const float*)(tile + (16 * s + 8 * half + i) * PITCH + (p0 + (lane & 31)) * 4);
    } else {
        const int j = lane & 15, col = p0 + (lane & 16) + (j & 3) * 4;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x2 v = lds_turned(tile + (16 * s + 8 * half + 4 * i + (j >> 2)) * PITCH + col * 2);
            f.w[2 * i] = v.x; f.w[2 * i + 1] = v.y;
        }
    }
    return f;
}
// ... and the channels as rows (32 from dt * 32), positions contracted in the order of an accumulator's rows
template <typename T, int PITCH> __device__ __forceinline__ MatFrag<T> map_rows(const char* tile, int dt, int p0, int j, int lane) {
    const int half = lane >> 5;
    const char* row = tile + (dt * 32 + (lane & 31)) * PITCH + (p0 + 16 * j + 4 * half) * (int)sizeof(T);
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
        const u32x4 a = *(const u32x4*)row, b = *(const u32x4*)(row + 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) { f.v[i] = __uint_as_float(a[i]); f.v[4 + i] = __uint_as_float(b[i]); }
    } else {
        const u32x2 a = *(const u32x2*)row, b = *(const u32x2*)(row + 16);
        f.w = u32x4{a.x, a.y, b.x, b.y};
    }
    return f;
}

template <typename T, int DT, int WT>
__global__ void __launch_bounds__(256) attend_grad_tokens_kernel(const AttendParams p) {
    using S = AttendTokenShape<T, DT, WT>;
    constexpr int KS = DT * 2, PX = S::PX, PITCH = S::PITCH, E = 16 / (int)sizeof(T), PIECES = PX / E, COUNT = DT * 32 * PIECES / 256;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wt = wave % WT, wp = wave / WT;
    const int ttiles = (p.L + 32 * WT - 1) / (32 * WT);
    unsigned item = xcd_contiguous_item(blockIdx.x, gridDim.x);
    const int tt = item % ttiles;
    item /= ttiles;
    const int split = item % p.splits, group = item / p.splits, head = group % p.kv, b = group / p.kv;

    // the lane's token
    const int token = tt * 32 * WT + wt * 32 + (lane & 31);
    const bool in = token < p.L && (!p.mask || p.mask[(size_t)b * p.L + token]);
    const size_t row = (((size_t)b * p.L + min(token, p.L - 1)) * p.kv + head) * p.D;
    MatFrag<T> k[KS], v[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int d = 16 * s + 8 * half;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) { k[s].v[i] = in && d < p.D ? ((const float*)p.k)[row + d + i] : 0.f; v[s].v[i] = in && d < p.D ? ((const float*)p.v)[row + d + i] : 0.f; }
        } else {
            k[s].w = v[s].w = u32x4{0, 0, 0, 0};
            if (in && d < p.D) { k[s].w = *(const u32x4*)((const T*)p.k + row + d); v[s].w = *(const u32x4*)((const T*)p.v + row + d); }
        }
    }
    f32x16 ak[DT], av[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) { mat_zero(ak[i]); mat_zero(av[i]); }

    const int per_head = (p.N + PX - 1) / PX;
    const long all = (long)per_head * p.per;
    const int first = (int)(all * split / p.splits), last = (int)(all * (split + 1) / p.splits);
    u32x4 rq[COUNT], rg[COUNT];
    float rl = 0.f;                                                  // threads 0 .. PX - 1: lse, PX .. 2 PX - 1: delta
    auto fetch = [&](int st) {
        const int g = st / per_head, n0 = (st - g * per_head) * PX;
        const size_t plane = (size_t)b * p.heads + head * p.per + g;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = tid + i * 256, d = c / PIECES, n = n0 + c % PIECES * E;
            rq[i] = rg[i] = u32x4{0, 0, 0, 0};
            if (d < p.D) {
                const T* at = (const T*)p.q + (plane * p.D + d) * p.N;
                const T* ag = (const T*)p.gout + (plane * p.D + d) * p.N;
                if (n + E <= p.N) { rq[i] = rg_load(at + n); rg[i] = rg_load(ag + n); }
                else { rq[i] = row_chunk(at, n, p.N); rg[i] = row_chunk(ag, n, p.N); }
            }
        }
        if (tid < 2 * PX) {
            const int n = n0 + tid % PX;
            if (n < p.N) {
                rl = tid < PX ? p.lse[plane * p.N + n] * LOG2E : p.delta[plane * p.N + n];
                if (tid < PX && rl == -__builtin_huge_valf()) rl = __builtin_huge_valf();        // (no token: all weights 0)
            } else rl = tid < PX ? __builtin_huge_valf() : 0.f;
        }
    };
    const float c2 = p.scale * LOG2E;
    if (first < last) fetch(first);
    for (int st = first; st < last; ++st) {
        char* const tq = lds + (S::BUFFERS == 2 ? (st - first) & 1 : 0) * S::STAGE;
        char* const tg = tq + S::TILE;
        float* const tl = (float*)(tg + S::TILE);
        if (S::BUFFERS == 1 && st > first) lds_barrier();
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = tid + i * 256, d = c / PIECES, o = c % PIECES * 16;
            *(u32x4*)(tq + d * PITCH + o) = rq[i];
            *(u32x4*)(tg + d * PITCH + o) = rg[i];
        }
        if (tid < 2 * PX) tl[tid] = rl;
        if (st + 1 < last) fetch(st + 1);
        lds_barrier();
        for (int p0 = wp * 32; p0 < PX; p0 += 32 * S::WP) {
            f32x16 s, dp;
            mat_zero(s);
            mat_zero(dp);
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                mat_mul<T>(s, map_turned<T, PITCH>(tq, p0, i, lane), k[i]);
                mat_mul<T>(dp, map_turned<T, PITCH>(tg, p0, i, lane), v[i]);
            }
            float e[16], ds[16];
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const u32x4 l4 = *(const u32x4*)(tl + p0 + 8 * r4 + 4 * half), d4 = *(const u32x4*)(tl + PX + p0 + 8 * r4 + 4 * half);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 4 * r4 + i;
                    e[r] = in ? __builtin_amdgcn_exp2f(fmaf(s[r], c2, -__uint_as_float(l4[i]))) : 0.f;
                    ds[r] = e[r] * (dp[r] - __uint_as_float(d4[i]));
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const MatFrag<T> fe = mat_from_acc<T>(e + 8 * j), fd = mat_from_acc<T>(ds + 8 * j);
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    mat_mul<T>(av[i], map_rows<T, PITCH>(tg, i, p0, j, lane), fe);
                    mat_mul<T>(ak[i], map_rows<T, PITCH>(tq, i, p0, j, lane), fd);
                }
            }
        }
    }
    if (token >= p.L) return;
    const size_t all_values = (size_t)p.B * p.L * p.kv * p.D;
    const bool direct = p.splits * S::WP == 1;
    float* const pk = direct ? nullptr : p.parts + (size_t)(split * S::WP + wp) * all_values;
    float* const pv = direct ? nullptr : pk + (size_t)p.splits * S::WP * all_values;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            const int d = i * 32 + acc_row(4 * r4, half);
            if (d >= p.D) continue;                                  // (D is a multiple of 8: the four rows are there or not)
            float gk[4], gv[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) { gk[e] = ak[i][4 * r4 + e] * p.scale; gv[e] = av[i][4 * r4 + e]; }
            if (direct) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (p.gk) stf((T*)p.gk + row + d + e, gk[e]);
                    if (p.gv) stf((T*)p.gv + row + d + e, gv[e]);
                }
            } else {
                *(u32x4*)(pk + row + d) = u32x4{__float_as_uint(gk[0]), __float_as_uint(gk[1]), __float_as_uint(gk[2]), __float_as_uint(gk[3])};
                *(u32x4*)(pv + row + d) = u32x4{__float_as_uint(gv[0]), __float_as_uint(gv[1]), __float_as_uint(gv[2]), __float_as_uint(gv[3])};
            }
        }
}

// ---- launches -----------------------------------------------------------------------------------------------------------------------
template <typename K> hipError_t attend_launch(K kernel, size_t items, int lds, const AttendParams& p, hipStream_t s) {
    hipError_t e = allow_dynamic_lds((const void*)kernel, lds);
    if (e != hipSuccess) return e;
    if (items * 256 >= ((size_t)1 << 32)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kernel, dim3((unsigned)items), dim3(256), lds, s, p);
    return hipGetLastError();
}
template <typename T, int DT, int PT, bool BY_TOKEN> hipError_t launch_attend_as(const AttendParams& p, hipStream_t s) {
    using S = AttendShape<T, DT, PT, BY_TOKEN>;
    const size_t tiles = ((size_t)p.per * p.N + S::COLUMNS - 1) / S::COLUMNS;
    hipError_t e = attend_launch(attend_kernel<T, DT, PT, BY_TOKEN>, (size_t)p.B * p.kv * tiles * p.splits, S::LDS, p, s);
    if (e != hipSuccess || p.splits == 1) return e;
    const size_t blocks = ((size_t)p.B * p.heads * p.D * p.N + 255) / 256;
    if (blocks * 256 >= ((size_t)1 << 32)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(attend_join_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, s, p);
    return hipGetLastError();
}
template <typename T, int DT> hipError_t launch_attend_head(const AttendParams& p, const AttendPlan& plan, hipStream_t s) {
    if (plan.by_token) return launch_attend_as<T, DT, 1, true>(p, s);
    if constexpr (sizeof(T) == 2 || DT <= 2) { if (plan.wide) return launch_attend_as<T, DT, 2, false>(p, s); }
    return launch_attend_as<T, DT, 1, false>(p, s);
}
template <typename T> hipError_t launch_attend_type(const AttendParams& p, const AttendPlan& plan, hipStream_t s) {
    switch ((p.D + 31) / 32) {
        case 1: return launch_attend_head<T, 1>(p, plan, s);
        case 2: return launch_attend_head<T, 2>(p, plan, s);
        case 3: return launch_attend_head<T, 3>(p, plan, s);
        default: return launch_attend_head<T, 4>(p, plan, s);
    }
}
template <typename T, int DT> hipError_t launch_attend_bwd_head(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s) {
    const size_t tiles = ((size_t)p.per * p.N + 127) / 128, groups = (size_t)p.B * p.kv;
    hipError_t e = attend_launch(attend_grad_q_kernel<T, DT>, groups * tiles, AttendGradShape<T, DT>::LDS, p, s);
    if (e != hipSuccess || (!p.gk && !p.gv)) return e;
    const size_t items = groups * p.splits * ((p.L + 32 * plan.token_waves - 1) / (32 * plan.token_waves));
    if constexpr (sizeof(T) == 2 || DT < 4) {                        // (fp32 heads of more than 96 channels: registers for four token waves alone)
        if (plan.token_waves == 2) return attend_launch(attend_grad_tokens_kernel<T, DT, 2>, items, AttendTokenShape<T, DT, 2>::LDS, p, s);
        if (plan.token_waves == 1) return attend_launch(attend_grad_tokens_kernel<T, DT, 1>, items, AttendTokenShape<T, DT, 1>::LDS, p, s);
    }
    return attend_launch(attend_grad_tokens_kernel<T, DT, 4>, items, AttendTokenShape<T, DT, 4>::LDS, p, s);
}
template <typename T> hipError_t launch_attend_bwd_type(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s) {
    switch ((p.D + 31) / 32) {
        case 1: return launch_attend_bwd_head<T, 1>(p, plan, s);
        case 2: return launch_attend_bwd_head<T, 2>(p, plan, s);
        case 3: return launch_attend_bwd_head<T, 3>(p, plan, s);
        default: return launch_attend_bwd_head<T, 4>(p, plan, s);
    }
}
// instantiated in a translation unit per storage type
hipError_t launch_attend_f32(const AttendParams& p, const AttendPlan& plan, hipStream_t s);
hipError_t launch_attend_bf16(const AttendParams& p, const AttendPlan& plan, hipStream_t s);
hipError_t launch_attend_f16(const AttendParams& p, const AttendPlan& plan, hipStream_t s);
hipError_t launch_attend_bwd_f32(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s);
hipError_t launch_attend_bwd_bf16(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s);
hipError_t launch_attend_bwd_f16(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s);

}  // namespace gspn
