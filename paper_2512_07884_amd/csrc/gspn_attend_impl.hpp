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

// 16 bits.  The weights are rounded for their products; of many tokens those errors come out as that of one more rounding of the result.  Of few tokens, with
// weights about a half, they are larger (1.6 times a rounding's error in all), and there is time, as the maps bound such calls: up to this many
// tokens the products take what the rounding left as well.  gq, which also has the rounding of out in it (delta), always takes it of ds: its error
// over 300 tokens was 1.5 times a rounding's, for 5 us of 124 of that step.
constexpr int SPLIT_MOST = 64;
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

// KS: steps of 16 channels that a head has (the last one filled with zeros), DT: tiles of 32.
// Rows of tokens in LDS: read along the row (16 bytes per lane; an odd number of 16-byte pieces: 16 rows on all banks) ...
template <typename T, int KS> constexpr int along_pitch() { return KS * 16 * (int)sizeof(T) + 16; }
// ... and across the rows, turned (four rows of 64 bytes on all banks; fp32: rows four apart on both halves of the banks)
template <typename T, int KS> constexpr int across_pitch() {
    constexpr int DT = (KS + 1) / 2;
    return sizeof(T) == 4 ? DT * 128 + 32 : (DT % 2 ? DT * 64 : DT * 64 + 64);
}

// operand A from rows of tokens: the channels contracted (step s), row r
template <typename T, int KS> __device__ __forceinline__ MatFrag<T> token_rows(const char* tile, int r, int s, int half) {
    return mat_contiguous<T>(tile + r * along_pitch<T, KS>() + (16 * s + 8 * half) * (int)sizeof(T));
}
// ... and the tokens contracted, in the order of an accumulator's rows (16 * s ...), channels dt * 32 ...
template <typename T, int PITCH> __device__ __forceinline__ MatFrag<T> token_columns(const char* tile, int dt, int s, int lane) {
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

// Eight channels of positions as operands: rows N apart from `row` (the same for the whole wave) on, the lane's own offset of `at` values.  `have`: the
// channels exist, all eight or none.
template <typename T> __device__ __forceinline__ MatFrag<T> position_channels(const T* row, size_t N, uint32_t at, bool have) {
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f.v[i] = have ? (row + i * N)[at] : 0.f;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t lo = 0, hi = 0;
            if (have) { lo = ((const uint16_t*)(row + (2 * i) * N))[at]; hi = ((const uint16_t*)(row + (2 * i + 1) * N))[at]; }
            f.w[i] = lo | hi << 16;
        }
    }
    return f;
}

// 32 neighbouring positions of a head's plane [D][N], which a wave brings in requests of 16 bytes along the rows, turns in LDS of its own (`buf`, BYTES of it) and
// gets back as operands with a lane per position; and results on the same way back.  (Two-byte requests per lane and channel: 77 tokens on
// two 128x128 latents 48 us, the gradient of q over 300 tokens on two 64x64 maps 70.)  fp32: rows of 144 bytes, so that the two halves of
// a wave, eight rows apart, meet other banks.
template <typename T, int KS> struct MapTile {
    static constexpr int E = 16 / (int)sizeof(T), PIECES = 32 / E, ROW = sizeof(T) == 4 ? 144 : 64, BYTES = KS * 16 * ROW;
    static constexpr int COUNT = KS * 16 * PIECES / 64;
    u32x4 r[COUNT];

    // the first position of tile i: a last tile that is not whole begins earlier (the same bits twice)
    static __device__ __forceinline__ int begin(int i, int N) { return N >= 32 ? min(i * 32, N - 32) : 0; }
    __device__ __forceinline__ void fetch(const T* plane, int D, int N, int n0, int lane) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = lane + 64 * i, d = c / PIECES, n = n0 + c % PIECES * E;
            const T* row = plane + (size_t)d * N;
            r[i] = u32x4{0, 0, 0, 0};
            if (d < D) {
                if (N >= 32) r[i] = rg_load(row + n);
                else r[i] = row_chunk(row, n, N);
            }
        }
    }
    __device__ __forceinline__ void put(char* buf, int lane) const {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = lane + 64 * i;
            *(u32x4*)(buf + c / PIECES * ROW + c % PIECES * 16) = r[i];
        }
    }
    static __device__ __forceinline__ void operands(const char* buf, MatFrag<T> (&f)[KS], int lane) {
        const int half = lane >> 5;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int i = 0; i < 8; ++i) f[s].v[i] = *(const float*)(buf + (16 * s + 8 * half + i) * ROW + (lane & 31) * 4);
            } else {
                const int j = lane & 15;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const u32x2 v = lds_turned(buf + (16 * s + 8 * half + 4 * i + (j >> 2)) * ROW + (lane & 16) * 2 + (j & 3) * 8);
                    f[s].w[2 * i] = v.x; f[s].w[2 * i + 1] = v.y;
                }
            }
        }
    }
    template <int DT> static __device__ __forceinline__ void store(char* buf, const f32x16 (&acc)[DT], float factor, T* plane, int D, int N, int n0, int lane) {
        const int half = lane >> 5;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int d = i * 32 + acc_row(k, half);
                if (i * 32 + 24 < KS * 16 || d < KS * 16) stf((T*)(buf + d * ROW) + (lane & 31), acc[i][k] * factor);
            }
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = lane + 64 * i, d = c / PIECES, n = n0 + c % PIECES * E;
            const u32x4 v = *(const u32x4*)(buf + d * ROW + c % PIECES * 16);
            T* row = plane + (size_t)d * N;
            if (d < D) {
                if (N >= 32) rg_store(row + n, v);
                else
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (n + e < N) rg_store_bits(row + n + e, rg_bits<T>(v, e));
            }
        }
    }
};
template <typename T> __device__ __forceinline__ float frag_value(const MatFrag<T>& f, int i) {
    if constexpr (sizeof(T) == 4) return f.v[i];
    else return rg_elem<T>(f.w, i);
}

// A stage of TB tokens on its way to LDS through the registers of 256 threads: keys and values of one head, and which of the tokens take part
template <typename T, int KS, int TB> struct TokenStage {
    static constexpr int E = 16 / (int)sizeof(T), PIECES = KS * 16 / E;            // 16-byte pieces of a token's row
    static constexpr int ALL = TB * PIECES, COUNT = (ALL + 255) / 256;             // per thread
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
            if (d < p.D && (ALL % 256 == 0 || c < ALL)) {
                const size_t at = (((size_t)b * p.L + t) * p.kv + head) * p.D + d;
                k[i] = *(const u32x4*)((const T*)p.k + at);
                v[i] = *(const u32x4*)((const T*)p.v + at);
            }
        }
    }
    // bits of the tokens that take part, 64 of them
    __device__ __forceinline__ uint64_t bits(int i) const { return __ballot(here[i] != 0); }
    // rows of k and v into LDS, zeros for tokens that take no part
    __device__ __forceinline__ void put(char* k_at, int k_pitch, char* v_at, int v_pitch, int tid) const {
        uint64_t w[(TB + 63) / 64];
#pragma unroll
        for (int i = 0; i < (TB + 63) / 64; ++i) w[i] = bits(i);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = tid + i * 256, r = c / PIECES, o = c % PIECES * 16;
            if (ALL % 256 && c >= ALL) break;
            const bool in = (w[TB > 64 ? r >> 6 : 0] >> (r & 63)) & 1;
            const u32x4 zero = {0, 0, 0, 0};
            *(u32x4*)(k_at + r * k_pitch + o) = in ? k[i] : zero;
            *(u32x4*)(v_at + r * v_pitch + o) = in ? v[i] : zero;
        }
    }
};

// All tokens of a head at once, `rows` of them (a multiple of 32; those past the end and those that take no part are zeros), and the words of 32 bits that say
// which take part
template <typename T, int KS, int THREADS>
__device__ __forceinline__ void all_tokens(const AttendParams& p, int b, int head, int rows, char* k_at, int k_pitch, char* v_at, int v_pitch, uint32_t* words, int tid) {
    constexpr int E = 16 / (int)sizeof(T), PIECES = KS * 16 / E;
    for (int i = tid; i < ((rows + 63) & ~63); i += THREADS) {
        const uint64_t w = __ballot(i < p.L && (!p.mask || p.mask[(size_t)b * p.L + i]));
        if ((tid & 63) == 0) { words[i >> 5] = (uint32_t)w; words[(i >> 5) + 1] = (uint32_t)(w >> 32); }
    }
#pragma unroll 4
    for (int c = tid; c < rows * PIECES; c += THREADS) {
        const int t = c / PIECES, d = c % PIECES * E;
        u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
        if (t < p.L && d < p.D && (!p.mask || p.mask[(size_t)b * p.L + t])) {
            const size_t at = (((size_t)b * p.L + t) * p.kv + head) * p.D + d;
            k = *(const u32x4*)((const T*)p.k + at);
            v = *(const u32x4*)((const T*)p.v + at);
        }
        *(u32x4*)(k_at + t * k_pitch + d * (int)sizeof(T)) = k;
        *(u32x4*)(v_at + t * v_pitch + d * (int)sizeof(T)) = v;
    }
}
// accumulators that start at 0 for tokens that take part and at -inf for the others (word: bit r = token r of the 32)
__device__ __forceinline__ void start_scores(f32x16& s, uint32_t word, int half) {
    if (word == 0xffffffffu) { mat_zero(s); return; }
    const uint32_t w = word >> (4 * half);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = (w >> (8 * (r >> 2) + (r & 3))) & 1 ? 0.f : -__builtin_huge_valf();
}

// The running state of the wave's 32 positions: output, maximum (in powers of two) and the lane's half of the sum
template <int DT> struct AttendState {
    f32x16 o[DT];
    float top, sum;
    __device__ __forceinline__ void start() {
        top = -__builtin_huge_valf(); sum = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) mat_zero(o[i]);
    }
};
// 32 tokens in LDS
template <typename T, int KS, bool BOTH>
__device__ __forceinline__ void attend_tokens(const char* kt, const char* vt, uint32_t word, const MatFrag<T> (&q)[KS], AttendState<(KS + 1) / 2>& a, float c2, int lane) {
    constexpr int DT = (KS + 1) / 2;
    const int half = lane >> 5;
    f32x16 s;
    start_scores(s, word, half);
#pragma unroll
    for (int i = 0; i < KS; ++i) mat_mul<T>(s, token_rows<T, KS>(kt, lane & 31, i, half), q[i]);
    float m = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) m = fmaxf(m, s[r]);
    m = other_half_max(m) * c2;
    // The maximum is a reference that keeps the powers in range: it is moved only where it has grown by more than 2^8
    if (__ballot(m > a.top + 8.f)) {
        const float next = fmaxf(a.top, m), shrink = next == -__builtin_huge_valf() ? 1.f : __builtin_amdgcn_exp2f(a.top - next);
        a.top = next;
        a.sum *= shrink;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) a.o[i][r] *= shrink;
    }
    const float ref = a.top == -__builtin_huge_valf() ? 0.f : a.top;
    float e[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) { e[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c2, -ref)); a.sum += e[r]; }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        MatFrag<T> w, rest;
        if constexpr (BOTH) {
            mat_split<T>(e + 8 * j, w, rest);
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const MatFrag<T> v = token_columns<T, across_pitch<T, KS>()>(vt, i, j, lane);
                mat_mul<T>(a.o[i], v, w);
                mat_mul<T>(a.o[i], v, rest);
            }
        } else {
            w = mat_from_acc<T>(e + 8 * j);
#pragma unroll
            for (int i = 0; i < DT; ++i) mat_mul<T>(a.o[i], token_columns<T, across_pitch<T, KS>()>(vt, i, j, lane), w);
        }
    }
}
__device__ __forceinline__ float attend_share(float l) { return l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l); }          // (no token: 0; NaN stays NaN)

// Many positions.  A wave holds 32 neighbouring positions of a head (lane and lane + 32: the same one, other channels).
// RESIDENT: the head's tokens stay in LDS, all of them, and each wave walks over tiles of positions without meeting the others again, the next tile on its
// way while it works; 77 tokens of 64 channels are 32 KB.  Else stages of 64 tokens, two of them in LDS, the one after them on its way in
// registers, and a tile per wave.
template <typename T, int KS> struct AttendShape {
    static constexpr int TB = 64;
    static constexpr int K_ROW = along_pitch<T, KS>(), V_ROW = across_pitch<T, KS>(), STAGE = TB * (K_ROW + V_ROW), MAP = MapTile<T, KS>::BYTES;
    static constexpr int BUFFERS = 2 * STAGE + 4 * MAP <= 160 * 1024 ? 2 : 1;
    static constexpr int LDS = BUFFERS * STAGE + 4 * MAP;            // (RESIDENT: resident_bytes)
};
constexpr int RESIDENT_MOST = 160 * 1024;
// Waves per SIMD that the kernels' registers leave room for, by which a call's workgroups are counted too.  (From two on a wave has 256 registers
// of one file, none in the accumulation file that takes a move per value read.)
constexpr int attend_waves(bool f32, int ks) { return f32 ? (ks <= 2 ? 4 : ks <= 3 ? 3 : 2) : (ks <= 4 ? 4 : ks <= 6 ? 3 : 2); }
constexpr int attend_grad_waves(bool f32, int ks) { return f32 ? (ks <= 2 ? 3 : ks <= 5 ? 2 : 1) : (ks <= 2 ? 4 : 2); }
// ... and workgroups of the kernel over the tokens on a CU (wt: waves along the tokens)
constexpr int attend_token_groups(bool f32, int ks, int wt) { return (f32 ? ks <= 3 : ks < 5 || (ks == 5 && wt == 4)) ? 2 : 1; }
// ... with the next tile of the maps in registers beside them; wide heads bring a tile when it is wanted, one map after the other
constexpr bool attend_ahead(bool f32, int ks) { return !f32 || ks <= 6; }
constexpr bool attend_grad_ahead(bool f32, int ks) { return f32 ? ks <= 3 : ks <= 6; }
inline int resident_rows(int L) { return (L + 31) & ~31; }
// rows of the tokens, the words, a tile of the map for each wave
inline size_t resident_bytes(int L, int row, int waves, int map) {
    return (size_t)resident_rows(L) * row + (((size_t)(resident_rows(L) / 32 + 2) * 4 + 15) & ~(size_t)15) + (size_t)waves * map;
}
__device__ __forceinline__ char* resident_map(char* lds, int rows, int row, int wave, int map) { return lds + rows * row + (((rows / 32 + 2) * 4 + 15) & ~15) + wave * map; }

template <typename T, int KS, int WAVES, bool RESIDENT, bool BOTH = false>
__global__ void __launch_bounds__(64 * WAVES, BOTH ? (KS <= 4 ? 3 : 2) : RESIDENT ? attend_waves(sizeof(T) == 4, KS) : (sizeof(T) == 2 || KS <= 5 ? 2 : 1)) attend_kernel(const AttendParams p) {
    using S = AttendShape<T, KS>;
    using Map = MapTile<T, KS>;
    constexpr int DT = (KS + 1) / 2;
    static_assert(RESIDENT || WAVES == 4, "stages go through 256 threads");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int per_head = (p.N + 31) / 32, tiles = per_head * p.per;
    const unsigned item = xcd_contiguous_item(blockIdx.x, gridDim.x);
    const int group = item / p.workers, worker = item - group * p.workers, head = group % p.kv, b = group / p.kv;
    const float c2 = p.scale * LOG2E;

    auto place = [&](int tile, size_t& plane, int& n0) {
        const int g = tile / per_head;
        plane = (size_t)b * p.heads + head * p.per + g;
        n0 = Map::begin(tile - g * per_head, p.N);
    };
    auto finish = [&](const AttendState<DT>& a, size_t plane, int n0, char* buf) {
        const float l = other_half_sum(a.sum);
        if (p.lse && half == 0 && n0 + lane < p.N) p.lse[plane * p.N + n0 + lane] = (a.top + __builtin_amdgcn_logf(l)) * LN2;
        Map::store(buf, a.o, attend_share(l), (T*)p.out + plane * p.D * p.N, p.D, p.N, n0, lane);
    };
    Map map;
    size_t plane;
    int n0;
    if constexpr (RESIDENT) {
        const int rows = (p.L + 31) & ~31;
        char* const vt = lds + rows * S::K_ROW;
        uint32_t* const words = (uint32_t*)(vt + rows * S::V_ROW);
        char* const buf = resident_map(lds, rows, S::K_ROW + S::V_ROW, wave, S::MAP);
        constexpr bool AHEAD = attend_ahead(sizeof(T) == 4, KS);
        int tile = worker * WAVES + wave;
        auto bring = [&] {
            place(tile, plane, n0);
            map.fetch((const T*)p.q + plane * p.D * p.N, p.D, p.N, n0, lane);
        };
        if (AHEAD && tile < tiles) bring();
        all_tokens<T, KS, 64 * WAVES>(p, b, head, rows, lds, S::K_ROW, vt, S::V_ROW, words, tid);
        __syncthreads();
        while (tile < tiles) {
            if (!AHEAD) bring();
            const size_t at = plane;
            const int n = n0;
            MatFrag<T> q[KS];
            map.put(buf, lane);
            Map::operands(buf, q, lane);
            tile += p.workers * WAVES;
            if (AHEAD && tile < tiles) bring();
            AttendState<DT> a;
            a.start();
            for (int i = 0; i < rows / 32; ++i) {
                const uint32_t word = __builtin_amdgcn_readfirstlane(words[i]);
                if (word) attend_tokens<T, KS, BOTH>(lds + i * 32 * S::K_ROW, vt + i * 32 * S::V_ROW, word, q, a, c2, lane);
            }
            finish(a, at, n, buf);
        }
    } else {
        char* const buf = lds + S::BUFFERS * S::STAGE + wave * S::MAP;
        const int stages = (p.L + S::TB - 1) / S::TB;
        place(min(worker * WAVES + wave, tiles - 1), plane, n0);     // (waves past the end: the last tile again, the same bits)
        map.fetch((const T*)p.q + plane * p.D * p.N, p.D, p.N, n0, lane);
        TokenStage<T, KS, S::TB> next;
        next.fetch(p, b, head, 0, tid);
        MatFrag<T> q[KS];
        map.put(buf, lane);
        Map::operands(buf, q, lane);
        AttendState<DT> a;
        a.start();
        for (int st = 0; st < stages; ++st) {
            char* const kt = lds + (S::BUFFERS == 2 ? st & 1 : 0) * S::STAGE;
            char* const vt = kt + S::TB * S::K_ROW;
            if (S::BUFFERS == 1 && st) lds_barrier();                // (the stage before has been read)
            next.put(kt, S::K_ROW, vt, S::V_ROW, tid);
            const uint64_t in = next.bits(0);
            if (st + 1 < stages) next.fetch(p, b, head, (st + 1) * S::TB, tid);
            lds_barrier();
#pragma unroll
            for (int i = 0; i < S::TB / 32; ++i) {
                const uint32_t word = (uint32_t)(in >> (32 * i));
                if (word) attend_tokens<T, KS, BOTH>(kt + 32 * i * S::K_ROW, vt + 32 * i * S::V_ROW, word, q, a, c2, lane);
            }
        }
        finish(a, plane, n0, buf);
    }
}

// Few positions: the four waves of a workgroup hold the same 32 columns (positions of the heads that share tokens, one head after the other) and take 32 of
// the 128 tokens of a stage each; their states meet in LDS.  Still few workgroups and many tokens: each takes a stretch of the tokens, and
// attend_join_kernel joins the stretches.
template <typename T, int KS> struct AttendFewShape {
    static constexpr int TB = 128, DT = (KS + 1) / 2;
    static constexpr int K_ROW = along_pitch<T, KS>(), V_ROW = across_pitch<T, KS>(), STAGE = TB * (K_ROW + V_ROW);
    static constexpr int BUFFERS = 2 * STAGE <= 160 * 1024 ? 2 : 1;
    static constexpr int JOIN = 4 * (DT * 32 + 2) * 32 * 4;
    // (a stretch of one stage needs one buffer: more workgroups on a CU)
    static int lds(int L, int splits) {
        const int need = ((L + TB - 1) / TB <= splits ? 1 : BUFFERS) * STAGE;
        return need > JOIN ? need : JOIN;
    }
    static constexpr bool AHEAD = sizeof(T) == 2 || KS <= 4;         // (fp32: no registers for a stage on its way beside wide heads)
};
template <typename T, int KS, bool BOTH>
__global__ void __launch_bounds__(256, (sizeof(T) == 2 ? KS <= 4 + !BOTH : KS <= 4) ? 2 : 1) attend_few_kernel(const AttendParams p) {
    using S = AttendFewShape<T, KS>;
    constexpr int TB = S::TB, DT = S::DT;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int columns = p.per * p.N, tiles = (columns + 31) / 32;
    unsigned item = xcd_contiguous_item(blockIdx.x, gridDim.x);
    const int split = item % p.splits;
    item /= p.splits;
    const int tile = item % tiles, group = item / tiles, head = group % p.kv, b = group / p.kv;
    const int stages = (p.L + TB - 1) / TB;
    const int first = (int)((long)stages * split / p.splits), last = (int)((long)stages * (split + 1) / p.splits);
    const size_t plane0 = (size_t)b * p.heads + head * p.per;        // the first of the heads that share the tokens
    auto offset = [&](int column) {                                  // of a column's first channel
        const int g = column / p.N;
        return (uint32_t)g * p.D * p.N + (column - g * p.N);
    };
    const float c2 = p.scale * LOG2E;

    MatFrag<T> q[KS];
    const uint32_t at = offset(min(tile * 32 + (lane & 31), columns - 1));
#pragma unroll
    for (int s = 0; s < KS; ++s)
        q[s] = position_channels<T>((const T*)p.q + plane0 * p.D * p.N + (size_t)(16 * s) * p.N, p.N, at + 8u * half * p.N, 16 * s + 8 * half < p.D);
    AttendState<DT> a;
    a.start();
    if (first < last) {
        TokenStage<T, KS, TB> next;
        if (S::AHEAD) next.fetch(p, b, head, first * TB, tid);
        for (int st = first; st < last; ++st) {
            if (!S::AHEAD) next.fetch(p, b, head, st * TB, tid);
            char* const kt = lds + (S::BUFFERS == 2 ? (st - first) & 1 : 0) * S::STAGE;
            char* const vt = kt + TB * S::K_ROW;
            if (S::BUFFERS == 1 && st > first) lds_barrier();       // (the stage before has been read)
            next.put(kt, S::K_ROW, vt, S::V_ROW, tid);
            const uint64_t in = wave >= 2 ? next.bits(1) : next.bits(0);
            if (S::AHEAD && st + 1 < last) next.fetch(p, b, head, (st + 1) * TB, tid);
            lds_barrier();
            const uint32_t word = (uint32_t)(in >> (wave & 1) * 32);
            if (word) attend_tokens<T, KS, BOTH>(kt + wave * 32 * S::K_ROW, vt + wave * 32 * S::V_ROW, word, q, a, c2, lane);
        }
    }
    a.sum = other_half_sum(a.sum);

    // the four waves' states meet in LDS: [wave][channel][column], then maximum and sum
    float* const join = (float*)lds;
    float* const tops = join + 4 * DT * 32 * 32;
    lds_barrier();
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) join[(wave * DT * 32 + i * 32 + acc_row(r, half)) * 32 + (lane & 31)] = a.o[i][r];
    if (half == 0) { tops[wave * 32 + lane] = a.top; tops[128 + wave * 32 + lane] = a.sum; }
    lds_barrier();
    const int n = tid & 31, column = tile * 32 + n;                 // a thread finishes every eighth channel of a column
    float m = tops[n], f[4], l = 0.f;
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, tops[w * 32 + n]);
    const float ref = m == -__builtin_huge_valf() ? 0.f : m;
#pragma unroll
    for (int w = 0; w < 4; ++w) { f[w] = __builtin_amdgcn_exp2f(tops[w * 32 + n] - ref); l += f[w] * tops[128 + w * 32 + n]; }
    if (column >= columns) return;
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
    const float share = attend_share(l);
    T* const out = (T*)p.out + plane0 * p.D * p.N + offset(column);
    for (int d = tid >> 5; d < p.D; d += 8) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) v += f[w] * join[(w * DT * 32 + d) * 32 + n];
        stf(out + (size_t)d * p.N, v * share);
    }
    if (p.lse && tid < 32) p.lse[plane0 * p.N + column] = (m + __builtin_amdgcn_logf(l)) * LN2;        // ([head][position] is the columns' own order)
}

// Joins the stretches of the tokens: 32 columns of a group and eight channels per workgroup.  The stretches' factors are worked out once per workgroup (eight threads
// per column) and shared; a thread then adds one channel of a column over them.
template <typename T> __global__ void __launch_bounds__(256) attend_join_kernel(const AttendParams p) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    float* const factor = (float*)lds;                               // [split][column]
    float* const strip = factor + p.splits * 32;                     // [8][column]
    const int columns = p.per * p.N, tiles = (columns + 31) / 32, slices = (p.D + 7) / 8;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const unsigned tile = blockIdx.x % tiles, slice = blockIdx.x / tiles % slices, group = blockIdx.x / tiles / slices;
    const int column = tile * 32 + x, c = min(column, columns - 1), d = slice * 8 + y;
    const size_t step = (size_t)p.B * p.kv * (p.D + 2) * columns;
    const float* const state = p.parts + (size_t)group * (p.D + 2) * columns + c;
    float m = -__builtin_huge_valf();
#pragma unroll 4
    for (int s = y; s < p.splits; s += 8) m = fmaxf(m, state[s * step + (size_t)p.D * columns]);
    strip[y * 32 + x] = m;
    __syncthreads();
    m = strip[x];
#pragma unroll
    for (int i = 1; i < 8; ++i) m = fmaxf(m, strip[i * 32 + x]);
    __syncthreads();
    const float ref = m == -__builtin_huge_valf() ? 0.f : m;
    float l = 0.f;
#pragma unroll 4
    for (int s = y; s < p.splits; s += 8) {
        const float f = __builtin_amdgcn_exp2f(state[s * step + (size_t)p.D * columns] - ref);
        factor[s * 32 + x] = f;
        l = fmaf(f, state[s * step + (size_t)(p.D + 1) * columns], l);
    }
    strip[y * 32 + x] = l;
    __syncthreads();
    l = strip[x];
#pragma unroll
    for (int i = 1; i < 8; ++i) l += strip[i * 32 + x];
    if (column >= columns || d >= p.D) return;
    float v = 0.f;
#pragma unroll 8
    for (int s = 0; s < p.splits; ++s) v = fmaf(factor[s * 32 + x], state[s * step + (size_t)d * columns], v);
    const int head = group % p.kv, b = group / p.kv, g = column / p.N;
    const size_t plane = (size_t)b * p.heads + head * p.per + g;
    stf((T*)p.out + (plane * p.D + d) * p.N + (column - g * p.N), v * attend_share(l));
    if (p.lse && d == 0) p.lse[plane * p.N + (column - g * p.N)] = (m + __builtin_amdgcn_logf(l)) * LN2;
}

// ---- backward -----------------------------------------------------------------------------------------------------------------------
//     p = exp(s - lse) ,  dp[t][n] = sum_d v[t][d] gout[d][n] ,  ds = p (dp - delta[n]) ,  delta[n] = sum_t p dp = sum_d gout out
//     gq[d][n] = scale sum_t ds k[t][d] ,   gk[t][d] = scale sum_n ds q[d][n] ,   gv[t][d] = sum_n p gout[d][n]
// Two launches: gq (and delta) with a lane per position as in the forward call, then gk and gv with a lane per token and the positions
// walked in stages.  p and ds are rounded to the storage type for the products, everything else is fp32.

// gq, and delta for the launch after it; positions and tokens as in attend_kernel.  Where up to 64 tokens take part delta is the sum over them, in a pass
// of its own; else the product of gout and out, which the rounding of out puts off by e: since the weights of a position add up to 1, the sum
// of its ds is then -e, and the second launch is given delta without it.
template <typename T, int KS> struct AttendGradShape {
    static constexpr int TB = 64, ROW = along_pitch<T, KS>(), STAGE = TB * 2 * ROW, MAP = MapTile<T, KS>::BYTES;
    static constexpr int BUFFERS = 2 * STAGE + 4 * MAP <= 160 * 1024 ? 2 : 1;
    static constexpr int LDS = BUFFERS * STAGE + 4 * MAP;            // (RESIDENT: resident_bytes)
};
// weights of 32 tokens, and the products of gout with their values
template <typename T, int KS>
__device__ __forceinline__ void attend_weights(const char* kt, const char* vt, uint32_t word, const MatFrag<T> (&q)[KS], const MatFrag<T> (&go)[KS],
                                               float ref, float c2, f32x16& e, f32x16& dp, int lane) {
    const int half = lane >> 5;
    start_scores(e, word, half);
    mat_zero(dp);
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        mat_mul<T>(e, token_rows<T, KS>(kt, lane & 31, i, half), q[i]);
        mat_mul<T>(dp, token_rows<T, KS>(vt, lane & 31, i, half), go[i]);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) e[r] = __builtin_amdgcn_exp2f(fmaf(e[r], c2, -ref));
}
template <typename T, int KS, int WAVES, bool RESIDENT>
__global__ void __launch_bounds__(64 * WAVES, RESIDENT ? attend_grad_waves(sizeof(T) == 4, KS) : (sizeof(T) == 2 ? KS < 7 : KS <= 3) ? 2 : 1) attend_grad_q_kernel(const AttendParams p) {
    using S = AttendGradShape<T, KS>;
    using Map = MapTile<T, KS>;
    constexpr int DT = (KS + 1) / 2;
    static_assert(RESIDENT || WAVES == 4, "stages go through 256 threads");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int per_head = (p.N + 31) / 32, tiles = per_head * p.per;
    const unsigned item = xcd_contiguous_item(blockIdx.x, gridDim.x);
    const int group = item / p.workers, worker = item - group * p.workers, head = group % p.kv, b = group / p.kv;
    const float c2 = p.scale * LOG2E;
    bool few = p.L <= 64;                                            // (of the tokens that take part: once they have been counted)

    constexpr bool AHEAD = attend_grad_ahead(sizeof(T) == 4, KS);
    Map maps[AHEAD ? 3 : 1];
    Map &mq = maps[0], &mg = maps[AHEAD ? 1 : 0], &mo = maps[AHEAD ? 2 : 0];
    float lse;
    size_t plane;
    int n0;
    auto bring = [&](Map& m, const void* from) { m.fetch((const T*)from + plane * p.D * p.N, p.D, p.N, n0, lane); };
    auto fetch = [&](int tile) {
        const int g = tile / per_head;
        plane = (size_t)b * p.heads + head * p.per + g;
        n0 = Map::begin(tile - g * per_head, p.N);
        bring(mq, p.q);
        if (AHEAD) {
            bring(mg, p.gout);
            if (!few) bring(mo, p.out);
        }
        lse = p.lse[plane * p.N + min(n0 + (lane & 31), p.N - 1)];
    };
    MatFrag<T> q[KS], go[KS];
    float delta, off, ref;                                           // off: the sum of ds
    f32x16 acc[DT];
    auto start = [&](char* buf) {
        mq.put(buf, lane);
        Map::operands(buf, q, lane);
        if (!AHEAD) bring(mg, p.gout);
        mg.put(buf, lane);
        Map::operands(buf, go, lane);
        delta = off = 0.f;
        if (!few) {
            MatFrag<T> out[KS];
            if (!AHEAD) bring(mo, p.out);
            mo.put(buf, lane);
            Map::operands(buf, out, lane);
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int i = 0; i < 8; ++i) delta = fmaf(frag_value<T>(go[s], i), frag_value<T>(out[s], i), delta);
            delta = other_half_sum(delta);
        }
        ref = lse == -__builtin_huge_valf() ? __builtin_huge_valf() : lse * LOG2E;              // (no token: all weights 0)
#pragma unroll
        for (int i = 0; i < DT; ++i) mat_zero(acc[i]);
    };
    // 32 tokens: towards delta, or their share of gq
    auto sum_delta = [&](const char* kt, const char* vt, uint32_t word) {
        f32x16 e, dp;
        attend_weights<T, KS>(kt, vt, word, q, go, ref, c2, e, dp, lane);
#pragma unroll
        for (int r = 0; r < 16; ++r) delta = fmaf(e[r], dp[r], delta);
    };
    auto step = [&](const char* kt, const char* vt, uint32_t word) {
        f32x16 e, dp;
        attend_weights<T, KS>(kt, vt, word, q, go, ref, c2, e, dp, lane);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float x[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) { x[r] = e[8 * j + r] * (dp[8 * j + r] - delta); off += x[r]; }
            MatFrag<T> ds, rest;
            mat_split<T>(x, ds, rest);
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const MatFrag<T> k = token_columns<T, S::ROW>(kt, i, j, lane);
                mat_mul<T>(acc[i], k, ds);
                if constexpr (sizeof(T) == 2) mat_mul<T>(acc[i], k, rest);
            }
        }
    };
    auto finish = [&](size_t at, int n, char* buf) {
        const float exact = delta + other_half_sum(off);
        if (half == 0 && n + lane < p.N) p.delta[at * p.N + n + lane] = exact;
        if (p.gq) Map::store(buf, acc, p.scale, (T*)p.gq + at * p.D * p.N, p.D, p.N, n, lane);
    };

    if constexpr (RESIDENT) {
        const int rows = (p.L + 31) & ~31;
        char* const vt = lds + rows * S::ROW;
        uint32_t* const words = (uint32_t*)(vt + rows * S::ROW);
        char* const buf = resident_map(lds, rows, 2 * S::ROW, wave, S::MAP);
        int tile = worker * WAVES + wave;
        if (AHEAD && tile < tiles) fetch(tile);
        all_tokens<T, KS, 64 * WAVES>(p, b, head, rows, lds, S::ROW, vt, S::ROW, words, tid);
        __syncthreads();
        if (!few && p.mask) {
            int have = 0;
            for (int i = lane; i < rows / 32; i += 64) have += __popc(words[i]);
#pragma unroll
            for (int d = 1; d < 64; d *= 2) have += __shfl_xor(have, d);
            few = __builtin_amdgcn_readfirstlane(have) <= 64;
        }
        while (tile < tiles) {
            if (!AHEAD) fetch(tile);
            const size_t at = plane;
            const int n = n0;
            start(buf);
            tile += p.workers * WAVES;
            if (AHEAD && tile < tiles) fetch(tile);
            if (few) {
                for (int i = 0; i < rows / 32; ++i) {
                    const uint32_t word = __builtin_amdgcn_readfirstlane(words[i]);
                    if (word) sum_delta(lds + i * 32 * S::ROW, vt + i * 32 * S::ROW, word);
                }
                delta = other_half_sum(delta);
            }
            for (int i = 0; i < rows / 32; ++i) {
                const uint32_t word = __builtin_amdgcn_readfirstlane(words[i]);
                if (word) step(lds + i * 32 * S::ROW, vt + i * 32 * S::ROW, word);
            }
            finish(at, n, buf);
        }
    } else {
        char* const buf = lds + S::BUFFERS * S::STAGE + wave * S::MAP;
        const int stages = (p.L + S::TB - 1) / S::TB;
        fetch(min(worker * WAVES + wave, tiles - 1));                // (waves past the end: the last tile again, the same bits)
        if (!few && p.mask) {
            int have = 0;
            for (int t = tid; t < p.L; t += 256) have += p.mask[(size_t)b * p.L + t] != 0;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) have += __shfl_xor(have, d);
            int* const counts = (int*)lds;
            if (lane == 0) counts[wave] = have;
            __syncthreads();
            few = __builtin_amdgcn_readfirstlane(counts[0] + counts[1] + counts[2] + counts[3]) <= 64;
            __syncthreads();
        }
        start(buf);
        if (few) {                                                   // over the tokens once more, with nothing on its way meanwhile
#pragma unroll 1
            for (int st = 0; st < stages; ++st) {
                TokenStage<T, KS, S::TB> here;
                here.fetch(p, b, head, st * S::TB, tid);
                const uint64_t in = here.bits(0);
                if (!in) continue;                                   // (the same for all waves)
                lds_barrier();
                here.put(lds, S::ROW, lds + S::TB * S::ROW, S::ROW, tid);
                lds_barrier();
#pragma unroll 1
                for (int i = 0; i < S::TB / 32; ++i) {
                    const uint32_t word = (uint32_t)(in >> (32 * i));
                    if (word) sum_delta(lds + 32 * i * S::ROW, lds + (S::TB + 32 * i) * S::ROW, word);
                }
            }
            delta = other_half_sum(delta);
            lds_barrier();
        }
        TokenStage<T, KS, S::TB> next;
        next.fetch(p, b, head, 0, tid);
        for (int st = 0; st < stages; ++st) {
            char* const kt = lds + (S::BUFFERS == 2 ? st & 1 : 0) * S::STAGE;
            char* const vt = kt + S::TB * S::ROW;
            if (S::BUFFERS == 1 && st) lds_barrier();
            next.put(kt, S::ROW, vt, S::ROW, tid);
            const uint64_t in = next.bits(0);
            if (st + 1 < stages) next.fetch(p, b, head, (st + 1) * S::TB, tid);
            lds_barrier();
            for (int i = 0; i < S::TB / 32; ++i) {
                const uint32_t word = (uint32_t)(in >> (32 * i));
                if (word) step(kt + 32 * i * S::ROW, vt + 32 * i * S::ROW, word);
            }
        }
        finish(plane, n0, buf);
    }
}

// gk and gv.  A lane is a token: WT waves of a workgroup hold 32 tokens each, 4 / WT waves the same tokens on other positions.  A stage is
// PX positions of a head: q and gout as they are stored, [channel][position]; the scores as [position][token], so that the weights are
// the operand of the products over the positions.
// Both maps are read from LDS along the positions and across them.  16 bits: rows without gaps, their 16-byte pieces exchanged by the row's number and the
// two halves of a piece by its bit 4, which puts the four rows of a turned request and the 32 rows of an 8-byte one on all banks.  fp32:
// rows 16 bytes longer than their values.
template <typename T, int KS, int WT> struct AttendTokenShape {
    static constexpr int WP = 4 / WT, PX = WP == 4 ? 128 : 64, PITCH = PX * (int)sizeof(T) + (sizeof(T) == 4 ? 16 : 0);
    static constexpr int TILE = (KS + 1) / 2 * 32 * PITCH, STAGE = 2 * TILE + 2 * PX * 4;       // (rows past the channels: read, their results are not stored)
    static constexpr int BUFFERS = 2 * STAGE <= 160 * 1024 ? 2 : 1;
    static constexpr int LDS = BUFFERS * STAGE;
};
template <int PX> __device__ __forceinline__ int map_swap(int r) { return PX == 128 ? (r & 3) * 4 + ((r >> 2) & 3) : ((r >> 1) & 1) * 4 + ((r >> 2) & 3); }
// byte of positions 4 * piece .. + 3 of row r (16 bits)
template <int PX> __device__ __forceinline__ int map_piece(int r, int piece) {
    return r * PX * 2 + (((piece >> 1) ^ map_swap<PX>(r)) << 4) + (((piece ^ (r >> 4)) & 1) << 3);
}

// operand A from [channel][position] in LDS: the positions as rows (from p0), channels contracted (step s)
template <typename T, int PX, int PITCH> __device__ __forceinline__ MatFrag<T> map_turned(const char* tile, int p0, int s, int lane) {
    const int half = lane >> 5;
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f.v[i] = *(const float*)(tile + (16 * s + 8 * half + i) * PITCH + (p0 + (lane & 31)) * 4);
    } else {
        const int j = lane & 15, piece = (p0 + (lane & 16)) / 4 + (j & 3);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x2 v = lds_turned(tile + map_piece<PX>(16 * s + 8 * half + 4 * i + (j >> 2), piece));
            f.w[2 * i] = v.x; f.w[2 * i + 1] = v.y;
        }
    }
    return f;
}
// ... and the channels as rows (32 from dt * 32), positions contracted in the order of an accumulator's rows
template <typename T, int PX, int PITCH> __device__ __forceinline__ MatFrag<T> map_rows(const char* tile, int dt, int p0, int j, int lane) {
    const int half = lane >> 5, r = dt * 32 + (lane & 31);
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
        const char* row = tile + r * PITCH + (p0 + 16 * j + 4 * half) * 4;
        const u32x4 a = *(const u32x4*)row, b = *(const u32x4*)(row + 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) { f.v[i] = __uint_as_float(a[i]); f.v[4 + i] = __uint_as_float(b[i]); }
    } else {
        const int piece = (p0 + 16 * j) / 4 + half;
        const u32x2 a = *(const u32x2*)(tile + map_piece<PX>(r, piece)), b = *(const u32x2*)(tile + map_piece<PX>(r, piece + 2));
        f.w = u32x4{a.x, a.y, b.x, b.y};
    }
    return f;
}

template <typename T, int KS, int WT>
__global__ void __launch_bounds__(256, attend_token_groups(sizeof(T) == 4, KS, WT)) attend_grad_tokens_kernel(const AttendParams p) {
    using S = AttendTokenShape<T, KS, WT>;
    constexpr bool SPLIT = sizeof(T) == 2 && WT < 4;                 // (fewer token waves: few tokens, and some other numbers of them)
    constexpr int DT = (KS + 1) / 2, PX = S::PX, PITCH = S::PITCH, E = 16 / (int)sizeof(T), PIECES = PX / E, ALL = KS * 16 * PIECES, COUNT = (ALL + 255) / 256;
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
    const bool some = __ballot(in) != 0;                             // (of the wave's tokens; else it only helps to bring the stages)
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
            if (d < p.D && (ALL % 256 == 0 || c < ALL)) {
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
            const int c = tid + i * 256, d = c / PIECES;
            if (ALL % 256 && c >= ALL) break;
            if constexpr (sizeof(T) == 4) {
                *(u32x4*)(tq + d * PITCH + c % PIECES * 16) = rq[i];
                *(u32x4*)(tg + d * PITCH + c % PIECES * 16) = rg[i];
            } else {
                const int o = d * PITCH + ((c % PIECES ^ map_swap<PX>(d)) << 4);
                const bool turn = d & 16;                            // the halves of the piece exchanged
                *(u32x4*)(tq + o) = turn ? u32x4{rq[i][2], rq[i][3], rq[i][0], rq[i][1]} : rq[i];
                *(u32x4*)(tg + o) = turn ? u32x4{rg[i][2], rg[i][3], rg[i][0], rg[i][1]} : rg[i];
            }
        }
        if (tid < 2 * PX) tl[tid] = rl;
        if (st + 1 < last) fetch(st + 1);
        lds_barrier();
#pragma unroll 1
        for (int p0 = some ? wp * 32 : PX; p0 < PX; p0 += 32 * S::WP) {
            f32x16 s, dp;
            mat_zero(s);
            mat_zero(dp);
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                mat_mul<T>(s, map_turned<T, PX, PITCH>(tq, p0, i, lane), k[i]);
                mat_mul<T>(dp, map_turned<T, PX, PITCH>(tg, p0, i, lane), v[i]);
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
                MatFrag<T> fe, fd, re, rd;
                if constexpr (SPLIT) {
                    mat_split<T>(e + 8 * j, fe, re);
                    mat_split<T>(ds + 8 * j, fd, rd);
                } else {
                    fe = mat_from_acc<T>(e + 8 * j);
                    fd = mat_from_acc<T>(ds + 8 * j);
                }
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    const MatFrag<T> g = map_rows<T, PX, PITCH>(tg, i, p0, j, lane), x = map_rows<T, PX, PITCH>(tq, i, p0, j, lane);
                    mat_mul<T>(av[i], g, fe);
                    mat_mul<T>(ak[i], x, fd);
                    if constexpr (SPLIT) { mat_mul<T>(av[i], g, re); mat_mul<T>(ak[i], x, rd); }
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
template <typename K> hipError_t attend_launch(K kernel, size_t items, int threads, int lds, const AttendParams& p, hipStream_t s) {
    hipError_t e = allow_dynamic_lds((const void*)kernel, RESIDENT_MOST);        // (the most that any call of it asks for)
    if (e != hipSuccess) return e;
    if (items * threads >= ((size_t)1 << 32)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kernel, dim3((unsigned)items), dim3(threads), lds, s, p);
    return hipGetLastError();
}
template <typename T, int KS> hipError_t launch_attend_many(const AttendParams& p, const AttendPlan& plan, hipStream_t s) {
    const size_t groups = (size_t)p.B * p.kv;
    if (plan.waves == 8) return attend_launch(attend_kernel<T, KS, 8, true>, groups * p.workers, 512, plan.lds, p, s);
    if constexpr (sizeof(T) == 2) {
        if (plan.resident && p.L <= SPLIT_MOST) return attend_launch(attend_kernel<T, KS, 4, true, true>, groups * p.workers, 256, plan.lds, p, s);
    }
    if (plan.resident) return attend_launch(attend_kernel<T, KS, 4, true>, groups * p.workers, 256, plan.lds, p, s);
    return attend_launch(attend_kernel<T, KS, 4, false>, groups * p.workers, 256, AttendShape<T, KS>::LDS, p, s);
}
template <typename T, int KS> hipError_t launch_attend_head(const AttendParams& p, const AttendPlan& plan, hipStream_t s) {
    if (plan.few) {
        const size_t tiles = ((size_t)p.per * p.N + 31) / 32;
        auto kernel = attend_few_kernel<T, KS, false>;
        if constexpr (sizeof(T) == 2) { if (p.L <= SPLIT_MOST) kernel = attend_few_kernel<T, KS, true>; }
        hipError_t e = attend_launch(kernel, (size_t)p.B * p.kv * tiles * p.splits, 256, AttendFewShape<T, KS>::lds(p.L, p.splits), p, s);
        if (e != hipSuccess || p.splits == 1) return e;
        return attend_launch(attend_join_kernel<T>, (size_t)p.B * p.kv * tiles * ((p.D + 7) / 8), 256, (p.splits + 8) * 32 * 4, p, s);
    }
    return launch_attend_many<T, KS>(p, plan, s);
}
template <typename T, int KS> hipError_t launch_grad_q(const AttendParams& p, const AttendPlan& plan, hipStream_t s) {
    const size_t groups = (size_t)p.B * p.kv;
    if constexpr (attend_grad_waves(sizeof(T) == 4, KS) > 1) {
        if (plan.waves == 8) return attend_launch(attend_grad_q_kernel<T, KS, 8, true>, groups * p.workers, 512, plan.lds, p, s);
    }
    if (plan.resident) return attend_launch(attend_grad_q_kernel<T, KS, 4, true>, groups * p.workers, 256, plan.lds, p, s);
    return attend_launch(attend_grad_q_kernel<T, KS, 4, false>, groups * p.workers, 256, AttendGradShape<T, KS>::LDS, p, s);
}
template <typename T, int KS> hipError_t launch_attend_bwd_head(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s) {
    AttendParams q = p;
    q.workers = plan.q.workers;
    hipError_t e = launch_grad_q<T, KS>(q, plan.q, s);
    if (e != hipSuccess || (!p.gk && !p.gv)) return e;
    const size_t items = (size_t)p.B * p.kv * p.splits * ((p.L + 32 * plan.token_waves - 1) / (32 * plan.token_waves));
    if constexpr (sizeof(T) == 2 || KS < 7) {                        // (fp32 heads of more than 96 channels: registers for four token waves alone)
        if (plan.token_waves == 2) return attend_launch(attend_grad_tokens_kernel<T, KS, 2>, items, 256, AttendTokenShape<T, KS, 2>::LDS, p, s);
        if (plan.token_waves == 1) return attend_launch(attend_grad_tokens_kernel<T, KS, 1>, items, 256, AttendTokenShape<T, KS, 1>::LDS, p, s);
    }
    return attend_launch(attend_grad_tokens_kernel<T, KS, 4>, items, 256, AttendTokenShape<T, KS, 4>::LDS, p, s);
}
// by the steps of 16 channels of a head
#define GSPN_BY_STEPS(call)                                                                                                               \
    switch ((p.D + 15) / 16) {                                                                                                            \
        case 1: return call<T, 1>(p, plan, s);                                                                                            \
        case 2: return call<T, 2>(p, plan, s);                                                                                            \
        case 3: return call<T, 3>(p, plan, s);                                                                                            \
        case 4: return call<T, 4>(p, plan, s);                                                                                            \
        case 5: return call<T, 5>(p, plan, s);                                                                                            \
        case 6: return call<T, 6>(p, plan, s);                                                                                            \
        case 7: return call<T, 7>(p, plan, s);                                                                                            \
        default: return call<T, 8>(p, plan, s);                                                                                           \
    }
template <typename T> hipError_t launch_attend_type(const AttendParams& p, const AttendPlan& plan, hipStream_t s) { GSPN_BY_STEPS(launch_attend_head) }
template <typename T> hipError_t launch_attend_bwd_type(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s) { GSPN_BY_STEPS(launch_attend_bwd_head) }
#undef GSPN_BY_STEPS
// instantiated in a translation unit per storage type
hipError_t launch_attend_f32(const AttendParams& p, const AttendPlan& plan, hipStream_t s);
hipError_t launch_attend_bf16(const AttendParams& p, const AttendPlan& plan, hipStream_t s);
hipError_t launch_attend_f16(const AttendParams& p, const AttendPlan& plan, hipStream_t s);
hipError_t launch_attend_bwd_f32(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s);
hipError_t launch_attend_bwd_bf16(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s);
hipError_t launch_attend_bwd_f16(const AttendParams& p, const AttendBackPlan& plan, hipStream_t s);

}  // namespace gspn
