// Operands of the matrix cores for the products and the attention on feature maps (gfx950), one form for the three storage types.
//
// A step multiplies 32 x 32 tiles over 16 positions of the contracted axis.  A lane feeds row (operand A) or column (B) lane % 32 and the
// eight positions that its half of the wave (lane / 32) has: an operand is eight values of storage type T per lane, whatever the positions
// are called, as long as A and B agree.  16-bit types: one v_mfma_f32_32x32x16; fp32: eight v_mfma_f32_32x32x2, value i of both halves each.
// Accumulator register r of a lane holds row 8*(r/4) + 4*(lane/32) + r%4, column lane%32, in fp32.  The columns of a result are thus where
// a following product wants its operand B: registers 8*s .. 8*s+7 are the operand of step s over the result's rows, with the positions
// acc_row(8*s + i, half).
#pragma once
#include "gspn_unaligned.hpp"

namespace gspn {

typedef __bf16 mat_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 mat_f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <typename T> struct MatFrag { u32x4 w; };                       // eight 16-bit values
template <> struct MatFrag<float> { float v[8]; };

__device__ __forceinline__ int acc_row(int r, int half) { return 8 * (r >> 2) + 4 * half + (r & 3); }

template <typename T> __device__ __forceinline__ void mat_mul(f32x16& c, const MatFrag<T>& a, const MatFrag<T>& b) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[i], b.v[i], c, 0, 0, 0);
    } else if constexpr (__is_same(T, f16_t)) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(mat_f16x8, a.w), __builtin_bit_cast(mat_f16x8, b.w), c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(mat_bf16x8, a.w), __builtin_bit_cast(mat_bf16x8, b.w), c, 0, 0, 0);
    }
}
__device__ __forceinline__ void mat_zero(f32x16& c) {
#pragma unroll
    for (int r = 0; r < 16; ++r) c[r] = 0.f;
}

// registers 8*s .. 8*s+7 of an accumulator as an operand (rounded to T, to nearest even)
template <typename T> __device__ __forceinline__ MatFrag<T> mat_from_acc(const float* v) {
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f.v[i] = v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) f.w[i] = pack_word<T>(v[2 * i], v[2 * i + 1]);
    }
    return f;
}

// ... as two operands, the rounded values and what the rounding left (rounded in its turn): their products add up to that of some twice as many bits
template <typename T> __device__ __forceinline__ void mat_split(const float* v, MatFrag<T>& hi, MatFrag<T>& lo) {
    hi = mat_from_acc<T>(v);
    if constexpr (sizeof(T) == 2) {
        float rest[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) rest[i] = v[i] - rg_elem<T>(hi.w, i);
        lo = mat_from_acc<T>(rest);
    }
}

typedef __attribute__((address_space(3))) char lds_char;
// (an LDS pointer in its own address space, for the instructions that take no other)
__device__ __forceinline__ lds_char* lds_ptr(const void* p) { return (lds_char*)(__attribute__((address_space(3))) void*)(void*)p; }

// eight consecutive values at p (16-byte aligned): an operand whose contracted axis is contiguous
template <typename T> __device__ __forceinline__ MatFrag<T> mat_contiguous(const char* p) {
    MatFrag<T> f;
    if constexpr (sizeof(T) == 4) {
        const u32x4 a = *(const u32x4*)p, b = *(const u32x4*)(p + 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) { f.v[i] = __uint_as_float(a[i]); f.v[4 + i] = __uint_as_float(b[i]); }
    } else {
        f.w = *(const u32x4*)p;
    }
    return f;
}

// 16-bit: four rows of 16 columns per 16 lanes, turned on the way (ds_read_b64_tr_b16): lane j of the 16 asks for the 8 bytes at row j / 4,
// columns 4 * (j % 4) .. + 3, and gets rows 0 .. 3 of column j
__device__ __forceinline__ u32x2 lds_turned(const char* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)lds_ptr(p)));
}

// a 16-byte piece moved down by s elements (0 .. all but one), zeros behind
template <typename T> __device__ __forceinline__ u32x4 piece_down(u32x4 v, int s) {
    uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
    const int bits = s * 8 * (int)sizeof(T);
    if (bits >= 64) { lo = hi; hi = 0; }
    const int b = bits & 63;
    lo = lo >> b | (hi << 1) << (63 - b);
    hi = hi >> b;
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// 16 bytes of a row from element `at` on, zeros from element `limit` on; every access lies within the row
template <typename T> __device__ __forceinline__ u32x4 row_chunk(const T* row, int at, int limit) {
    constexpr int E = 16 / (int)sizeof(T);
    u32x4 v = {0, 0, 0, 0};
    if (at + E <= limit) v = rg_load(row + at);
    else if (at < limit) {
        if (limit >= E) v = piece_down<T>(rg_load(row + (limit - E)), at - (limit - E));
        else {
            if constexpr (sizeof(T) == 4) {
                if (at + 0 < limit) v[0] = ((const uint32_t*)row)[at + 0];
                if (at + 1 < limit) v[1] = ((const uint32_t*)row)[at + 1];
                if (at + 2 < limit) v[2] = ((const uint32_t*)row)[at + 2];
            } else {
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (at + i < limit) v[i >> 1] |= (uint32_t)((const uint16_t*)row)[at + i] << (16 * (i & 1));
            }
        }
    }
    return v;
}

// eight values of a row from element `at` on, widened; `n` of them exist (the rest: 0)
template <typename T> __device__ __forceinline__ void row_values(const T* p, int n, float* v) {
    if (n >= 8) {
        if constexpr (sizeof(T) == 4) {
            const u32x4 a = rg_load(p), b = rg_load(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(a[i]); v[4 + i] = __uint_as_float(b[i]); }
        } else {
            const u32x4 a = rg_load(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = rg_elem<T>(a, i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? ldf(p + i) : 0.f;
    }
}
// ... for rows that end inside the eight values, out of the way of the code that all others run
template <typename T> __device__ __forceinline__ void row_values_slow(const T* p, int n, float* v) {
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
        const float x = i < n ? ldf(p + i) : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e == i ? x : v[e];
    }
}
template <typename T> __device__ __forceinline__ void row_store(T* p, int n, const float* v) {
    if (n >= 8) {
        if constexpr (sizeof(T) == 4) {
            rg_store(p, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
            rg_store(p + 4, u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])});
        } else {
            rg_store(p, u32x4{pack_word<T>(v[0], v[1]), pack_word<T>(v[2], v[3]), pack_word<T>(v[4], v[5]), pack_word<T>(v[6], v[7])});
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) stf(p + i, v[i]);
    }
}

}  // namespace gspn
