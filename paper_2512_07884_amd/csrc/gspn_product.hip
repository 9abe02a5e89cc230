// Host side of the products with an epilogue (gspn_product_impl.hpp): which tile a call runs, and the sums over partial results.
#include "gspn_product_impl.hpp"

namespace gspn {

namespace {

size_t tiles_of(const ProductParams& p, bool gated, int bm, int bn, int images) {
    const int rows = gated ? bm / 2 : bm;
    return (size_t)((p.M + rows - 1) / rows) * ((p.N + bn - 1) / bn) * images;
}

// 256 x 256 in 16 bits reads each operand half as often as 128 x 128, but a CU holds one of those: where three quarters of what the CUs compute is wanted, or
// three fifths over a long contraction.
bool huge_tiles(const ProductParams& p, int form, bool gated, int images, int dtype) {
    if (dtype == 0 || p.K < 256) return false;
    const bool direct = gated ? product_direct<ProductShape<bf16_t, PRODUCT_FORWARD, OUT_GATED, 2, 2, 4, 4, 1>>(p, form, 8, 2)
                              : product_direct<ProductShape<bf16_t, PRODUCT_FORWARD, OUT_PROJECT, 2, 2, 4, 4, 1>>(p, form, 8, 2);
    if (!direct) return false;
    const size_t tiles = tiles_of(p, gated, 256, 256, images), rows = (gated ? 2 : 1) * (size_t)p.M;
    const double used = (double)rows * p.N * images / ((double)((tiles + 255) / 256) * 256 * 65536);
    return used >= 0.75 || (used >= 0.6 && p.K >= 2048);
}
// The gradient of the matrix: 64 x 64 where those, with the pixels cut into as many stretches as make two workgroups for every CU, use three quarters of them.
// 128 x 128 at its best number of stretches and 64 x 64 as chosen (us): bf16 512 x 512 on two 64x64 maps 27 18, 1536 x 384 on four 32x32 26 17, 2048 x 1024 on two
// 64x64 62 52, 1152 x 1152 (not three quarters) 44 51; fp32 2048 x 256 on eight 32x32 87 71, 1152 x 144 on two 64x64 68 38.
bool medium_gradient(const ProductParams& p) {
    const size_t tiles = tiles_of(p, false, 64, 64, 1);
    // (its stages are 128 pixels of an image, the larger tile's 32: of small images most of them would be empty)
    if ((p.K + 127) / 128 * 4 * 2 > (p.K + 31) / 32 * 3) return false;
    return p.M <= 64 || p.N <= 64 || (tiles <= 512 && 512 / tiles * tiles >= 384);
}
// Large tiles where there are two for every CU; flat ones where there are nearly as many of those; smaller ones, with several waves over the contracted axis,
// where there are not.  Rows of fewer pixels than a tile has columns are requested piece by piece, so a narrower tile comes first.
// Times (us) on 128 x 128, 32 x 128, 64 x 64, 64 x 32 tiles: bf16 1152 x 144 on two 64x64 maps 13 14 14 25, 384 x 384 on eight 28x28 13 9 9 12, 144 x 1152 on two
// 64x64 23 12 12 13, 512 x 512 on one 33x33 15 9 8 8, 768 x 768 on 64 of 7x7 38 57 22 20, 1024 x 1024 on two 64x64 26 34 32 52; fp32 1024 x 1024 on two
// 64x64 135 136 142 149, 96 x 96 on 64 of 56x56 72 52 65 111, 384 x 384 on eight 28x28 32 25 24 24, 96 x 384 on one 14x14 30 10 11 8.
int product_tile(const ProductParams& p, int form, int outcome, int dtype) {
    const bool gated = outcome == OUT_GATED || outcome == OUT_GATED_GRAD;
    if (form == PRODUCT_GRAD_MATRIX) return medium_gradient(p) ? TILE_MEDIUM : (huge_tiles(p, form, false, 1, dtype) ? TILE_HUGE : TILE_LARGE);
    if (p.N < 64) return TILE_SMALL;
    if (p.N >= 128) {
        if (huge_tiles(p, form, gated, p.images, dtype)) return TILE_HUGE;
        if (tiles_of(p, gated, 128, 128, p.images) >= 512 && (dtype != 0 || p.K >= 512) && p.M > 32) return TILE_LARGE;
        if (tiles_of(p, gated, gated ? 64 : 32, 128, p.images) >= (dtype == 0 ? 256 : 448)) return TILE_FLAT;
    }
    return tiles_of(p, gated, 64, 64, p.images) >= 128 ? TILE_MEDIUM : TILE_SMALL;
}
// a tile's side, its columns and the waves along them
void tile_columns(int tile, int* bn, int* wn) {
    *bn = tile == TILE_HUGE ? 256 : (tile == TILE_MEDIUM ? 64 : (tile == TILE_SMALL ? 32 : 128));
    *wn = tile == TILE_SMALL ? 1 : (tile == TILE_LARGE || tile == TILE_MEDIUM ? 2 : 4);
}

// Few parts: a thread adds those of four neighbouring results, in order
template <typename T> __global__ void __launch_bounds__(256) sum_few_kernel(const float* __restrict__ in, T* __restrict__ out, int parts, size_t n, const float* __restrict__ in2, T* __restrict__ out2) {
    if (blockIdx.y) { in = in2; out = out2; }
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    const int have = (int)min((size_t)4, n - i);
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 0; k < parts; ++k) {
        if (have == 4) {
            const u32x4 v = rg_load(in + (size_t)k * n + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += __uint_as_float(v[e]);
        } else {
            for (int e = 0; e < have; ++e) sum[e] += in[(size_t)k * n + i + e];
        }
    }
    for (int e = 0; e < have; ++e) stf(out + i + e, sum[e]);
}
// Many parts of few results (a thousand threads per 32 of them): 32 neighbouring results per workgroup, each thread every 32nd part of one, the 32 sums added in order
template <typename T> __global__ void __launch_bounds__(1024) sum_many_kernel(const float* __restrict__ in, T* __restrict__ out, int parts, size_t n, const float* __restrict__ in2, T* __restrict__ out2) {
    if (blockIdx.y) { in = in2; out = out2; }
    __shared__ float strip[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const size_t i = (size_t)blockIdx.x * 32 + x;
    float sum = 0.f;
    if (i < n)
#pragma unroll 4
        for (int k = y; k < parts; k += 32) sum += in[(size_t)k * n + i];
    strip[y][x] = sum;
    __syncthreads();
    if (y == 0 && i < n) {
#pragma unroll
        for (int k = 1; k < 32; ++k) sum += strip[k][x];
        stf(out + i, sum);
    }
}
template <typename T> hipError_t sum_parts_as(const float* in, void* out_, int parts, size_t n, hipStream_t s, const float* in2, void* out2_) {
    T *const out = (T*)out_, *const out2 = (T*)out2_;
    const unsigned sums = out2 ? 2 : 1;
    const bool many = parts > 16 && n <= 32768;
    const size_t blocks = many ? (n + 31) / 32 : (n + 1023) / 1024;
    if (blocks * 1024 >= ((size_t)1 << 32)) return hipErrorInvalidValue;
    if (many) hipLaunchKernelGGL(sum_many_kernel<T>, dim3((unsigned)blocks, sums), dim3(1024), 0, s, in, out, parts, n, in2, out2);
    else hipLaunchKernelGGL(sum_few_kernel<T>, dim3((unsigned)blocks, sums), dim3(256), 0, s, in, out, parts, n, in2, out2);
    return hipGetLastError();
}

constexpr int ROW_SUM = 4096;                          // values of a row that a wave adds
template <typename T> __global__ void __launch_bounds__(256) row_sums_kernel(const T* __restrict__ g, float* __restrict__ parts, int images, int M, int N) {
    const int lane = threadIdx.x & 63, chunks = (N + ROW_SUM - 1) / ROW_SUM;
    const size_t item = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (item >= (size_t)images * chunks * M) return;
    const size_t part = item / M;
    const int m = (int)(item - part * M), image = (int)(part / chunks), chunk = (int)(part - (size_t)image * chunks);
    const T* row = g + ((size_t)image * M + m) * N;
    const int end = min(N, (chunk + 1) * ROW_SUM);
    float sum = 0.f, v[8];
    for (int n = chunk * ROW_SUM + lane * 8; n < end; n += 512) {
        row_values(row + n, min(8, end - n), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[e];
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) parts[part * M + m] = sum;
}

}  // namespace

int product_sum_parts(const ProductParams& p, int outcome, int dtype) {
    int bn, wn;
    tile_columns(product_tile(p, PRODUCT_FORWARD, outcome, dtype), &bn, &wn);
    return p.images * ((p.N + bn - 1) / bn) * wn;
}

// Stretches of the pixels: two workgroups for every CU (256 x 256: one), each with six stages of 64 pixels (fp32: 32) at least
int product_splits(const ProductParams& p, int dtype) {
    const int tile = product_tile(p, PRODUCT_GRAD_MATRIX, OUT_PLAIN, dtype);
    const int side = tile == TILE_HUGE ? 256 : (tile == TILE_LARGE ? 128 : 64), stage = dtype == 0 ? 32 : 64;
    const size_t tiles = tiles_of(p, false, side, side, 1), stages = (size_t)((p.K + stage - 1) / stage) * p.images;
    // (a call of 64 x 64 has two of them in a stage)
    size_t n = tile == TILE_HUGE ? 256 / tiles : (tile == TILE_LARGE ? (512 + tiles / 2) / tiles : 512 / tiles);
    if (n > stages / 6) n = stages / 6;
    return n < 1 ? 1 : (int)n;
}

hipError_t launch_product(const ProductParams& p, int form, int outcome, int dtype, hipStream_t s) {
    const int tile = product_tile(p, form, outcome, dtype);
    return dtype == 0 ? launch_product_f32(p, form, outcome, tile, s)
         : dtype == 1 ? launch_product_bf16(p, form, outcome, tile, s) : launch_product_f16(p, form, outcome, tile, s);
}

hipError_t launch_sum_parts(const float* in, void* out, int parts, size_t n, int dtype, hipStream_t s, const float* in2, void* out2) {
    return dtype == 0 ? sum_parts_as<float>(in, out, parts, n, s, in2, out2)
         : dtype == 1 ? sum_parts_as<bf16_t>(in, out, parts, n, s, in2, out2) : sum_parts_as<f16_t>(in, out, parts, n, s, in2, out2);
}

int row_sum_parts(int images, int, int N) { return images * ((N + ROW_SUM - 1) / ROW_SUM); }

hipError_t launch_row_sums(const void* g, void* out, float* parts, int images, int M, int N, int dtype, hipStream_t s) {
    const size_t blocks = ((size_t)row_sum_parts(images, M, N) * M + 3) / 4;
    if (blocks * 256 >= ((size_t)1 << 32)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks), block(256);
    if (dtype == 0) hipLaunchKernelGGL(row_sums_kernel<float>, grid, block, 0, s, (const float*)g, parts, images, M, N);
    else if (dtype == 1) hipLaunchKernelGGL(row_sums_kernel<bf16_t>, grid, block, 0, s, (const bf16_t*)g, parts, images, M, N);
    else hipLaunchKernelGGL(row_sums_kernel<f16_t>, grid, block, 0, s, (const f16_t*)g, parts, images, M, N);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_sum_parts(parts, out, row_sum_parts(images, M, N), (size_t)M, dtype, s);
}

}  // namespace gspn
