// Products with 4-bit weights: y[r][n] = sum_k x[r][k] W[n][k].
//
// A tile is 16 rows of W x 128 columns, 1 KB: lane l = 16 q + r of a wave holds the 16 bytes of row r, group q (32 columns, one scale),
// so a load of a wave reads 1 KB of consecutive memory and every lane needs one scale byte per tile.  The four dwords of a lane are the A
// operands of four 16x16x32 matrix instructions: instruction j contracts over the columns 32 q + 8 j .. + 7 of every group q, and x is
// laid out in the same order (the order of a contraction does not matter).
#pragma once
#include "q4.h"

// x as B operands: [row tile of 16][tile of 128 columns][plane][j][lane][8], zero beyond rows and K.  PLANES = 1: bf16; 3: fp32 exactly.
template <typename T, int PLANES>
__global__ void w4_stage_kernel(const T* __restrict__ x, int64_t ld, int rows, int k, int kt, uint4* __restrict__ xs) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t total = (int64_t)((rows + 15) / 16) * kt * 256;
    if (id >= total) return;
    const int lane = (int)(id & 63), j = (int)(id >> 6) & 3;
    const int64_t tile = id >> 8;
    const int t = (int)(tile % kt), row = (int)(tile / kt) * 16 + (lane & 15), k0 = t * 128 + (lane >> 4) * 32 + j * 8;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = row < rows && k0 + i < k ? ld1(x + row * ld + k0 + i) : 0.f;
    u32x4_t o[PLANES];
    q4_operand<PLANES>(v, o);
#pragma unroll
    for (int p = 0; p < PLANES; ++p) xs[((tile * PLANES + p) * 4 + j) * 64 + lane] = __builtin_bit_cast(uint4, o[p]);
}

struct W4Args {
    const u32x4_t* codes;
    const uint32_t* scales;
    int n, k, nt, kt, ks;
    const u32x4_t* xs;
    int rows;
    void* y;
    int64_t ldy;
    float* part;        // partial sums [split][rows][n], null: the block writes y
    int units;          // groups of four tiles (512 columns) per split
};

// A block owns NT tiles of rows of W and R tiles of rows of x; its waves share K in units of 512 columns.
template <typename T, int NT, int R, int PLANES>
__global__ __launch_bounds__(512) void w4_kernel(W4Args a) {
    extern __shared__ float w4_lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * NT, rt0 = blockIdx.z * R, rts = (a.rows + 15) >> 4;
    const int u0 = blockIdx.y * a.units, u1 = min(a.ks, u0 + a.units);
    f32x4_t acc[NT][R] = {};
    for (int u = u0 + wave; u < u1; u += waves) {
        uint32_t sc[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) sc[i] = a.scales[((int64_t)min(n0 + i, a.nt - 1) * a.ks + u) * 64 + lane];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int t = u * 4 + c;
            if (t >= a.kt) break;
            u32x4_t w[NT];
#pragma unroll
            for (int i = 0; i < NT; ++i) w[i] = a.codes[((int64_t)min(n0 + i, a.nt - 1) * a.kt + t) * 64 + lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32x4_t b[R][PLANES];
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int p = 0; p < PLANES; ++p)
                        b[r][p] = a.xs[((((int64_t)min(rt0 + r, rts - 1) * a.kt + t) * PLANES + p) * 4 + j) * 64 + lane];
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const u32x4_t m = q4_decode8(w[i][j], (sc[i] >> (8 * c)) << 23);
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int p = 0; p < PLANES; ++p) acc[i][r] = q4_mfma(m, b[r][p], acc[i][r]);
                }
            }
        }
    }
    // the waves' parts, added in the order of the waves
    f32x4_t* lds = reinterpret_cast<f32x4_t*>(w4_lds);
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int r = 0; r < R; ++r) lds[(wave * NT * R + i * R + r) * 64 + lane] = acc[i][r];
    __syncthreads();
    for (int e = wave; e < NT * R; e += waves) {
        f32x4_t s = lds[e * 64 + lane];
        for (int w = 1; w < waves; ++w) s += lds[(w * NT * R + e) * 64 + lane];
        const int row = (rt0 + e % R) * 16 + (lane & 15), n = (n0 + e / R) * 16 + (lane >> 4) * 4;
        if (row >= a.rows) continue;
        if (a.part) {
            float* o = a.part + ((int64_t)blockIdx.y * a.rows + row) * a.n + n;
#pragma unroll
            for (int i = 0; i < 4; ++i) if (n + i < a.n) o[i] = s[i];
        } else {
            T* o = static_cast<T*>(a.y) + row * a.ldy + n;
#pragma unroll
            for (int i = 0; i < 4; ++i) if (n + i < a.n) st1(o + i, s[i]);
        }
    }
}

template <typename T>
__global__ void w4_sum_kernel(const float* __restrict__ part, int splits, int rows, int n, T* __restrict__ y, int64_t ldy) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, total = (int64_t)rows * n;
    if (id >= total) return;
    float s = part[id];
    for (int i = 1; i < splits; ++i) s += part[i * total + id];
    st1(y + id / n * ldy + id % n, s);
}

// Weights [n][k] (fp32 or bf16, rows `ld` apart) to tiles: 16 lanes take one group of 32 columns.
template <typename T>
__global__ void w4_pack_kernel(const T* __restrict__ w, int64_t ld, int n, int k, int nt, int kt, int ks, uint8_t* __restrict__ codes,
                               uint8_t* __restrict__ scales) {
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4;
    const int l = threadIdx.x & 15, groups = ks * 16;
    const int64_t row = item / groups;
    const int g = (int)(item % groups);
    if (row >= (int64_t)nt * 16) return;                 // whole rows of 16 lanes leave together
    const int c = g * 32 + 2 * l;
    const float x0 = row < n && c < k ? ld1(w + row * ld + c) : 0.f, x1 = row < n && c + 1 < k ? ld1(w + row * ld + c + 1) : 0.f;
    const bool bad = row16_or(!q4_finite(x0) || !q4_finite(x1)) != 0;
    const int s = q4_scale_byte(row16_max(fmaxf(fabsf(x0), fabsf(x1))));
    const int64_t nti = row >> 4;
    const int r = (int)(row & 15), q = g & 3, t = g >> 2;
    if (t < kt) codes[((nti * kt + t) * 64 + q * 16 + r) * 16 + l] = bad ? 0 : (uint8_t)q4_encode2(x0, x1, __uint_as_float((uint32_t)s << 23));
    if (l == 0) scales[((nti * ks + (t >> 2)) * 64 + q * 16 + r) * 4 + (t & 3)] = bad ? Q4_NAN : (uint8_t)s;
}
