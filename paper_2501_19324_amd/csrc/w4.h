// Products with 4-bit weights: y[r][n] = sum_k x[r][k] W[n][k].
//
// A tile is 16 rows of W x 128 columns, 1 KB: lane l = 16 q + r of a wave holds the 16 bytes of row r, group q (32 columns, one scale),
// so a load of a wave reads 1 KB of consecutive memory and every lane needs one scale byte per tile.  The four dwords of a lane are the A
// operands of four 16x16x32 matrix instructions: instruction j contracts over the columns 32 q + 8 j .. + 7 of every group q, and x is
// laid out in the same order (the order of a contraction does not matter).
#pragma once
#include "q4.h"

struct W4Args {
    const u32x4_t* codes;
    const uint32_t* scales;
    int n, k, nt, kt, ks;
    const void* x;
    int64_t ldx;
    int rows;
    void* y;
    int64_t ldy;
    float* part;        // partial sums [split][rows][n], null: the block writes y
    int tiles, splits;  // tiles of 128 columns per split
};
template <typename T> constexpr int w4_planes = sizeof(T) == 4 ? 3 : 1;

// Eight values of x from column k0 on.  WIDE (k >= 8): one or two loads of 16 bytes wherever the row starts (the memory takes them at any address of the type), the
// last ones of a row moved back to end with it; w4_tail then brings their values to their places.  Else value by value.
// (Rows of an odd length loaded value by value, the rule before: 256 rows, 5000 x 5001: 54 us, now 30; 16 rows: 22, now 9.)
template <typename T> struct W4Piece;
template <> struct W4Piece<bf16_t> { u32x4_t v; };
template <> struct W4Piece<float> { f32x4_t a, b; };
template <bool WIDE> __device__ __forceinline__ void w4_load(const bf16_t* row, int k0, int k, W4Piece<bf16_t>& o) {
    if constexpr (WIDE) {
        o.v = *reinterpret_cast<const u32x4_any_t*>(row + min(k0, k - 8));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = row[min(k0 + 2 * i, k - 1)].v, hi = row[min(k0 + 2 * i + 1, k - 1)].v;
            o.v[i] = (k0 + 2 * i < k ? lo : 0u) | (k0 + 2 * i + 1 < k ? hi << 16 : 0u);
        }
    }
}
template <bool WIDE> __device__ __forceinline__ void w4_load(const float* row, int k0, int k, W4Piece<float>& o) {
    if constexpr (WIDE) {
        o.a = *reinterpret_cast<const f32x4_any_t*>(row + min(k0, k - 8));
        o.b = *reinterpret_cast<const f32x4_any_t*>(row + min(k0, k - 8) + 4);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p = row[min(k0 + i, k - 1)], q = row[min(k0 + 4 + i, k - 1)];
            o.a[i] = k0 + i < k ? p : 0.f;
            o.b[i] = k0 + 4 + i < k ? q : 0.f;
        }
    }
}
// the piece `by` values further on (0 .. 8 or more), zeros behind it
__device__ __forceinline__ void w4_tail(W4Piece<bf16_t>& x, int by) {
    uint64_t lo = u64_of(x.v[0], x.v[1]), hi = u64_of(x.v[2], x.v[3]);
    const int bits = 16 * (by & 3);
    if (by & 4) lo = hi, hi = 0;
    if (bits) lo = (lo >> bits) | (hi << (64 - bits)), hi >>= bits;
    if (by >= 8) lo = hi = 0;
    x.v = u32x4_t{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
__device__ __forceinline__ void w4_tail(W4Piece<float>& x, int by) {
    float v[8] = {x.a[0], x.a[1], x.a[2], x.a[3], x.b[0], x.b[1], x.b[2], x.b[3]};
#pragma unroll
    for (int s = 1; s < 8; s *= 2)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = by & s ? (i + s < 8 ? v[i + s] : 0.f) : v[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = by >= 8 ? 0.f : v[i];
    x.a = f32x4_t{v[0], v[1], v[2], v[3]};
    x.b = f32x4_t{v[4], v[5], v[6], v[7]};
}
// the piece as operands, one per plane, `stride` vectors apart
__device__ __forceinline__ void w4_put(const W4Piece<bf16_t>& x, u32x4_t* at, int) { *at = x.v; }
__device__ __forceinline__ void w4_put(const W4Piece<float>& x, u32x4_t* at, int stride) {
    const float v[8] = {x.a[0], x.a[1], x.a[2], x.a[3], x.b[0], x.b[1], x.b[2], x.b[3]};
    u32x4_t o[3];
    q4_operand<3>(v, o);
    at[0] = o[0];
    at[stride] = o[1];
    at[2 * stride] = o[2];
}
template <int NT> struct W4Tile { u32x4_t w[NT]; uint32_t s[NT]; };
template <int NT> __device__ __forceinline__ void w4_load(const W4Args& a, int n0, int t, int lane, W4Tile<NT>& o) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int n = min(n0 + i, a.nt - 1);
        o.w[i] = a.codes[((int64_t)n * a.kt + t) * 64 + lane];
        o.s[i] = a.scales[((int64_t)n * a.ks + (t >> 2)) * 64 + lane];
    }
}
// four results (rows of W n .. n + 3) of row `row` of x.  The splits' rows are padded to whole vectors.
__host__ __device__ inline int w4_padded(int n) { return (n + 3) & ~3; }
template <typename T> __device__ __forceinline__ void w4_store(const W4Args& a, int split, int row, int n, f32x4_t s) {
    if (row >= a.rows || n >= a.n) return;
    if (a.part) {
        *reinterpret_cast<f32x4_t*>(a.part + ((int64_t)split * a.rows + row) * w4_padded(a.n) + n) = s;
        return;
    }
    T* o = static_cast<T*>(a.y) + row * a.ldy + n;
    if (n + 3 < a.n) {
        if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2_any_t*>(o) = u32x2_t{f2bf2(s[0], s[1]), f2bf2(s[2], s[3])};
        else *reinterpret_cast<f32x4_any_t*>(o) = s;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) if (n + i < a.n) st1(o + i, s[i]);
    }
}

// Up to 16 rows of x (XL * 4 of them).  A block owns NT tiles of rows of W, its waves share the columns.  A wave brings its part of x into operand order through
// LDS of its own: no barrier until the waves' sums are added, in the order of the waves.  Columns of the matrix instruction beyond the rows of x
// repeat some row; nobody reads their results.
// Bound by the weights' bytes: 7B gate and up, one row: 72 MB in 13.2 us with launch, 5.4 TB/s; what x costs is read once per block, from L2.
// waves that a block may have: their parts of x, and their sums, share 64 KB (fp32 with up to 16 rows: 96 KB)
template <typename T, int XL> constexpr int w4_few_waves = w4_planes<T> == 3 && XL == 4 ? 8 : 16;
template <typename T, int NT, int XL, bool WIDE>
__global__ __launch_bounds__((64 * w4_few_waves<T, XL>)) void w4_few_kernel(W4Args a) {
    constexpr int P = w4_planes<T>, WAVES = w4_few_waves<T, XL>, XR = XL * 4, PLANE = 16 * XR;
    __shared__ u32x4_t lds[WAVES * (P * PLANE > NT * 64 ? P * PLANE : NT * 64)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * NT;
    // the tiles of columns, dealt to the waves in runs
    const int t0 = (int)((int64_t)a.kt * wave / waves), t1 = (int)((int64_t)a.kt * (wave + 1) / waves);
    u32x4_t* stage = lds + wave * P * PLANE;                // [plane][j][q][row]
    const T* row[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) row[i] = static_cast<const T*>(a.x) + (int64_t)min(i * 4 + (lane >> 4), a.rows - 1) * a.ldx;
    const int k8 = lane & 15;                               // the piece of a row's 128 columns; operand k8 % 4 of group k8 / 4
    f32x4_t acc[NT] = {};
    W4Tile<NT> w[2];
    W4Piece<T> x[2][XL];
    auto load = [&](int t, W4Tile<NT>& w_, W4Piece<T>(&x_)[XL]) {
        t = min(t, t1 - 1);
#pragma unroll
        for (int i = 0; i < XL; ++i) w4_load<WIDE>(row[i], t * 128 + k8 * 8, a.k, x_[i]);
        w4_load<NT>(a, n0, t, lane, w_);
    };
    auto work = [&](int t, const W4Tile<NT>& w_, W4Piece<T>(&x_)[XL]) {
        if (WIDE && t * 128 + 128 > a.k)
#pragma unroll
            for (int i = 0; i < XL; ++i) w4_tail(x_[i], max(0, t * 128 + k8 * 8 - (a.k - 8)));
        wave_order();                                       // behind the reads of the tile before
#pragma unroll
        for (int i = 0; i < XL; ++i) w4_put(x_[i], stage + ((k8 & 3) * 4 + (k8 >> 2)) * XR + i * 4 + (lane >> 4), PLANE);
        wave_order();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4_t b[P];
#pragma unroll
            for (int p = 0; p < P; ++p) b[p] = stage[p * PLANE + (j * 4 + (lane >> 4)) * XR + (lane & (XR - 1))];
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const u32x4_t m = q4_decode8(w_.w[i][j], (w_.s[i] >> (8 * (t & 3))) << 23);
#pragma unroll
                for (int p = 0; p < P; ++p) acc[i] = q4_mfma(m, b[p], acc[i]);
            }
        }
    };
    if (t0 < t1) {
        load(t0, w[0], x[0]);
        for (int t = t0;;) {
            load(t + 1, w[1], x[1]);
            work(t, w[0], x[0]);
            if (++t >= t1) break;
            load(t + 1, w[0], x[0]);
            work(t, w[1], x[1]);
            if (++t >= t1) break;
        }
    }
    __syncthreads();                                        // the stages become the sums' place
    f32x4_t* sums = reinterpret_cast<f32x4_t*>(lds);
#pragma unroll
    for (int i = 0; i < NT; ++i) sums[(wave * NT + i) * 64 + lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < NT; i += waves) {
        f32x4_t s = sums[i * 64 + lane];
        for (int v = 1; v < waves; ++v) s += sums[(v * NT + i) * 64 + lane];
        w4_store<T>(a, 0, lane & 15, (n0 + i) * 16 + (lane >> 4) * 4, s);
    }
}

// More rows: a block of four waves owns 16 tiles of rows of W, four to a wave, and XT tiles of rows of x.  x goes through LDS in operand order, shared by the
// waves; a wave decodes its own weights, which stay in registers for XT products each.  Splits start at multiples of four tiles of columns, so that
// a word of scale bytes serves one turn of the loop.
//  - Loads run three tiles ahead: a tile is 0.4 us of matrix work, less than a load takes.
//  - 16 lanes load 256 consecutive bytes of one row of x (with 16 rows x 64 bytes the loads of x alone took 22 of 51 us at 64 rows of the 7B gate and up product).
//    They write to 16 different operands: slot r of operand (j, q) is kept at r ^ (4 q + j), or all of them would hit the same banks.
//  - Splits are the fastest index of the grid: with eight of them an XCD's L2 sees one part of x (256 rows, 7B down: 90 -> 70 us).  Then come the blocks of rows
//    of x, which share their weights (256 rows, 7B gate and up: 99 -> 80 us).
// 256 rows, 3584 x 18944: 45 us, 770 TFLOP/s, and 5 us for the sums; 37888 x 3584: 80 us, 870 TFLOP/s.  A plain bf16 product of 8192^3 reaches 1220 here.  Bound by
// the products and the reads of LDS in turn: a wave takes 25 clocks for a product instead of 16, at the 1.8 GHz that such a load leaves; a second block per CU
// changes little, reading the operands of a group ahead or twice the rows of W per wave nothing.
template <typename T, int XT, bool WIDE>
__global__ __launch_bounds__(256) void w4_many_kernel(W4Args a) {
    constexpr int P = w4_planes<T>, NT = 4, DW = 4, DX = 4;
    __shared__ u32x4_t lds[2][P][XT * 256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int split = blockIdx.x % a.splits, rest = blockIdx.x / a.splits, row_blocks = (a.rows + XT * 16 - 1) / (XT * 16);
    const int n0 = (rest / row_blocks * 4 + wave) * NT, r0 = rest % row_blocks * XT * 16;
    const int t0 = split * a.tiles, t1 = min(a.kt, t0 + a.tiles);
    f32x4_t acc[NT][XT] = {};
    u32x4_t w[DW][NT];
    uint32_t scale[2][NT];
    W4Piece<T> x[DX][XT];
    // piece i of a thread: row 16 i + tid / 16 of the block's, columns 8 (tid % 16) of the tile's 128
    const int k8 = tid & 15, slot = (tid >> 4) ^ ((k8 >> 2) * 4 + (k8 & 3));
    const T* row[XT];
#pragma unroll
    for (int i = 0; i < XT; ++i) row[i] = static_cast<const T*>(a.x) + (int64_t)min(r0 + i * 16 + (tid >> 4), a.rows - 1) * a.ldx;
    const u32x4_t* codes[NT];
    const uint32_t* scales[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int64_t n = min(n0 + i, a.nt - 1);
        codes[i] = a.codes + n * a.kt * 64;
        scales[i] = a.scales + n * a.ks * 64;
    }
    auto load_x = [&](int t, W4Piece<T>(&x_)[XT]) {
        t = min(t, t1 - 1);
#pragma unroll
        for (int i = 0; i < XT; ++i) w4_load<WIDE>(row[i], t * 128 + k8 * 8, a.k, x_[i]);
    };
    auto put_x = [&](int t, W4Piece<T>(&x_)[XT], int buf) {
        if (WIDE && t < t1 && t * 128 + 128 > a.k)
#pragma unroll
            for (int i = 0; i < XT; ++i) w4_tail(x_[i], max(0, t * 128 + k8 * 8 - (a.k - 8)));
#pragma unroll
        for (int i = 0; i < XT; ++i) w4_put(x_[i], &lds[buf][0][(i * 4 + (k8 & 3)) * 64 + (k8 >> 2) * 16 + slot], XT * 256);
    };
    auto load_w = [&](int t, u32x4_t(&w_)[NT]) {
        t = min(t, t1 - 1);
#pragma unroll
        for (int i = 0; i < NT; ++i) w_[i] = codes[i][t * 64 + lane];
    };
    auto load_s = [&](int t, uint32_t(&s_)[NT]) {
        t = min(t, t1 - 1) >> 2;
#pragma unroll
        for (int i = 0; i < NT; ++i) s_[i] = scales[i][t * 64 + lane];
    };
    const int q = lane >> 4, r = lane & 15;
    int place[4];                                           // where operand j keeps this lane's slot
#pragma unroll
    for (int j = 0; j < 4; ++j) place[j] = j * 64 + q * 16 + (r ^ (4 * q + j));
    auto work = [&](int shift, int buf, const u32x4_t(&w_)[NT], const uint32_t(&s_)[NT]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4_t m[NT], b[XT][P];
#pragma unroll
            for (int e = 0; e < XT; ++e)
#pragma unroll
                for (int p = 0; p < P; ++p) b[e][p] = lds[buf][p][e * 256 + place[j]];
#pragma unroll
            for (int i = 0; i < NT; ++i) m[i] = q4_decode8(w_[i][j], shift == 24 ? s_[i] >> 1 : s_[i] << (23 - shift));
#pragma unroll
            for (int e = 0; e < XT; ++e)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < NT; ++i) acc[i][e] = q4_mfma(m[i], b[e][p], acc[i][e]);
        }
    };
#pragma unroll
    for (int s = 0; s < DX; ++s) load_x(t0 + s, x[s]);
    load_s(t0, scale[0]);
#pragma unroll
    for (int s = 0; s < DW - 1; ++s) load_w(t0 + s, w[s]);
    put_x(t0, x[0], 0);
    __syncthreads();
    for (int t = t0; t < t1; t += 2 * DW) {                 // two turns: the scales have two buffers
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            load_s(t + (h + 1) * DW, scale[1 - h]);
#pragma unroll
            for (int s = 0; s < DW; ++s) {
                const int u = t + h * DW + s;
                load_x(u + DX, x[s % DX]);
                load_w(u + DW - 1, w[(s + DW - 1) % DW]);
                if (u < t1) {
                    put_x(u + 1, x[(s + 1) % DX], (s + 1) & 1);
                    work(8 * s, s & 1, w[s], scale[h]);
                }
                __syncthreads();
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < XT; ++e) w4_store<T>(a, split, r0 + e * 16 + (lane & 15), (n0 + i) * 16 + (lane >> 4) * 4, acc[i][e]);
}

// the splits' sums, in order; four results to a thread
template <typename T>
__global__ __launch_bounds__(256) void w4_sum_kernel(W4Args a) {
    const int quads = w4_padded(a.n) / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, total = (int64_t)a.rows * quads;
    if (id >= total) return;
    const f32x4_t* part = reinterpret_cast<const f32x4_t*>(a.part) + id;
    f32x4_t s = part[0];
#pragma unroll 4
    for (int i = 1; i < a.splits; ++i) s += part[i * total];
    W4Args y = a;
    y.part = nullptr;
    w4_store<T>(y, 0, (int)(id / quads), (int)(id % quads) * 4, s);
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
