// A paged KV cache in bf16 or fp32: its layout, norms and rotation of queries and keys, entries in and out.
//
// Page [kv head][2][16 HD] values, 16 tokens, E values in 16 bytes.  Keys [HD / 4E][4][16 tokens][E]: lane l = 16 c + t of a wave loads 16 bytes, the A operand of
// the products q.K (rows: tokens).  Values [HD / 4E][4][16 dims][E / 4][4 tokens]: lane l = 16 c + d loads for the tokens 4 c .. + 3 the dims d and, in bf16, d + 16,
// the A operands of V^T P^T (rows: dims), whose contraction order (tokens 4 c + i) is the one in which the matrix instruction leaves the scores.  So every load of a wave
// is 1 KB of consecutive memory and an operand as it is.
#pragma once
#include "q4.h"

#define KVC_PAGE 16

struct KvcCache {
    char* pool;
    const int* table;
    const int* kv_len;
    int n_pages, hkv, batch, max_pages;
};
template <typename C, int HD> struct KvcLayout {
    static constexpr int E = 16 / sizeof(C), N = HD / (4 * E);      // values in 16 bytes; 16-byte loads of a wave for the keys (or values) of a page
    static constexpr int BLOCK = 2 * KVC_PAGE * HD;                // values of a (page, head)
    __device__ static __forceinline__ int key(int t, int d) { return d / E * (16 * E) + t * E + d % E; }
    __device__ static __forceinline__ int value(int t, int d) { return KVC_PAGE * HD + d / (4 * E) * (64 * E) + t / 4 * (16 * E) + d % 16 * E + d % (4 * E) / 16 * 4 + t % 4; }
};
// address of a (page, head) block; a slot that the table has no page of the pool for gives null
template <typename C, int HD> __device__ __forceinline__ C* kvc_entry(const KvcCache& c, int seq, int slot, int head) {
    if ((unsigned)seq >= (unsigned)c.batch || slot < 0 || slot >= c.max_pages * KVC_PAGE) return nullptr;
    const int id = c.table[(int64_t)seq * c.max_pages + slot / KVC_PAGE];
    return (unsigned)id < (unsigned)c.n_pages ? reinterpret_cast<C*>(c.pool) + ((int64_t)id * c.hkv + head) * KvcLayout<C, HD>::BLOCK : nullptr;
}

// eight consecutive values at any address of their type
__device__ __forceinline__ void kvc_load8(const bf16_t* p, float o[8]) {
    const u32x4_t r = *reinterpret_cast<const u32x4_any_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[2 * i] = __uint_as_float(r[i] << 16), o[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
}
__device__ __forceinline__ void kvc_load8(const float* p, float o[8]) {
    const f32x4_t a = *reinterpret_cast<const f32x4_any_t*>(p), b = *reinterpret_cast<const f32x4_any_t*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = a[i], o[4 + i] = b[i];
}
__device__ __forceinline__ void kvc_store8(bf16_t* p, const float v[8]) {
    *reinterpret_cast<u32x4_any_t*>(p) = u32x4_t{f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7])};
}
__device__ __forceinline__ void kvc_store8(float* p, const float v[8]) {
    *reinterpret_cast<f32x4_any_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_any_t*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
}

// ---- norms and rotation, and entries in
struct KvcHeads { const void* x; void* out; const void* weight; int64_t row, head, out_row, out_head; int n; };
struct KvcRows {
    KvcHeads q, k;          // n = 0: none; k.out is not used where keys go into the cache
    const void* v;          // values [rows][k.n], or null: no cache
    int64_t v_row, v_head;
    const int *position, *seq, *slot;
    const double* freq;
    int rot_dim;            // 0: no rotation
    float magnitude, eps;
    int rows;
    KvcCache c;
};

// Sum over the LANES neighbouring lanes of a head
template <int LANES> __device__ __forceinline__ float kvc_head_sum(float v) {
    v += __uint_as_float(dpp_move<0xB1>(__float_as_uint(v)));
    if (LANES >= 4) v += __uint_as_float(dpp_move<0x4E>(__float_as_uint(v)));
    if (LANES >= 8) v += __uint_as_float(dpp_move<0x141>(__float_as_uint(v)));
    if (LANES >= 16) v += __uint_as_float(dpp_move<0x140>(__float_as_uint(v)));
    return v;
}
// 1 / sqrt(mean of squares + eps).  Where the squares leave the range of fp32, or are too small for all of their bits beside so small an eps, x is scaled
// by a power of two.
template <int HD> __device__ __forceinline__ float kvc_norm(float x[16], float eps) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s = __builtin_fmaf(x[i], x[i], s);
    s = kvc_head_sum<HD / 16>(s);
    if (s < 0x1p126f && (s > 0x1p-90f || eps > 0x1p-90f)) return rsqrtf(__builtin_fmaf(s, 1.f / HD, eps));
    const float by = s < 1.f ? 0x1p70f : 0x1p-70f;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        x[i] *= by;
        s = __builtin_fmaf(x[i], x[i], s);
    }
    s = kvc_head_sum<HD / 16>(s);
    return rsqrtf(__builtin_fmaf(s, 1.f / HD, eps * by * by));
}

// HD / 16 lanes take a head, eight of its pairs each: in halves the pair i is (i, i + rot / 2) and, behind the rotation, (rot + j, rot + rest / 2 + j); interleaved it is
// (2 i, 2 i + 1).  WIDE: a lane's pairs are two runs of eight neighbours, read and written 16 bytes at a time; halves of a rotation of which 16 is no divisor go value by value.
// A block takes 16 * 256 / HD neighbouring (row, head) and forms the angles of its rows once, one to a thread, for all their heads.  The turns position * freq / 2 pi are
// formed and reduced in 64 bits: in 32 an angle at position 10^5 is off by some 2^-8.
template <typename T, typename C, int HD, bool INTERLEAVED, bool WIDE, bool CACHE>
__global__ __launch_bounds__(256) void kvc_rows_kernel(KvcRows a) {
    constexpr int LANES = HD / 16, ITEMS = 256 / LANES, P = HD / 2;
    typedef KvcLayout<C, HD> L;
    __shared__ float2 turn[ITEMS * P];
    const int heads = a.q.n + a.k.n * (CACHE ? 2 : 1), total = a.rows * heads;
    const int item0 = blockIdx.x * ITEMS, item = item0 + threadIdx.x / LANES, part = threadIdx.x % LANES;
    const bool there = item < total;
    const int row = (there ? item : total - 1) / heads;
    int h = (there ? item : total - 1) - row * heads;
    const bool is_q = h < a.q.n, is_v = CACHE && h >= a.q.n + a.k.n;
    if (!is_q) h -= is_v ? a.q.n + a.k.n : a.q.n;
    const T* x = is_q ? static_cast<const T*>(a.q.x) + row * a.q.row + h * a.q.head
                      : is_v ? static_cast<const T*>(a.v) + row * a.v_row + h * a.v_head : static_cast<const T*>(a.k.x) + row * a.k.row + h * a.k.head;
    // places of the lane's pairs
    const int half = a.rot_dim / 2, rest = (HD - a.rot_dim) / 2;
    auto place = [&](int i, int& first, int& second) {
        if (INTERLEAVED) first = 2 * i, second = 2 * i + 1;
        else if (i < half) first = i, second = i + half;
        else first = a.rot_dim + i - half, second = first + rest;
    };
    int d0, d1;
    if (INTERLEAVED || is_v) d0 = part * 16, d1 = d0 + 8;
    else place(part * 8, d0, d1);
    float y[16];                                            // the run from d0, the run from d1; value by value: pair by pair
    if (WIDE || is_v) {
        kvc_load8(x + d0, y);
        kvc_load8(x + d1, y + 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int p, q;
            place(part * 8 + i, p, q);
            y[i] = ld1(x + p);
            y[8 + i] = ld1(x + q);
        }
    }
    C* entry = nullptr;
    int slot = 0;
    if (CACHE && !is_q) {
        slot = a.slot[row];
        entry = kvc_entry<C, HD>(a.c, a.seq[row], slot, h);
        slot %= KVC_PAGE;
    }
    if (a.rot_dim) {
        const int row0 = item0 / heads, rows = min(item0 + ITEMS - 1, total - 1) / heads - row0 + 1;
        for (int i = threadIdx.x; i < rows * P; i += 256) {
            const int p = i % P;
            float s = 0.f, c = 1.f;
            if (p < half) {
                const double turns = a.position[row0 + i / P] * (a.freq[p] * 0.15915494309189533577);
                sincospif((float)(2. * (turns - __builtin_rint(turns))), &s, &c);
                s *= a.magnitude;
                c *= a.magnitude;
            }
            turn[i] = make_float2(c, s);
        }
        __syncthreads();
    }
    if (!there) return;
    if (!is_v) {
        const T* weight = static_cast<const T*>(is_q ? a.q.weight : a.k.weight);
        if (weight) {
            const float r = kvc_norm<HD>(y, a.eps);
            float w[16];
            if (WIDE) {
                kvc_load8(weight + d0, w);
                kvc_load8(weight + d1, w + 8);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    int p, q;
                    place(part * 8 + i, p, q);
                    w[i] = ld1(weight + p);
                    w[8 + i] = ld1(weight + q);
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = y[i] * r * w[i];
        }
        if (a.rot_dim) {
            const float2* t = turn + (row - item0 / heads) * P + part * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float &u = y[INTERLEAVED ? 2 * i : i], &w = y[INTERLEAVED ? 2 * i + 1 : 8 + i];
                const float2 cs = t[i];
                const float u_ = u * cs.x - w * cs.y, w_ = w * cs.x + u * cs.y;
                // what does not turn stays as it is, infinities too
                if (part * 8 + i < half) u = u_, w = w_;
            }
        }
    }
    if (!CACHE || is_q) {
        T* out = is_q ? static_cast<T*>(a.q.out) + row * a.q.out_row + h * a.q.out_head : static_cast<T*>(a.k.out) + row * a.k.out_row + h * a.k.out_head;
        if (WIDE) {
            kvc_store8(out + d0, y);
            kvc_store8(out + d1, y + 8);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                int p, q;
                place(part * 8 + i, p, q);
                st1(out + p, y[i]);
                st1(out + q, y[8 + i]);
            }
        }
        return;
    }
    if (!entry) return;
    if (is_v) {
#pragma unroll
        for (int i = 0; i < 16; ++i) st1(entry + L::value(slot, part * 16 + i), y[i]);
    } else if (WIDE) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int d = r ? d1 : d0;
            if (sizeof(C) == 2) kvc_store8(entry + L::key(slot, d), y + 8 * r);
            else {
                *reinterpret_cast<f32x4_t*>(entry + L::key(slot, d)) = f32x4_t{y[8 * r], y[8 * r + 1], y[8 * r + 2], y[8 * r + 3]};
                *reinterpret_cast<f32x4_t*>(entry + L::key(slot, d + 4)) = f32x4_t{y[8 * r + 4], y[8 * r + 5], y[8 * r + 6], y[8 * r + 7]};
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int p, q;
            place(part * 8 + i, p, q);
            st1(entry + L::key(slot, p), y[i]);
            st1(entry + L::key(slot, q), y[8 + i]);
        }
    }
}

// ---- entries out: eight values of a key or a value to a lane
template <typename C, int HD>
__global__ __launch_bounds__(256) void kvc_read_kernel(KvcCache c, const int* __restrict__ seq, const int* __restrict__ slot, int rows, C* __restrict__ k, C* __restrict__ v) {
    typedef KvcLayout<C, HD> L;
    constexpr int LANES = HD / 8;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, item = id / LANES;
    const int d = (int)(id % LANES) * 8, head = (int)(item / 2 % c.hkv);
    const int64_t row = item / 2 / c.hkv;
    const bool is_v = item & 1;
    if (row >= rows) return;
    const int s = slot[row];
    const C* entry = kvc_entry<C, HD>(c, seq[row], s, head);
    C o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = entry ? entry[is_v ? L::value(s % KVC_PAGE, d + i) : L::key(s % KVC_PAGE, d + i)] : C{};
    C* dst = (is_v ? v : k) + (row * c.hkv + head) * HD + d;
#pragma unroll
    for (int i = 0; i < 8 / L::E; ++i) {
        u32x4_t w;
        __builtin_memcpy(&w, o + i * L::E, 16);
        reinterpret_cast<u32x4_t*>(dst)[i] = w;
    }
}
