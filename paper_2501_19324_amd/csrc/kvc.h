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
    int value_blocks;
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

// the value of lane K of the quad
template <int K> __device__ __forceinline__ uint32_t kvc_of_lane(uint32_t x) { return dpp_move<K * 0x55>(x); }
// One value of each lane of a quad, the lane's own number deciding which of four: lane l gets x[l] of lane K
template <int K> __device__ __forceinline__ uint32_t kvc_take(const uint32_t x[4], int l) {
    const uint32_t a = kvc_of_lane<K>(x[0]), b = kvc_of_lane<K>(x[1]), c = kvc_of_lane<K>(x[2]), d = kvc_of_lane<K>(x[3]);
    const uint32_t e = l & 1 ? b : a, f = l & 1 ? d : c;
    return l & 2 ? f : e;
}
// Values into their pages: a block takes 16 rows of a head (of several, where they are short), a quad of lanes G dims of four rows.  The four tokens whose values lie together in a page are mostly four
// rows that follow each other, at any place among the rows: the quad that has the first of them loads all four, one to a lane, exchanges, and stores a dim's four tokens at once.  Rows
// that are not among four such go value by value.
// Bound by bytes: 7937 rows of 28 heads of 128 and 4, bf16 (146 MB with queries and keys), 31 us, 36 with every value loaded and stored by itself; of 16 heads of 64 (98 MB) 24.
template <typename C, int HD> struct KvcValueBlock {
    static constexpr int ROWS = 16, G = sizeof(C) == 2 ? 8 : 4, QUADS = HD / G, HEADS = QUADS >= 16 ? 1 : 16 / QUADS;      // quads of a row's values; heads of a block
};
template <typename T, typename C, int HD> __device__ __forceinline__ void kvc_write_values(const KvcRows& a, int block) {
    typedef KvcLayout<C, HD> L;
    typedef KvcValueBlock<C, HD> B;
    constexpr int G = B::G, R = B::ROWS;
    __shared__ int s_seq[R + 6], s_slot[R + 6], s_page[R];  // of the rows from r0 - 3 on; of those from r0 on
    __shared__ bool s_full[R + 3];                          // the row is the first of four (rows from r0 - 3 on)
    const int t = threadIdx.x, l = t & 3, parts = (a.k.n + B::HEADS - 1) / B::HEADS, r0 = block / parts * R, h0 = block % parts * B::HEADS;
    if (t < R + 6) {
        const int r = r0 - 3 + t;
        const bool is = r >= 0 && r < a.rows;
        s_seq[t] = is ? a.seq[r] : -1;
        s_slot[t] = is ? a.slot[r] : -1;
    }
    __syncthreads();
    if (t < R + 3) {
        const int slot = s_slot[t], seq = s_seq[t];
        bool full = slot >= 0 && (slot & 3) == 0;
#pragma unroll
        for (int e = 1; e < 4; ++e) full &= (s_seq[t + e] == seq) & (s_slot[t + e] == slot + e);
        s_full[t] = full;
        if (t >= 3) {
            int id = -1;
            if ((unsigned)seq < (unsigned)a.c.batch && slot >= 0 && slot < a.c.max_pages * KVC_PAGE) id = a.c.table[(int64_t)seq * a.c.max_pages + slot / KVC_PAGE];
            s_page[t - 3] = (unsigned)id < (unsigned)a.c.n_pages ? id : -1;
        }
    }
    __syncthreads();
    for (int quad = t >> 2; quad < 4 * B::QUADS * B::HEADS; quad += 64) {
        const int s = quad % B::QUADS, i0 = quad / B::QUADS % 4 * 4, h = h0 + quad / B::QUADS / 4;
        if (h >= a.k.n) continue;
        const T* x = static_cast<const T*>(a.v) + h * a.v_head + s * G;
        C* pool = reinterpret_cast<C*>(a.c.pool) + (int64_t)h * L::BLOCK;
        auto entry = [&](int i) { return pool + (int64_t)s_page[i] * a.c.hkv * L::BLOCK; };
        int first = -1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = i0 + e, slot = s_slot[i + 3];
            if (s_full[i + 3]) first = i;
            else if (s_page[i] >= 0 && !((slot & 3) && s_full[i + 3 - (slot & 3)])) {
#pragma unroll
                for (int d = 0; d < G / 4; ++d)
                    st1(entry(i) + L::value(slot % KVC_PAGE, s * G + l * (G / 4) + d), ld1(x + (int64_t)(r0 + i) * a.v_row + l * (G / 4) + d));
            }
        }
        if (first < 0 || s_page[first] < 0) continue;       // (the same for the whole quad)
        x += (int64_t)(r0 + first + l) * a.v_row;
        C* dst = entry(first) + L::value(s_slot[first + 3] % KVC_PAGE, s * G + l);
        if constexpr (sizeof(C) == 2) {                     // dims l and 4 + l
            float y[8];
            kvc_load8(x, y);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint32_t p = f2bf2(y[4 * b], y[4 * b + 1]), q = f2bf2(y[4 * b + 2], y[4 * b + 3]);
                // (both are moved before one is chosen: a move in a branch finds the lanes of the other branch switched off)
                const uint32_t p0 = kvc_of_lane<0>(p), p1 = kvc_of_lane<1>(p), p2 = kvc_of_lane<2>(p), p3 = kvc_of_lane<3>(p);
                const uint32_t q0 = kvc_of_lane<0>(q), q1 = kvc_of_lane<1>(q), q2 = kvc_of_lane<2>(q), q3 = kvc_of_lane<3>(q);
                const uint32_t t0 = l & 2 ? q0 : p0, t1 = l & 2 ? q1 : p1, t2 = l & 2 ? q2 : p2, t3 = l & 2 ? q3 : p3;
                const uint32_t pick = l & 1 ? 0x07060302u : 0x05040100u;
                *reinterpret_cast<u32x2_t*>(dst + 4 * b * L::E) = u32x2_t{__builtin_amdgcn_perm(t1, t0, pick), __builtin_amdgcn_perm(t3, t2, pick)};
            }
        } else {
            const f32x4_t y = *reinterpret_cast<const f32x4_any_t*>(x);
            const uint32_t z[4] = {__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])};
            *reinterpret_cast<u32x4_t*>(dst) = u32x4_t{kvc_take<0>(z, l), kvc_take<1>(z, l), kvc_take<2>(z, l), kvc_take<3>(z, l)};
        }
    }
}

// HD / 16 lanes take a head, 16 of its dims each: eight pairs where they are interleaved, (2 i, 2 i + 1), or in halves, (i, i + rot / 2) and, behind the rotation, (rot + j, rot + rest / 2 + j),
// as two runs of eight neighbours, read and written 16 bytes at a time.  Halves of a rotation of which 16 is no divisor (SPLIT) take 16 neighbours and exchange
// with the lanes that have their partners through LDS (8192 rows of 32 heads, bf16: 35 us, 85 with pairs read one by one).
// A block takes 16 * 256 / HD neighbouring (row, head) and forms the angles of its rows once, one to a thread, for all their heads.  The turns position * freq / 2 pi are
// formed and reduced in 64 bits: in 32 an angle at position 10^5 is off by some 2^-8.  Norm and rotation are computed in fp32 and rounded once.
// Bound by bytes: 8192 rows of 32 heads, bf16 (134 MB), 23.8 us, 5.6 TB/s; 7937 rows of 72 heads, fp32 (585 MB), 116 us, 5.0 TB/s; 16 prompts of 480 .. 512 tokens, 72B heads, fp32 into a bf16 cache (618 MB),
// 127 us, 4.9 TB/s.  Single tokens of 64 sequences: 4.6 us, a chain of latencies (row numbers, table, stores).
template <typename T, typename C, int HD, bool INTERLEAVED, bool SPLIT, bool CACHE>
__global__ __launch_bounds__(256) void kvc_rows_kernel(KvcRows a) {
    constexpr int LANES = HD / 16, ITEMS = 256 / LANES, P = HD / 2, LINE = HD + LANES;
    typedef KvcLayout<C, HD> L;
    __shared__ float2 turn[ITEMS * P];
    __shared__ float lines[SPLIT ? ITEMS * LINE : 1];       // 17 words to a lane's 16 dims: lanes on different banks
    const int heads = a.q.n + a.k.n, total = a.rows * heads;
    // Blocks that write values are spread evenly among the others, so that a row's pieces are read at about one time.
    int block = blockIdx.x;
    if (CACHE) {
        const int before = (int)((uint64_t)block * a.value_blocks / gridDim.x), after = (int)((uint64_t)(block + 1) * a.value_blocks / gridDim.x);
        if (after > before) {
            kvc_write_values<T, C, HD>(a, before);
            return;
        }
        block -= before;
    }
    const int item0 = block * ITEMS, item = item0 + threadIdx.x / LANES, part = threadIdx.x % LANES;
    const bool there = item < total;
    const int row = (there ? item : total - 1) / heads;
    int h = (there ? item : total - 1) - row * heads;
    const bool is_q = h < a.q.n;
    if (!is_q) h -= a.q.n;
    const T* x = is_q ? static_cast<const T*>(a.q.x) + row * a.q.row + h * a.q.head : static_cast<const T*>(a.k.x) + row * a.k.row + h * a.k.head;
    const int half = a.rot_dim / 2;
    int d0 = part * 16, d1 = d0 + 8;
    if (!INTERLEAVED && !SPLIT) {
        const int i = part * 8, rest = (HD - a.rot_dim) / 2;
        if (i < half) d0 = i, d1 = i + half;
        else d0 = half + i, d1 = d0 + rest;
    }
    float y[16];                                            // the run from d0, the run from d1
    kvc_load8(x + d0, y);
    kvc_load8(x + d1, y + 8);
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
    const T* weight = static_cast<const T*>(is_q ? a.q.weight : a.k.weight);
    if (weight) {
        const float r = kvc_norm<HD>(y, a.eps);
        float w[16];
        kvc_load8(weight + d0, w);
        kvc_load8(weight + d1, w + 8);
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = y[i] * r * w[i];
    }
    if (a.rot_dim) {
        const float2* t = turn + (row - item0 / heads) * P;
        if constexpr (SPLIT) {
            float* line = lines + threadIdx.x / LANES * LINE;
#pragma unroll
            for (int i = 0; i < 16; ++i) line[part * 17 + i] = y[i];
            wave_order();                                   // (the lanes of a head lie in one wave)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int d = d0 + i, other = d < half ? d + half : d - half;
                if (d >= a.rot_dim) continue;               // what does not turn stays as it is, infinities too
                const float2 cs = t[d < half ? d : other];
                const float o = line[other + other / 16];
                y[i] = d < half ? y[i] * cs.x - o * cs.y : y[i] * cs.x + o * cs.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float &u = y[INTERLEAVED ? 2 * i : i], &w = y[INTERLEAVED ? 2 * i + 1 : 8 + i];
                const float2 cs = t[part * 8 + i];
                const float u_ = u * cs.x - w * cs.y, w_ = w * cs.x + u * cs.y;
                if (part * 8 + i < half) u = u_, w = w_;
            }
        }
    }
    if (!CACHE || is_q) {
        T* out = is_q ? static_cast<T*>(a.q.out) + row * a.q.out_row + h * a.q.out_head : static_cast<T*>(a.k.out) + row * a.k.out_row + h * a.k.out_head;
        kvc_store8(out + d0, y);
        kvc_store8(out + d1, y + 8);
        return;
    }
    if (!entry) return;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int d = r ? d1 : d0;
        if (sizeof(C) == 2) kvc_store8(entry + L::key(slot, d), y + 8 * r);
        else {
            *reinterpret_cast<f32x4_t*>(entry + L::key(slot, d)) = f32x4_t{y[8 * r], y[8 * r + 1], y[8 * r + 2], y[8 * r + 3]};
            *reinterpret_cast<f32x4_t*>(entry + L::key(slot, d + 4)) = f32x4_t{y[8 * r + 4], y[8 * r + 5], y[8 * r + 6], y[8 * r + 7]};
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
