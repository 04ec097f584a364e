// Attention over the paged bf16 / fp32 cache: chunks of new tokens or single ones, with a sliding window and first tokens that stay visible.
//
// A column is a (row, head of the group) of one (sequence, kv head): column c is row c / group, head c % group.  Scores are S^T[token][column] = K Q^T, what
// is gathered is O^T[dim][column] += V^T P^T, both in tiles of 16 x 16 whose accumulators hold row 4 (lane / 16) + i, column lane % 16: a column's probabilities leave the first product in
// the lanes in which the second one wants them, and only the maximum and the sum cross lanes.  One pass over the entries with a running maximum (base 2) and sum in fp32.
#pragma once
#include "kvc.h"

struct KvcAttn {
    KvcCache c;
    const void* q;
    int64_t q_row, q_head;
    const int* row_start;   // [batch + 1]; null: row b is sequence b's
    int total_rows, max_rows, heads, group;
    float factor2;          // |scale| * log2(e); never 0 or NaN
    bool negative;          // scale < 0: q changes its sign instead
    bool plain;             // scale is 0 or NaN: q is multiplied by it and factor2 is log2(e), so that -inf means "not seen" and nothing else
    float scale;
    void* out;
    int64_t o_row, o_head;
    float* lse;             // [rows][heads] or null
    int max_kv, window, sinks;
    int lists, tiles, tile_cols;    // (sequence, kv head) pairs, tiles of columns of each
    int split, splits;      // chunks to a part, most parts
    bool by_length;         // the blocks of the longest sequences go first
    float* part_o;          // [rows][heads][splits][hd], unnormalised
    float2* part_ml;        // [rows][heads][splits]: maximum (base 2), sum
};
// rows of sequence b: the first one and how many; entries it has
__device__ __forceinline__ void kvc_rows(const KvcAttn& a, int b, int& r0, int& count, int& n) {
    r0 = b;
    count = b < a.total_rows ? 1 : 0;
    if (a.row_start) {
        r0 = min(max(a.row_start[b], 0), a.total_rows);
        count = min(min(max(a.row_start[b + 1], r0), a.total_rows) - r0, a.max_rows);
    }
    n = min(min(max(a.c.kv_len[b], 0), a.max_kv), a.c.max_pages * KVC_PAGE);
}
// What the columns col0 .. col1 - 1 of a sequence see, in chunks of CH slots: the first `front` chunks (sinks), then those from `from` on, `chunks` in all.
struct KvcSpan {
    int end;                // no column sees a slot from here on
    int safe;               // every column sees the slots below (those of the window: from `low` on)
    int near, low;          // some column's window begins at `near`, every column's has begun at `low`
    int front, from, chunks;
};
template <int CH> __device__ __forceinline__ KvcSpan kvc_span(const KvcAttn& a, int count, int n, int col0, int col1) {
    KvcSpan s;
    const int p0 = n - count + col0 / a.group, p1 = n - count + (col1 - 1) / a.group;      // slots of the first and the last row
    s.end = max(p1 + 1, 0);
    s.safe = max(p0 + 1, 0);
    s.near = a.window ? max(p0 - a.window + 1, 0) : 0;
    s.low = a.window ? max(p1 - a.window + 1, 0) : 0;
    s.front = (min(min(a.sinks, s.near), s.end) + CH - 1) / CH;
    s.from = max(s.near / CH, s.front);
    s.chunks = s.front + max((s.end + CH - 1) / CH - s.from, 0);
    return s;
}
// first slot of the i-th chunk
template <int CH> __device__ __forceinline__ int kvc_slot(const KvcSpan& s, int i) { return (i < s.front ? i : i - s.front + s.from) * CH; }
__device__ __forceinline__ int kvc_parts(const KvcAttn& a, const KvcSpan& s) { return a.splits == 1 ? 1 : max(1, (s.chunks + a.split - 1) / a.split); }
// what one column sees
struct KvcColumn {
    int low, high, sinks;
    __device__ __forceinline__ bool sees(int slot) const { return slot < high && (slot >= low || slot < sinks); }
};
__device__ __forceinline__ KvcColumn kvc_column(const KvcAttn& a, int count, int n, int col, int cols) {
    const int p = n - count + col / a.group;
    return KvcColumn{a.window ? p - a.window + 1 : 0, col < cols ? p + 1 : 0, a.sinks};
}

// Sequences of unlike lengths make blocks of unlike times: the longest go first where the blocks do not all run at once.  The i-th sequence in that order, among
// every 64 together; the same for all lanes of a whole wave.
__device__ __forceinline__ int kvc_by_length(const KvcAttn& a, int i) {
    if (!a.by_length) return i;
    const int lane = threadIdx.x & 63, first = i & ~63;
    const int len = first + lane < a.c.batch ? min(max(a.c.kv_len[first + lane], 0), 1 << 24) : -1;
    const int key = len * 64 + 63 - lane;                   // no two alike
    int before = 0;
#pragma unroll 8
    for (int u = 0; u < 64; ++u) before += __builtin_amdgcn_readlane(key, u) > key;
    return first + __builtin_ctzll(__ballot(before == (i & 63)));
}

// The work of block `id`: a list, that is a (sequence, kv head), and a tile of its columns; the last tile first, which sees most.  Blocks go to the eight XCDs in turn: the
// tiles of a list, which read the same entries, are neighbours on one XCD and its L2.  Fewer than eight lists that divide eight share them out evenly.
__host__ __device__ __forceinline__ int kvc_blocks(int lists, int tiles) { return lists < 8 && 8 % lists == 0 ? (tiles + 8 / lists - 1) / (8 / lists) * 8 : (lists + 7) / 8 * 8 * tiles; }
__device__ __forceinline__ bool kvc_work(const KvcAttn& a, int id, int& list, int& tile) {
    const int xcd = id & 7, at = id >> 3;
    if (a.lists < 8 && 8 % a.lists == 0) {
        list = xcd % a.lists;
        tile = at * (8 / a.lists) + xcd / a.lists;
    } else {
        list = at / a.tiles * 8 + xcd;
        tile = at % a.tiles;
    }
    tile = a.tiles - 1 - tile;
    return list < a.lists && tile >= 0;
}

// Activations of type T over a cache of type C.
//   bf16 over bf16: operands as they are.  A probability enters the second product rounded to bf16, off by at most 2^-8 of itself like a
//     result that is rounded to bf16 itself; the sum it is divided by has all of its bits.
//   fp32 over bf16: q and probabilities in three bf16 parts, which hold all 24 bits; three matrix instructions each.  They are cut, not rounded, so that all have the sign of the whole, and
//     none is 0 where the whole is not (2^-30 of it stands in): an infinite key or value meets no 0 that would make a NaN of it.
//   fp32 over fp32: matrix instructions in fp32.
template <typename T, typename C, int HD> struct KvcMath {
    typedef KvcLayout<C, HD> L;
    static constexpr bool F32 = sizeof(C) == 4;
    static constexpr int N = L::N, PAGES = F32 ? 1 : 2, CH = PAGES * KVC_PAGE, PLANES = !F32 && sizeof(T) == 4 ? 3 : 1;
    struct Q { u32x4_t w[N][PLANES]; };
    struct Entries { u32x4_t w[PAGES][N]; };        // keys, or values, of a chunk

    // operands of a tile of 16 columns: column lane % 16, dims 4E j + E (lane / 16) ..
    static __device__ __forceinline__ void load_q(const KvcAttn& a, int r0, int head, int col, int cols, int lane, Q& q) {
        const int use = min(col, cols - 1);
        const T* src = static_cast<const T*>(a.q) + (int64_t)(r0 + use / a.group) * a.q_row + (int64_t)(head * a.group + use % a.group) * a.q_head + (lane >> 4) * L::E;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float x[8];
            if constexpr (F32) {
                const f32x4_t v = *reinterpret_cast<const f32x4_any_t*>(src + j * 4 * L::E);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = v[i];
            } else kvc_load8(src + j * 4 * L::E, x);
#pragma unroll
            for (int i = 0; i < L::E; ++i) {
                x[i] = a.plain ? x[i] * a.scale : a.negative ? -x[i] : x[i];
                if (col >= cols) x[i] = 0.f;
            }
            if constexpr (F32) q.w[j][0] = u32x4_t{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
            else if constexpr (PLANES == 1) q4_operand<1>(x, q.w[j]);
            else {
                float rest[3][8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {               // (an infinity: all three parts are it)
                    const float least = x[i] * 0x1p-30f, x1 = x[i] - first_part(x[i]);
                    rest[0][i] = x[i];
                    rest[1][i] = fabsf(x1) > fabsf(least) ? x1 : least;
                    const float x2 = rest[1][i] - first_part(rest[1][i]);
                    rest[2][i] = fabsf(x2) > fabsf(least) ? x2 : least;
                }
#pragma unroll
                for (int e = 0; e < 3; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i) q.w[j][e][i] = first_parts(rest[e][2 * i], rest[e][2 * i + 1]);
            }
        }
    }
    static __device__ __forceinline__ float first_part(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }
    static __device__ __forceinline__ uint32_t first_parts(float x, float y) { return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u); }
    static __device__ __forceinline__ f32x4_t mfma4(uint32_t x, uint32_t y, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x), __uint_as_float(y), c, 0, 0, 0);
    }
    // scores of a page: rows (tokens) 4 (lane / 16) + i, column lane % 16
    static __device__ __forceinline__ f32x4_t scores(const u32x4_t k[N], const Q& q) {
        f32x4_t s = {};
#pragma unroll
        for (int j = 0; j < N; ++j)
            if constexpr (F32) {
#pragma unroll
                for (int i = 0; i < 4; ++i) s = mfma4(k[j][i], q.w[j][0][i], s);
            } else {
#pragma unroll
                for (int x = 0; x < PLANES; ++x) s = q4_mfma(k[j], q.w[j][x], s);
            }
        return s;
    }
    // probabilities of a chunk as operands
    struct P { u32x4_t w[PLANES]; };
    static __device__ __forceinline__ P weights(const f32x4_t s[PAGES]) {
        P p;
        if constexpr (F32) p.w[0] = u32x4_t{__float_as_uint(s[0][0]), __float_as_uint(s[0][1]), __float_as_uint(s[0][2]), __float_as_uint(s[0][3])};
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = s[i / 2][2 * (i & 1)], y = s[i / 2][2 * (i & 1) + 1];
                if constexpr (PLANES == 1) p.w[0][i] = f2bf2(x, y);
                else {                                      // (a probability is not negative)
                    const float xl = x * 0x1p-30f, yl = y * 0x1p-30f;
                    const float x1 = fmaxf(x - first_part(x), xl), y1 = fmaxf(y - first_part(y), yl);
                    p.w[0][i] = first_parts(x, y);
                    p.w[1][i] = first_parts(x1, y1);
                    p.w[2][i] = first_parts(fmaxf(x1 - first_part(x1), xl), fmaxf(y1 - first_part(y1), yl));
                }
            }
        return p;
    }
    // o += V^T P^T, block d of 16 dims
    static __device__ __forceinline__ void gather(const Entries& v, const P& p, f32x4_t o[HD / 16]) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if constexpr (F32) {
#pragma unroll
                for (int i = 0; i < 4; ++i) o[j] = mfma4(v.w[0][j][i], p.w[0][i], o[j]);
            } else {
                const u32x4_t x = v.w[0][j], y = v.w[1][j], lo = {x[0], x[1], y[0], y[1]}, hi = {x[2], x[3], y[2], y[3]};
#pragma unroll
                for (int e = 0; e < PLANES; ++e) {
                    o[2 * j] = q4_mfma(lo, p.w[e], o[2 * j]);
                    o[2 * j + 1] = q4_mfma(hi, p.w[e], o[2 * j + 1]);
                }
            }
    }
    // Whether a value among the entries is an infinity or a NaN: 0 times it is not 0.
    static __device__ __forceinline__ bool unbounded(const Entries& v) {
        f32x4_t z = {};
        P zero;
#pragma unroll
        for (int e = 0; e < PLANES; ++e) zero.w[e] = u32x4_t{};
        f32x4_t all[HD / 16];
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) all[d] = z;
        gather(v, zero, all);
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) z += all[d];
        return __any(!(z[0] + z[1] + z[2] + z[3] == 0.f));
    }
    // Values of the entries that no column of the tile sees, cleared: what lies there may be NaN, and 0 * NaN is NaN.  `seen(slot)`: some column does.
    template <typename F> static __device__ __forceinline__ void clear(Entries& v, int slot0, int there, F seen) {
        const int quad = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int p = 0; p < PAGES; ++p) {
            const int at = slot0 + p * KVC_PAGE + quad * 4;
            uint32_t m[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) m[i] = ((there >> p) & 1) && seen(at + i) ? 0xFFFFFFFFu : 0u;
#pragma unroll
            for (int j = 0; j < N; ++j)
                if constexpr (F32) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) v.w[p][j][i] &= m[i];
                } else {
                    const uint32_t a = (m[0] & 0xFFFFu) | (m[1] & 0xFFFF0000u), b = (m[2] & 0xFFFFu) | (m[3] & 0xFFFF0000u);
                    v.w[p][j] &= u32x4_t{a, b, a, b};
                }
        }
    }
    // The second product value by value, for a chunk that holds an infinity or a NaN which some columns must not meet
    static __device__ void gather_one_by_one(const C* const page[PAGES], int there, int slot0, const f32x4_t s[PAGES], const KvcColumn& see, f32x4_t o[HD / 16]) {
        const int lane = threadIdx.x & 63, quad = lane >> 4;
#pragma unroll
        for (int p = 0; p < PAGES; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll 1
                for (int from = 0; from < 4; ++from) {
                    const float w = __shfl(s[p][i], from * 16 + (lane & 15), 64);
                    if (!((there >> p) & 1) || !see.sees(slot0 + p * KVC_PAGE + from * 4 + i)) continue;
#pragma unroll
                    for (int d = 0; d < HD / 16; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[d][e] = __builtin_fmaf(w, ld1(page[p] + L::value(from * 4 + i, d * 16 + quad * 4 + e)), o[d][e]);
                }
    }
};

// the (page, head) blocks of a chunk; bit p of `there` is clear where the table names no page of the pool
template <typename C, int HD, int PAGES> __device__ __forceinline__ void kvc_pages(const KvcCache& c, int seq, int head, int slot0, const C* page[PAGES], int& there) {
    there = 0;
#pragma unroll
    for (int p = 0; p < PAGES; ++p) {
        const int i = slot0 / KVC_PAGE + p;
        int id = i < c.max_pages ? c.table[(int64_t)seq * c.max_pages + i] : -1;
        if ((unsigned)id < (unsigned)c.n_pages) there |= 1 << p;
        else id = 0;
        page[p] = reinterpret_cast<const C*>(c.pool) + ((int64_t)id * c.hkv + head) * KvcLayout<C, HD>::BLOCK;
    }
}

// Scores of a chunk -> probabilities in their place; the maximum moves where it has to, and what was gathered is scaled.  factor2 > 0; top is in units of the exponent.
template <int PAGES, int NB>
__device__ __forceinline__ void kvc_softmax(f32x4_t s[PAGES], float factor2, float& top, float& sum, f32x4_t o[NB]) {
    float best = -INFINITY;
#pragma unroll
    for (int p = 0; p < PAGES; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) best = fmaxf(best, s[p][i]);
    best = rows4_max(best);
    best = fmaxf(top, best * factor2);
    // (probabilities up to 2^8 lose nothing in 32 bits, nor in bf16)
    if (__any(best > top + 8.f)) {
        const float scale = __builtin_amdgcn_exp2f(top - (best == -INFINITY ? 0.f : best));
        sum *= scale;
#pragma unroll
        for (int d = 0; d < NB; ++d) o[d] *= scale;
        top = best;
    }
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int p = 0; p < PAGES; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[p][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[p][i], factor2, -base));
            sum += s[p][i];
        }
}
// what a column has gathered, rows (dims) dim .. + 3, to its place or to the join
template <typename T, int HD>
__device__ __forceinline__ void kvc_finish(const KvcAttn& a, int64_t row, int qh, int dim, bool first, f32x4_t acc, float top, float total, int part, int parts) {
    if (parts > 1) {
        const int64_t at = (row * a.heads + qh) * a.splits + part;
        *reinterpret_cast<f32x4_t*>(a.part_o + at * HD + dim) = acc;
        if (first) a.part_ml[at] = make_float2(top, total);
        return;
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    T* dst = static_cast<T*>(a.out) + row * a.o_row + qh * a.o_head + dim;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2_any_t*>(dst) = u32x2_t{f2bf2(acc[0] * inv, acc[1] * inv), f2bf2(acc[2] * inv, acc[3] * inv)};
    else *reinterpret_cast<f32x4_any_t*>(dst) = acc * inv;
    if (first && a.lse) a.lse[row * a.heads + qh] = total == 0.f ? -INFINITY : (top == -INFINITY ? 0.f : top) * 0.6931471805599453f + logf(total);
}
// One chunk against one tile of columns, keys and values as operands: the scores, then `border` decides what has to be masked
template <typename M, int HD, typename C>
__device__ __forceinline__ void kvc_chunk(const KvcAttn& a, const typename M::Q& q, const typename M::Entries& k, typename M::Entries& v, const C* const page[M::PAGES], int there,
                                          int slot0, const KvcSpan& span, const KvcColumn& see, float& top, float& sum, f32x4_t o[HD / 16]) {
    const int quad = (threadIdx.x & 63) >> 4;
    f32x4_t s[M::PAGES];
#pragma unroll
    for (int p = 0; p < M::PAGES; ++p) s[p] = M::scores(k.w[p], q);
    // every column sees all of it: it ends before the first row's slot, and begins in every window or ends among the sinks
    const bool whole = there == (1 << M::PAGES) - 1 && slot0 + M::CH <= span.safe && (slot0 >= span.low || slot0 + M::CH <= a.sinks);
    if (whole) {
        kvc_softmax<M::PAGES, HD / 16>(s, a.factor2, top, sum, o);
        M::gather(v, M::weights(s), o);
        return;
    }
    M::clear(v, slot0, there, [&](int slot) { return slot < span.end && (slot >= span.near || slot < a.sinks); });
#pragma unroll
    for (int p = 0; p < M::PAGES; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[p][i] = ((there >> p) & 1) && see.sees(slot0 + p * KVC_PAGE + quad * 4 + i) ? s[p][i] : -INFINITY;
    kvc_softmax<M::PAGES, HD / 16>(s, a.factor2, top, sum, o);
    if (M::unbounded(v)) M::gather_one_by_one(page, there, slot0, s, see, o);
    else M::gather(v, M::weights(s), o);
}

// A block owns a tile of 16 columns of one (sequence, kv head) and one part of its chunks, which its waves take in turn, each with its own running
// maximum and sum; they are joined in LDS.  The next chunk is requested before this one is worked on, the table entries one chunk earlier still.
template <typename T, typename C, int HD>
__global__ __launch_bounds__(512, 2) void kvc_attn_kernel(KvcAttn a) {
    typedef KvcMath<T, C, HD> M;
    constexpr int NB = HD / 16, WAVES = 8;
    __shared__ __align__(16) float lds_o[WAVES][NB][64][4];
    __shared__ float lds_ml[WAVES][2][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, quad = lane >> 4;
    int list, tile;
    if (!kvc_work(a, blockIdx.x, list, tile)) return;
    const int b = kvc_by_length(a, list / a.c.hkv), head = list % a.c.hkv, col0 = tile * 16, col = col0 + (lane & 15);
    int r0, count, n;
    kvc_rows(a, b, r0, count, n);
    const int cols = count * a.group;
    if (col0 >= cols) return;
    const KvcSpan span = kvc_span<M::CH>(a, count, n, col0, min(cols, col0 + 16));
    const int parts = kvc_parts(a, span);
    if ((int)blockIdx.y >= parts) return;
    const KvcColumn see = kvc_column(a, count, n, col, cols);
    const int end = min((int)(blockIdx.y + 1) * a.split, span.chunks);

    typename M::Entries k[2], v[2];
    const C* page[3][M::PAGES];                             // of the chunk worked on, the next one, the one after it
    int there[3];
    typename M::Q q;
    f32x4_t o[NB] = {};
    float top = -INFINITY, sum = 0.f;
    auto load = [&](const C* const pg[M::PAGES], typename M::Entries& k_, typename M::Entries& v_) {
#pragma unroll
        for (int p = 0; p < M::PAGES; ++p)
#pragma unroll
            for (int j = 0; j < M::N; ++j) {
                k_.w[p][j] = reinterpret_cast<const u32x4_t*>(pg[p])[j * 64 + lane];
                v_.w[p][j] = reinterpret_cast<const u32x4_t*>(pg[p] + KVC_PAGE * HD)[j * 64 + lane];
            }
    };
    auto table = [&](int i, const C* pg[M::PAGES], int& there_) { kvc_pages<C, HD, M::PAGES>(a.c, b, head, kvc_slot<M::CH>(span, min(i, max(span.chunks - 1, 0))), pg, there_); };
    int i = blockIdx.y * a.split + wave;
    M::load_q(a, r0, head, col, cols, lane, q);
    if (i < end) {
        table(i, page[0], there[0]);
        load(page[0], k[0], v[0]);
        table(i + waves, page[1], there[1]);
    }
    while (i < end) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (i + waves < end) load(page[1], k[1 - u], v[1 - u]);
            table(i + 2 * waves, page[2], there[2]);
            kvc_chunk<M, HD, C>(a, q, k[u], v[u], page[0], there[0], kvc_slot<M::CH>(span, i), span, see, top, sum, o);
#pragma unroll
            for (int p = 0; p < M::PAGES; ++p) page[0][p] = page[1][p], page[1][p] = page[2][p];
            there[0] = there[1], there[1] = there[2];
            i += waves;
            if (i >= end) break;
        }
    }
    sum = rows4_sum(sum);
    if (quad == 0) lds_ml[wave][0][lane] = top, lds_ml[wave][1][lane] = sum;
#pragma unroll
    for (int d = 0; d < NB; ++d) *reinterpret_cast<f32x4_t*>(lds_o[wave][d][lane]) = o[d];
    __syncthreads();
    for (int d = wave; d < NB; d += waves) {
        const int c = lane & 15;
        float best = -INFINITY, total = 0.f;
        for (int w = 0; w < waves; ++w) best = fmaxf(best, lds_ml[w][0][c]);
        const float base = best == -INFINITY ? 0.f : best;
        f32x4_t acc = {};
        for (int w = 0; w < waves; ++w) {
            const float scale = __builtin_amdgcn_exp2f(lds_ml[w][0][c] - base);
            total += scale * lds_ml[w][1][c];
            acc += scale * *reinterpret_cast<const f32x4_t*>(lds_o[w][d][lane]);
        }
        if (col < cols) kvc_finish<T, HD>(a, r0 + col / a.group, head * a.group + col % a.group, d * 16 + quad * 4, d == 0 && quad == 0, acc, best, total, blockIdx.y, parts);
    }
}

// Joins the parts of the entries: 16 lanes per (row, head), HD / 16 dims each, 16 parts' maxima and sums at once.  CH: slots to a chunk.
template <typename T, int HD, int CH>
__global__ __launch_bounds__(256) void kvc_join_kernel(KvcAttn a) {
    constexpr int N = HD / 16;
    const int l = threadIdx.x & 15;
    const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4;
    if (id >= (int64_t)a.c.batch * a.max_rows * a.heads) return;        // 16 lanes leave together
    const int qh = (int)(id % a.heads), r = (int)(id / a.heads % a.max_rows), b = (int)(id / a.heads / a.max_rows);
    int r0, count, n;
    kvc_rows(a, b, r0, count, n);
    if (r >= count) return;
    const int cols = count * a.group, col0 = (r * a.group + qh % a.group) / a.tile_cols * a.tile_cols;
    const KvcSpan span = kvc_span<CH>(a, count, n, col0, min(cols, col0 + a.tile_cols));
    const int parts = kvc_parts(a, span);
    if (parts == 1) return;                                 // a single part went to its place
    const int64_t row = r0 + r, at = (row * a.heads + qh) * a.splits;
    float best = -INFINITY;
    for (int s = l; s < parts; s += 16) best = fmaxf(best, a.part_ml[at + s].x);
    best = row16_max(best);
    const float base = best == -INFINITY ? 0.f : best;
    float total = 0.f, acc[N] = {};
    for (int s0 = 0; s0 < parts; s0 += 16) {
        float scale = 0.f;
        if (s0 + l < parts) {
            const float2 ml = a.part_ml[at + s0 + l];
            scale = __builtin_amdgcn_exp2f(ml.x - base);
            total += scale * ml.y;
        }
        const int m = min(16, parts - s0);
        const float* p = a.part_o + (at + s0) * HD + l * N;
        for (int s = 0; s < m; ++s) {
            const float w = __shfl(scale, s, 16);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] += w * p[s * HD + i];
        }
    }
    total = row16_sum(total);
    const float inv = total == 0.f ? 0.f : 1.f / total;
    T* dst = static_cast<T*>(a.out) + row * a.o_row + qh * a.o_head + l * N;
#pragma unroll
    for (int i = 0; i < N; ++i) st1(dst + i, acc[i] * inv);
    if (l == 0 && a.lse) a.lse[row * a.heads + qh] = total == 0.f ? -INFINITY : base * 0.6931471805599453f + logf(total);
}
