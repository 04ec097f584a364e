// Attention over the paged bf16 / fp32 cache: chunks of new tokens or single ones, with a sliding window and first tokens that stay visible.
//
// A column is a (row, head of the group) of one (sequence, kv head): column c is row c / group, head c % group.  Scores are S^T[token][column] = K Q^T, what
// is gathered is O^T[dim][column] += V^T P^T, both in tiles of 16 x 16 whose accumulators hold row 4 (lane / 16) + i, column lane % 16: a column's probabilities leave the first product in
// the lanes in which the second one wants them, and only the maximum and the sum cross lanes.  One pass over the entries with a running maximum and sum in fp32.
#pragma once
#include "kvc.h"

// Division of 0 <= n < 2^30 by a number that the host knows: inverse = 2^32 / d + 1 gives at most one too much; for d = 1 it is 2^32 - 1, one too little
struct KvcDivisor {
    uint32_t d, inverse;
    __device__ __forceinline__ int operator()(int n) const {
        const int q = (int)__umulhi((uint32_t)n, inverse);
        const int rest = n - q * (int)d;
        return q + (rest >= (int)d) - (rest < 0);
    }
};
struct KvcAttn {
    KvcCache c;
    const void* q;
    int64_t q_row, q_head;
    const int* row_start;   // [batch + 1]; null: row b is sequence b's
    int total_rows, max_rows, heads;
    KvcDivisor group, by_heads, by_tiles;    // heads of a kv head; by the kv heads and by the tiles
    float factor;           // |scale|; 1 where q is multiplied by it
    float factor2;          // the same * log2(e): finite, never 0
    float slack;            // 8 / factor2, finite: a score may pass the running maximum by so much
    bool negative;          // scale < 0: q changes its sign instead
    bool plain;             // scale is 0, infinite or NaN: q is multiplied by it, so that -inf means "not seen" and nothing else
    float scale;
    void* out;
    int64_t o_row, o_head;
    float* lse;             // [rows][heads] or null
    int max_kv, window, sinks;
    int ch;                 // slots of a chunk, or of a step of the kernel for many columns
    int lists, tiles, tile_cols;    // (sequence, kv head) pairs, tiles of columns of each
    int split, splits;      // chunks to a part, most parts
    bool by_length;         // the blocks of the longest sequences go first
    bool packed;            // blocks without columns lie behind the others
    float* part_o;          // [rows][heads][splits][hd], unnormalised
    float2* part_ml;        // [rows][heads][splits]: maximum, sum
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
// What the columns col0 .. col1 - 1 of a sequence see, in chunks (steps) of CH slots: the first `front` chunks (sinks), then those from `from` on, `chunks` in all.
struct KvcSpan {
    int end;                // no column sees a slot from here on
    int safe;               // every column sees the slots below (those of the window: from `low` on)
    int near, low;          // some column's window begins at `near`, every column's has begun at `low`
    int front, from, chunks;
};
__device__ __forceinline__ KvcSpan kvc_span(const KvcAttn& a, int CH, int count, int n, int col0, int col1) {
    KvcSpan s;
    const int p0 = n - count + a.group(col0), p1 = n - count + a.group(col1 - 1);      // slots of the first and the last row
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
// All bits where bit p of `there` is set.  (A mask that the compiler cannot look through: of branches on such a bit it has inverted one and not the other that went by the same comparison.)
__device__ __forceinline__ int kvc_on(int there, int p) {
    int on = -((there >> p) & 1);
    asm("" : "+v"(on));
    return on;
}
// what one column sees
struct KvcColumn {
    int low, high, sinks;
    __device__ __forceinline__ bool sees(int slot) const { return (slot < high) & ((slot >= low) | (slot < sinks)); }
};
__device__ __forceinline__ KvcColumn kvc_column(const KvcAttn& a, int count, int n, int col, int cols) {
    const int p = n - count + a.group(col);
    return KvcColumn{a.window ? p - a.window + 1 : 0, col < cols ? p + 1 : 0, a.sinks};
}

// Sequences of unlike lengths make blocks of unlike times: the longest go first where the blocks do not all run at once.  The i-th sequence in that order, among
// every 64 together, by the first eight bits of their lengths (of max_kv's): bit by bit, those that have it go before those that do not.  The same for all lanes of a whole wave.
__device__ __forceinline__ int kvc_by_length(const KvcAttn& a, int i) {
    if (!a.by_length) return i;
    const int lane = threadIdx.x & 63, first = i & ~63;
    const int key = first + lane < a.c.batch ? min(max(a.c.kv_len[first + lane], 0), a.max_kv) >> max(24 - __clz(a.max_kv), 0) : -1;
    uint64_t among = __ballot(key >= 0);
    int rank = i & 63;
#pragma unroll
    for (int bit = 7; bit >= 0; --bit) {
        const uint64_t have = __ballot((key >> bit) & 1) & among;
        const int n = __popcll(have);
        among = rank < n ? have : among & ~have;
        rank -= rank < n ? 0 : n;
    }
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(among >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)among, 0));
    return first + __builtin_ctzll(__ballot(((among >> lane) & 1) && before == rank));
}

// The place of a lane's sequence in the same order, among the up to 64 sequences of a wave's lanes that are `there` (the others keep their lanes, behind)
__device__ __forceinline__ int kvc_rank(bool there, int n, int max_kv) {
    const int lane = threadIdx.x & 63, key = n >> max(24 - __clz(max_kv), 0);
    const uint64_t all = __ballot(there);
    uint64_t among = all;
    int rank = 0;
#pragma unroll
    for (int bit = 7; bit >= 0; --bit) {
        const bool mine = (key >> bit) & 1;
        const uint64_t have = __ballot(mine) & all;
        rank += mine ? 0 : __popcll(among & have);
        among &= mine ? have : ~have;
    }
    return there ? rank + __popcll(among & ((1ull << lane) - 1)) : lane;
}

// The work of block `id`: a list, that is a (sequence, kv head), a tile of its columns, and a part of their chunks; the last tile first, which sees most.  Blocks go to the eight XCDs in
// turn: the tiles of a list, which read the same entries, are neighbours on one XCD and its L2.  Fewer than eight lists that divide eight share the XCDs out evenly.
// An XCD deals its blocks to 32 CUs in turn; where lists have several tiles every second round goes backwards, so that a CU whose first block is among the longest does not get the longest of every
// round (17 .. 128 rows, 16 sequences x 16 heads of 64, fp32: 45 us against 48 .. 51; 72B heads, 1024 .. 8192 entries: 204 against 209).  With one tile the longest first alone does better (256 single tokens of
// 4096 .. 8192: 534 against 549).  Blocks without columns, of sequences with fewer rows than others, would upset the rounds: `packed` counts the tiles that there are, sequence by sequence in the order of their lengths.
__host__ __device__ __forceinline__ int kvc_blocks(int lists, int tiles, int splits) {
    return (lists < 8 && 8 % lists == 0 ? (tiles + 8 / lists - 1) / (8 / lists) * 8 : (lists + 7) / 8 * 8 * tiles) * splits;
}
struct KvcWork {
    int b, head, tile, part;
    int r0, count, n;       // of the sequence: first row, rows, entries
};
__device__ __forceinline__ bool kvc_work(const KvcAttn& a, int id, KvcWork& w) {
    const int xcd = id & 7, all = gridDim.x >> 3;
    int at = id >> 3;
    if (a.tiles > 1 && (at & 32) && (at | 31) < all) at ^= 31;
    w.part = 0;
    if (a.splits > 1) {
        w.part = at / (all / a.splits);
        at -= w.part * (all / a.splits);
    }
    if (a.packed) {                                         // a lane to a sequence
        const int lane = threadIdx.x & 63;
        int r0 = 0, count = 0, n = 0;
        if (lane < a.c.batch) kvc_rows(a, lane, r0, count, n);
        const int sees = a.window && n - a.window - count > a.sinks ? a.window + count + a.sinks : n;
        const int rank = kvc_rank(lane < a.c.batch, sees, a.max_kv);
        const int from = __builtin_amdgcn_ds_permute(rank * 4, lane);       // lane r: the sequence that is r-th
        const int tiles = __shfl((count * (int)a.group.d + a.tile_cols - 1) >> (31 - __clz(a.tile_cols)), from);
        auto before = [&](int r) { return (r * a.c.hkv - xcd + 7) >> 3; };  // lists of this XCD before the r-th sequence's
        const int blocks = lane < a.c.batch ? (before(lane + 1) - before(lane)) * tiles : 0;
        int sum = blocks;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int other = __shfl_up(sum, d);
            sum += lane >= d ? other : 0;
        }
        const int r = __popcll(__ballot(sum <= at));
        if (r >= a.c.batch) return false;
        const int t = __builtin_amdgcn_readlane(tiles, r), start = at - (__builtin_amdgcn_readlane(sum, r) - __builtin_amdgcn_readlane(blocks, r)), which = start / t;
        w.b = __builtin_amdgcn_readlane(from, r);
        w.tile = t - 1 - (start - which * t);
        w.head = (before(r) + which) * 8 + xcd - r * a.c.hkv;
        w.r0 = __builtin_amdgcn_readlane(r0, w.b);
        w.count = __builtin_amdgcn_readlane(count, w.b);
        w.n = __builtin_amdgcn_readlane(n, w.b);
        return true;
    }
    int list;
    if (a.lists < 8 && 8 % a.lists == 0) {
        list = xcd % a.lists;
        w.tile = at * (8 / a.lists) + xcd / a.lists;
    } else {
        const int eight = a.by_tiles(at);
        list = eight * 8 + xcd;
        w.tile = at - eight * a.tiles;
    }
    w.tile = a.tiles - 1 - w.tile;
    if (list >= a.lists || w.tile < 0) return false;
    const int i = a.by_heads(list);
    w.head = list - i * a.c.hkv;
    w.b = kvc_by_length(a, i);
    kvc_rows(a, w.b, w.r0, w.count, w.n);
    return true;
}

// Activations of type T over a cache of type C.
//   bf16 over bf16: q as it is, a probability in two bf16 parts, which hold 16 bits (2^-16 of it, as over the 4-bit cache, where its result is rounded to 8 bits); one bf16 number was off by up to 2^-8
//     and cost a third more error than the rounding of the result alone (2.2e-3 against 1.66e-3 of it in the mean).
//   fp32 over bf16: q and probabilities in three bf16 parts, which hold all 24 bits; three matrix instructions each.
//   First parts are cut, not rounded, so that all have the sign of the whole, and from 2^-100 on none is 0 where the whole is not (2^-22 of the first or 2^-30 of the whole is added, or stands in): an
//     infinite key or value meets no 0 that would make a NaN of it.
//   fp32 over fp32: matrix instructions in fp32.
template <typename T, typename C, int HD> struct KvcMath {
    typedef KvcLayout<C, HD> L;
    static constexpr bool F32 = sizeof(C) == 4;
    static constexpr int N = L::N, PAGES = F32 ? 1 : 2, CH = PAGES * KVC_PAGE, PLANES = !F32 && sizeof(T) == 4 ? 3 : 1, PARTS = F32 ? 1 : sizeof(T) == 4 ? 3 : 2;     // of q; of a probability
    struct Q { u32x4_t w[N][PLANES]; };
    struct Entries { u32x4_t w[PAGES][N]; };        // keys, or values, of a chunk as pages hold them
    struct Values { u32x4_t w[HD / 16]; };          // values as operands: block d of 16 dims, rows (dims) lane % 16, tokens 4 (lane / 16) + i of the first page, then of the second
    static __device__ __forceinline__ Values operands(const Entries& e) {
        Values v;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
            if constexpr (F32) v.w[d] = e.w[0][d];
            else v.w[d] = u32x4_t{e.w[0][d / 2][2 * (d & 1)], e.w[0][d / 2][2 * (d & 1) + 1], e.w[PAGES - 1][d / 2][2 * (d & 1)], e.w[PAGES - 1][d / 2][2 * (d & 1) + 1]};
        return v;
    }

    // operands of a tile of 16 columns: column lane % 16, dims 4E j + E (lane / 16) ..
    static __device__ __forceinline__ void load_q(const KvcAttn& a, int r0, int head, int col, int cols, int lane, Q& q) {
        const int use = min(col, cols - 1), row = a.group(use), group = (int)a.group.d;
        const T* src = static_cast<const T*>(a.q) + (int64_t)(r0 + row) * a.q_row + (int64_t)(head * group + use - row * group) * a.q_head + (lane >> 4) * L::E;
        if constexpr (PLANES == 1)
            if (!a.plain) {                                 // (the bits as they are)
                const uint32_t sign = !a.negative ? 0u : F32 ? 0x80000000u : 0x80008000u, keep = col < cols ? 0xFFFFFFFFu : 0u;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    u32x4_t v = *reinterpret_cast<const u32x4_any_t*>(src + j * 4 * L::E);
                    q.w[j][0] = (v ^ sign) & keep;
                }
                return;
            }
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
    // Scores of a chunk, rows (tokens) 4 (lane / 16) + i of each page, column lane % 16 of each tile.  The sums go side by side: a matrix instruction that waits for the one
    // before it leaves the unit idle.
    template <int NT> static __device__ __forceinline__ void scores(const Entries& k, const Q q[NT], f32x4_t s[NT][PAGES]) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int p = 0; p < PAGES; ++p) s[t][p] = f32x4_t{};
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int x = 0; x < (F32 ? 4 : PLANES); ++x)
#pragma unroll
                for (int p = 0; p < PAGES; ++p)
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if constexpr (F32) s[t][p] = mfma4(k.w[p][j][x], q[t].w[j][0][x], s[t][p]);
                        else s[t][p] = q4_mfma(k.w[p][j], q[t].w[j][x], s[t][p]);
                    }
    }
    // probabilities of a chunk as operands
    struct P { u32x4_t w[PARTS]; };
    static __device__ __forceinline__ P weights(const f32x4_t s[PAGES]) {
        P p;
        if constexpr (F32) p.w[0] = u32x4_t{__float_as_uint(s[0][0]), __float_as_uint(s[0][1]), __float_as_uint(s[0][2]), __float_as_uint(s[0][3])};
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = s[i / 2][2 * (i & 1)], y = s[i / 2][2 * (i & 1) + 1];
                if constexpr (PARTS == 2) {
                    constexpr float LESS = -1.f + 0x1p-22f;
                    p.w[0][i] = first_parts(x, y);
                    p.w[1][i] = f2bf2(__builtin_fmaf(first_part(x), LESS, x), __builtin_fmaf(first_part(y), LESS, y));
                } else {                                    // (a probability is not negative)
                    const float x1 = __builtin_fmaf(x, 0x1p-30f, x - first_part(x)), y1 = __builtin_fmaf(y, 0x1p-30f, y - first_part(y));
                    const float x2 = __builtin_fmaf(x, 0x1p-30f, x1 - first_part(x1)), y2 = __builtin_fmaf(y, 0x1p-30f, y1 - first_part(y1));
                    p.w[0][i] = first_parts(x, y);
                    p.w[1][i] = first_parts(x1, y1);
                    p.w[2][i] = first_parts(x2, y2);
                }
            }
        return p;
    }
    // o += V^T P^T, block d of 16 dims, for every tile; sums side by side
    template <int NT> static __device__ __forceinline__ void gather(const Values& v, const P p[NT], f32x4_t o[NT][HD / 16]) {
        constexpr int SIDE = HD / 16 < 4 ? HD / 16 : 4;
#pragma unroll
        for (int d0 = 0; d0 < HD / 16; d0 += SIDE)
#pragma unroll
            for (int e = 0; e < (F32 ? 4 : PARTS); ++e)
#pragma unroll
                for (int d = d0; d < d0 + SIDE; ++d)
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if constexpr (F32) o[t][d] = mfma4(v.w[d][e], p[t].w[0][e], o[t][d]);
                        else o[t][d] = q4_mfma(v.w[d], p[t].w[e], o[t][d]);
                    }
    }
    // Whether a value among the entries is an infinity or a NaN: 0 times it is not 0.
    static __device__ __forceinline__ bool unbounded(const Values& v) {
        f32x4_t z = {};
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
            if constexpr (F32) {
#pragma unroll
                for (int i = 0; i < 4; ++i) z = mfma4(v.w[d][i], 0u, z);
            } else z = q4_mfma(v.w[d], u32x4_t{}, z);
        return __any(!(z[0] + z[1] + z[2] + z[3] == 0.f));
    }
    // slot of the tokens that dword i of an operand holds (the first of two in bf16)
    static __device__ __forceinline__ int slot_of(int slot0, int i) {
        const int quad = (threadIdx.x & 63) >> 4;
        return F32 ? slot0 + quad * 4 + i : slot0 + i / 2 * KVC_PAGE + quad * 4 + 2 * (i & 1);
    }
    // Values of the entries that no column of the tile sees, cleared: what lies there may be NaN, and 0 * NaN is NaN.
    static __device__ __forceinline__ void clear(Values& v, int slot0, int there, const KvcSpan& span, int sinks) {
        u32x4_t m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int slot = slot_of(slot0, i), end = span.end & kvc_on(there, F32 ? 0 : i / 2);
            auto seen = [&](int at) { return (at < end) & ((at >= span.near) | (at < sinks)); };
            m[i] = F32 ? -(uint32_t)seen(slot) : (-(uint32_t)seen(slot) & 0xFFFFu) | (-(uint32_t)seen(slot + 1) & 0xFFFF0000u);
        }
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) v.w[d] &= m;
    }
    // Infinities and NaN among the values reach the columns that see them and no others: products of marks (rows: dims) and of what is seen, shaped like the one of values and
    // probabilities, count them; `strip` takes them out of the values.
    static __device__ __forceinline__ uint32_t strip1(uint32_t w) {
        if constexpr (F32) return (w & 0x7F800000u) == 0x7F800000u ? 0u : w;
        return ((w & 0x7F80u) == 0x7F80u ? 0u : w & 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0u : w & 0xFFFF0000u);
    }
    static __device__ __forceinline__ void strip(Values& v) {
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) v.w[d][i] = strip1(v.w[d][i]);
    }
    // 1 where a value is `what` (bits of its type), or NaN where what is 0
    static __device__ __forceinline__ uint32_t mark1(uint32_t w, uint32_t what) {
        if constexpr (F32) return (what ? w == what : (w & 0x7FFFFFFFu) > 0x7F800000u) ? 0x3F800000u : 0u;
        const uint32_t lo = w & 0xFFFFu, hi = w >> 16;
        return ((what ? lo == what : (lo & 0x7FFFu) > 0x7F80u) ? 0x3F80u : 0u) | ((what ? hi == what : (hi & 0x7FFFu) > 0x7F80u) ? 0x3F800000u : 0u);
    }
    template <int NT> static __device__ __forceinline__ void add_unbounded(const Values& v, const KvcColumn see[NT], int slot0, f32x4_t o[NT][HD / 16]) {
        u32x4_t sees[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int slot = slot_of(slot0, i);
                if constexpr (F32) sees[t][i] = see[t].sees(slot) ? 0x3F800000u : 0u;
                else sees[t][i] = (see[t].sees(slot) ? 0x3F80u : 0u) | (see[t].sees(slot + 1) ? 0x3F800000u : 0u);
            }
        constexpr uint32_t PLUS = F32 ? 0x7F800000u : 0x7F80u, MINUS = F32 ? 0xFF800000u : 0xFF80u;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
#pragma unroll
            for (int kind = 0; kind < 3; ++kind) {
                const uint32_t what = kind == 0 ? PLUS : kind == 1 ? MINUS : 0u;
                const float add = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : __uint_as_float(0x7FC00000u);
                u32x4_t mark;
#pragma unroll
                for (int i = 0; i < 4; ++i) mark[i] = mark1(v.w[d][i], what);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    f32x4_t many = {};
                    if constexpr (F32) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) many = mfma4(mark[i], sees[t][i], many);
                    } else many = q4_mfma(mark, sees[t], many);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[t][d][e] += many[e] > 0.f ? add : 0.f;
                }
                __builtin_amdgcn_sched_barrier(0);          // (marks of one block and kind at a time: registers)
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

// The weight 2^(factor2 (s - top)) of a score, or of what was gathered under another maximum.  The difference is formed first and is 0 at the maximum.  (factor2 s - fl(factor2 top) in one
// multiply-add keeps the rounding of the second product, half a step of it: beyond 2^31 that is 128 and more, and the weights of the largest scores themselves were 0 or infinite.)
__device__ __forceinline__ float kvc_weight(const KvcAttn& a, float s, float base) { return __builtin_amdgcn_exp2f((s - base) * a.factor2); }
__device__ __forceinline__ float kvc_base(float top) { return top == -INFINITY ? 0.f : top; }
__device__ __forceinline__ float kvc_lse(const KvcAttn& a, float top, float total) { return total == 0.f ? -INFINITY : kvc_base(top) * a.factor + logf(total); }

// The running state of a lane's column.  `top`, the largest score q.K, is the same in its four lanes, `sum` each lane's own.
struct KvcRun {
    float top = -INFINITY, base = 0.f, limit = -INFINITY, sum = 0.f;      // base: top, or 0 where that is -inf; limit: of scores that need no new maximum
};
// Scores of a chunk -> probabilities in their place; the maximum moves, and what was gathered is scaled, only where a score passes it by so much that a probability would pass 2^8 (up to
// there they lose nothing in 32 bits, nor in bf16): seldom after the first chunks, so the lanes of a column exchange their maxima there and nowhere else.  factor2 > 0.
template <int PAGES, int NB>
__device__ __forceinline__ void kvc_softmax(f32x4_t s[PAGES], const KvcAttn& a, KvcRun& r, f32x4_t o[NB]) {
    float best = s[0][0];
#pragma unroll
    for (int i = 1; i < 4 * PAGES; ++i) best = fmaxf(best, s[i / 4][i % 4]);
    if (__any(best > r.limit)) {
        const float top = fmaxf(r.top, rows4_max(best)), base = kvc_base(top);
        const float scale = kvc_weight(a, r.top, base);
        r.sum *= scale;
#pragma unroll
        for (int d = 0; d < NB; ++d) o[d] *= scale;
        r.top = top;
        r.base = base;
        r.limit = top + a.slack;
    }
#pragma unroll
    for (int p = 0; p < PAGES; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[p][i] = kvc_weight(a, s[p][i], r.base);
            r.sum += s[p][i];
        }
}
// What a column has gathered, blocks of 16 dims from d on (dims 16 d + 4 (lane / 16) + i each), to its place or to the join
template <typename T, int HD, int COUNT>
__device__ __forceinline__ void kvc_finish(const KvcAttn& a, int r0, int head, int col, int d, const f32x4_t acc[COUNT], float top, float total, int part, int parts) {
    const int quad = (threadIdx.x & 63) >> 4, row = a.group(col), qh = head * (int)a.group.d + col - row * (int)a.group.d;
    const int64_t line = (int64_t)(r0 + row) * a.heads + qh;
    if (parts > 1) {
        const int64_t at = line * a.splits + part;
        float* dst = a.part_o + at * HD + d * 16 + quad * 4;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) *reinterpret_cast<f32x4_t*>(dst + i * 16) = acc[i];
        if (d == 0 && quad == 0) a.part_ml[at] = make_float2(top, total);
        return;
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    T* dst = static_cast<T*>(a.out) + (int64_t)(r0 + row) * a.o_row + qh * a.o_head + d * 16 + quad * 4;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const f32x4_t x = acc[i] * inv;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2_any_t*>(dst + i * 16) = u32x2_t{f2bf2(x[0], x[1]), f2bf2(x[2], x[3])};
        else *reinterpret_cast<f32x4_any_t*>(dst + i * 16) = x;
    }
    if (d == 0 && quad == 0 && a.lse) a.lse[line] = kvc_lse(a, top, total);
}
// Scores that a column must not see, where a chunk is not seen whole by all of them
template <typename M, int NT> __device__ __forceinline__ void kvc_mask_scores(const KvcColumn see[NT], int slot0, int there, f32x4_t s[NT][M::PAGES]) {
    const int quad = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int p = 0; p < M::PAGES; ++p) {
            const KvcColumn c{see[t].low, see[t].high & kvc_on(there, p), see[t].sinks};
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t][p][e] = c.sees(slot0 + p * KVC_PAGE + quad * 4 + e) ? s[t][p][e] : -INFINITY;
        }
}
// every column sees all of the chunk: it ends before the first row's slot, and begins in every window or ends among the sinks
template <typename M> __device__ __forceinline__ bool kvc_whole(const KvcAttn& a, const KvcSpan& span, int slot0, int there) {
    return there == (1 << M::PAGES) - 1 && slot0 + M::CH <= span.safe && (slot0 >= span.low || slot0 + M::CH <= a.sinks);
}
// The values of such a chunk: what no column sees is cleared, and an infinity or a NaN must not reach the columns that do not see it, as 0 times it
template <typename M, int HD, int NT>
__device__ __forceinline__ void kvc_bound_values(const KvcAttn& a, const KvcSpan& span, const KvcColumn see[NT], int slot0, int there, typename M::Values& v, f32x4_t o[NT][HD / 16]) {
    M::clear(v, slot0, there, span, a.sinks);
    if (!M::unbounded(v)) return;
    M::template add_unbounded<NT>(v, see, slot0, o);
    M::strip(v);
}

// Few columns (single tokens), and everything over an fp32 cache: a block owns a tile of 16 columns of one (sequence, kv head) and one part of its chunks, which its waves take in
// turn, each with its own running maximum and sum; they are joined in LDS.  The next chunk's keys are requested as soon as this one's are used up, the values likewise, the table entries
// one chunk earlier still: one set of registers for each instead of two, and eight waves on a CU.
// Bound by bytes: 256 sequences of 4096 .. 8192 entries, 7B heads, bf16 (3.24 GB): 537 us, 6.0 TB/s, what a read alone reaches (572 with two whole chunks of registers, 558 with four waves to a
// block); with a window of 1024 and 4 sinks (543 MB) 102 us, 5.3 TB/s.  One sequence of 1279 entries: 10 us, five chunks to a wave, one latency each.  fp32, 16 x 16 heads of 64, 17 .. 128
// rows: 43 us, matrix instructions in fp32 at 68 TFLOP/s; 63 with the kernel of many columns, whose waves have no columns in a last tile.
template <typename T, typename C, int HD>
__global__ __launch_bounds__(512, 2) void kvc_attn_few_kernel(KvcAttn a) {
    typedef KvcMath<T, C, HD> M;
    constexpr int NB = HD / 16, WAVES = 8;
    __shared__ __align__(16) float lds_o[WAVES][NB][64][4];
    __shared__ float lds_ml[WAVES][2][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, quad = lane >> 4;
    KvcWork work;
    if (!kvc_work(a, blockIdx.x, work)) return;
    const int b = work.b, head = work.head, part = work.part, r0 = work.r0, count = work.count, n = work.n, cols = count * (int)a.group.d, col0 = work.tile * 16, col = col0 + (lane & 15);
    if (col0 >= cols) return;
    const KvcSpan span = kvc_span(a, M::CH, count, n, col0, min(cols, col0 + 16));
    const int parts = kvc_parts(a, span);
    if (part >= parts) return;
    const int end = min((part + 1) * a.split, span.chunks);

    typename M::Entries k, v;
    typename M::Q q[1];
    const KvcColumn see[1] = {kvc_column(a, count, n, col, cols)};
    f32x4_t o[1][NB] = {};
    KvcRun run;
    int i = part * a.split + wave;
    // (past the end the wave's last chunk is requested again)
    auto table = [&](int i, const C* pg[M::PAGES], int& there_) { kvc_pages<C, HD, M::PAGES>(a.c, b, head, kvc_slot<M::CH>(span, i < end ? i : end - 1 - (end - 1 - wave + waves * 4096) % waves), pg, there_); };
    auto load = [&](const C* const pg[M::PAGES], int offset, typename M::Entries& e) {
#pragma unroll
        for (int p = 0; p < M::PAGES; ++p)
#pragma unroll
            for (int j = 0; j < M::N; ++j) e.w[p][j] = reinterpret_cast<const u32x4_t*>(pg[p] + offset)[j * 64 + lane];
    };
    const C* page[M::PAGES];                                // of the chunk whose entries are requested next
    int there = 0, there_next = 0;
    if (i < end) {
        table(i, page, there);
        load(page, 0, k);
        load(page, KVC_PAGE * HD, v);
        table(i + waves, page, there_next);
    }
    M::load_q(a, r0, head, col, cols, lane, q[0]);
    for (; i < end; i += waves) {
        const int slot0 = kvc_slot<M::CH>(span, i);
        f32x4_t s[1][M::PAGES];
        M::template scores<1>(k, q, s);
        __builtin_amdgcn_sched_barrier(0);
        load(page, 0, k);
        __builtin_amdgcn_sched_barrier(0);
        const bool whole = kvc_whole<M>(a, span, slot0, there);
        if (!whole) kvc_mask_scores<M, 1>(see, slot0, there, s);
        kvc_softmax<M::PAGES, NB>(s[0], a, run, o[0]);
        typename M::Values vo = M::operands(v);
        if (!whole) kvc_bound_values<M, HD, 1>(a, span, see, slot0, there, vo, o);
        const typename M::P w[1] = {M::weights(s[0])};
        M::template gather<1>(vo, w, o);
        __builtin_amdgcn_sched_barrier(0);
        load(page, KVC_PAGE * HD, v);
        there = there_next;
        table(i + 2 * waves, page, there_next);
        __builtin_amdgcn_sched_barrier(0);
    }
    const float sum = rows4_sum(run.sum);
    if (quad == 0) lds_ml[wave][0][lane] = run.top, lds_ml[wave][1][lane] = sum;
#pragma unroll
    for (int d = 0; d < NB; ++d) *reinterpret_cast<f32x4_t*>(lds_o[wave][d][lane]) = o[0][d];
    __syncthreads();
    for (int d = wave; d < NB; d += waves) {
        const int c = lane & 15;
        float best = -INFINITY, total = 0.f;
        for (int w = 0; w < waves; ++w) best = fmaxf(best, lds_ml[w][0][c]);
        const float base = kvc_base(best);
        f32x4_t acc = {};
        for (int w = 0; w < waves; ++w) {
            const float scale = kvc_weight(a, lds_ml[w][0][c], base);
            total += scale * lds_ml[w][1][c];
            acc += scale * *reinterpret_cast<const f32x4_t*>(lds_o[w][d][lane]);
        }
        if (col < cols) kvc_finish<T, HD, 1>(a, r0, head, col, d, &acc, best, total, part, parts);
    }
}

// COUNT KB straight into LDS, 16 bytes to a lane and instruction (the instruction's offset goes into both addresses)
template <int COUNT> __device__ __forceinline__ void kvc_copy(uint32_t lds, uint32_t lane16, const char* base) {
    if constexpr (COUNT > 4) {
        kvc_copy<4>(lds, lane16, base);
        kvc_copy<COUNT - 4>(lds + 4096, lane16, base + 4096);
    } else if constexpr (COUNT == 4)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:0x400\n\tglobal_load_lds_dwordx4 %1, %2 offset:0x800\n\t"
                     "global_load_lds_dwordx4 %1, %2 offset:0xc00" ::"s"(lds), "v"(lane16), "s"(base) : "memory");
    else if constexpr (COUNT == 2)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:0x400" ::"s"(lds), "v"(lane16), "s"(base) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(lane16), "s"(base) : "memory");
}

// Many columns over a bf16 cache (chunks of prompts, steps, scoring): a block of four waves owns 64 * NT columns, NT tiles to a wave, and one part of their steps of U chunks.  The steps go through a ring of
// R stages in LDS, straight from memory (pages are operands as they are), a quarter of each by every wave.  The one barrier of a step stands in the middle of its last chunk,
// when all of the step's operands are in registers: behind it the next step's keys are read and this one's stage is requested anew.
// 2048 rows of a 7B prompt's 8192 entries: 305 us, 690 TFLOP/s, or 1035 with the second parts of the probabilities, of the 1396 that a plain product of 8192^3 reaches (348 with NT = 1; 229 with
// probabilities of 8 bits).  Per 32 entries and 16 columns there are 24 matrix instructions and 78 others, 8 of them exponentials, which a wave does in turn; two waves on a SIMD, of different blocks, overlap them in part.
// Steps without a mask have a loop of their own: where both kinds met in one, every operand was copied.  The instance of NT = 2 at 128 dims spills 33 of 256 registers, all of them in the steps with
// a mask, whose reloads wait for the ring's copies too; also where a window makes more of those it is ahead of NT = 1 (2048 rows of 8192, window 2000: 107 and 113 us).
// 16 sequences of 17 .. 128 rows, 72B heads, fp32 (three parts), window 1000: 106 us, 0.87 executed PFLOP/s.  64 sequences of 128 .. 5120 entries, 5 rows each, 7B heads: 76 .. 78 us with the join, 4.5 TB/s;
// 256 of 2048 entries, 8 rows: 201 us, 5.5 TB/s.
template <typename T, typename C, int HD, int NT> struct KvcMany {
    static constexpr bool SMALL = NT == 1 && sizeof(T) == sizeof(C);
    static constexpr int U = SMALL ? 1 : 2, R = SMALL ? 3 : 2, CH = U * KvcMath<T, C, HD>::CH;      // CH: slots of a step
};
template <typename T, typename C, int HD, int NT>
__global__ __launch_bounds__(256, 2) void kvc_attn_many_kernel(KvcAttn a) {
    typedef KvcMath<T, C, HD> M;
    typedef KvcLayout<C, HD> L;
    typedef KvcMany<T, C, HD, NT> K;
    constexpr int NB = HD / 16, N = M::N, U = K::U, R = K::R, CH = K::CH, PAGES = U * M::PAGES, OWN = PAGES * 2 * N / 4, COLS = 64 * NT;      // a wave requests OWN of a stage's KB
    constexpr int SPAN = 64 / PAGES;                        // steps whose table entries a wave holds, one to a lane
    static_assert(2 * N % OWN == 0, "a wave's share lies in one page");
    __shared__ u32x4_t ring[R][PAGES][2 * N][64];           // keys, then values of each page
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quad = lane >> 4;
    KvcWork work;
    if (!kvc_work(a, blockIdx.x, work)) return;
    const int b = work.b, head = work.head, part = work.part, r0 = work.r0, count = work.count, n = work.n, cols = count * (int)a.group.d, col0 = work.tile * COLS;
    if (col0 >= cols) return;
    const KvcSpan span = kvc_span(a, CH, count, n, col0, min(cols, col0 + COLS));
    const int parts = kvc_parts(a, span);
    if (part >= parts) return;
    const int begin = part * a.split, end = min(begin + a.split, span.chunks);
    // this wave's columns, what they see, and the steps that all of them see whole (but for missing pages)
    const int colw = col0 + wave * 16 * NT;
    const bool mine = colw < cols;
    const KvcSpan own = kvc_span(a, CH, count, n, min(colw, cols - 1), min(cols, colw + 16 * NT));
    const int whole0 = max(span.front, span.front + (own.low + CH - 1) / CH - span.from), whole1 = mine ? span.front + own.safe / CH - span.from : 0;
    KvcColumn see[NT];
    typename M::Q q[NT];
    f32x4_t o[NT][NB];
    KvcRun run[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int col = colw + 16 * t + (lane & 15);
        see[t] = kvc_column(a, count, n, col, cols);
        M::load_q(a, r0, head, col, cols, lane, q[t]);
#pragma unroll
        for (int d = 0; d < NB; ++d) o[t][d] = f32x4_t{};
    }
    int ids = 0, ids_from = begin - SPAN;                   // of the step ids_from + lane / PAGES, its page lane % PAGES
    uint64_t ids_there = 0;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)ring + wave * OWN * 1024;
    auto request = [&](int i, int stage) {                  // returns which of the step's pages are there
        if (i - ids_from >= SPAN) {
            ids_from = i;
            const int at = kvc_slot<CH>(span, min(i + lane / PAGES, span.chunks - 1)) / KVC_PAGE + lane % PAGES;
            ids = at < a.c.max_pages ? a.c.table[(int64_t)b * a.c.max_pages + at] : -1;
            if ((unsigned)ids >= (unsigned)a.c.n_pages) ids = -1;
            asm volatile("" : "+v"(ids));                   // (waited for here, not at every use)
            ids_there = __ballot(ids >= 0);
        }
        const int at = (i - ids_from) * PAGES;
        const int id = max(__builtin_amdgcn_readlane(ids, at + wave * OWN / (2 * N)), 0);
        const char* src = a.c.pool + ((int64_t)id * a.c.hkv + head) * (L::BLOCK * (int64_t)sizeof(C)) + wave * OWN % (2 * N) * 1024;
        kvc_copy<OWN>(lds0 + stage * (PAGES * 2 * N * 1024), lane * 16, src);
        return (int)(ids_there >> at) & ((1 << PAGES) - 1);
    };
    typename M::Entries k, v;
    auto read_k = [&](int stage, int u) {
#pragma unroll
        for (int x = 0; x < M::PAGES * N; ++x) k.w[x / N][x % N] = ring[stage][u * M::PAGES + x / N][x % N][lane];
    };
    auto read_v = [&](int stage, int u) {
#pragma unroll
        for (int x = 0; x < M::PAGES * N; ++x) v.w[x / N][x % N] = ring[stage][u * M::PAGES + x / N][N + x % N][lane];
    };
    if (begin < end) {
        int there[R];                                       // of this step, the next one, ...
#pragma unroll
        for (int i = 0; i < R; ++i) there[i] = begin + i < end ? request(begin + i, i) : 0;
        if (begin + R <= end) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((R - 1) * OWN) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        read_k(0, 0);
        int stage = 0;
        auto turn = [&](int i) {                            // the next step's entries have landed, this one's are in registers
            // (of the steps i + 1 .. i + R - 1, requested in turn, all but the first may still be on their way; near the end there are fewer)
            if (i + R <= end) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((R - 2) * OWN) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const int last = i + R < end ? request(i + R, stage) : 0;
#pragma unroll
            for (int x = 0; x + 1 < R; ++x) there[x] = there[x + 1];
            there[R - 1] = last;
            stage = stage == R - 1 ? 0 : stage + 1;
            read_k(stage, 0);
        };
        auto step = [&](auto border, int i) {
            const int there_i = there[0], slot = border.value ? kvc_slot<CH>(span, i) : 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int slot0 = slot + u * M::CH, there0 = there_i >> (u * M::PAGES);
                read_v(stage, u);
                f32x4_t s[NT][M::PAGES];
                M::template scores<NT>(k, q, s);
                if constexpr (border.value) kvc_mask_scores<M, NT>(see, slot0, there0, s);
#pragma unroll
                for (int t = 0; t < NT; ++t) kvc_softmax<M::PAGES, NB>(s[t], a, run[t], o[t]);
                typename M::Values vo;
                if constexpr (border.value) {
                    vo = M::operands(v);
                    kvc_bound_values<M, HD, NT>(a, own, see, slot0, there0, vo, o);
                }
                if (u == U - 1) turn(i);
                else read_k(stage, u + 1);
                if constexpr (!border.value) vo = M::operands(v);
                typename M::P w[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) w[t] = M::weights(s[t]);
                M::template gather<NT>(vo, w, o);
            }
        };
        for (int i = begin; i < end; ++i) {
            // (a loop of its own for what needs no mask: where the two kinds of steps met in one, the rare one cost the other copies of its operands)
            for (; i >= whole0 && i < min(end, whole1) && there[0] == (1 << PAGES) - 1; ++i) step(std::false_type{}, i);
            if (i >= end) break;
            const int slot0 = kvc_slot<CH>(span, i);
            if (!mine || slot0 >= own.end || (slot0 + CH <= own.near && slot0 >= a.sinks)) turn(i);      // (the other waves need this one's copies)
            else step(std::true_type{}, i);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");      // nothing is in flight into LDS when the block ends
    }
    if (!mine) return;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int col = colw + 16 * t + (lane & 15);
        const float total = rows4_sum(run[t].sum);
        if (col < cols) kvc_finish<T, HD, NB>(a, r0, head, col, 0, o[t], run[t].top, total, part, parts);
    }
}

// Joins the parts of the entries: 16 lanes per (row, head), HD / 16 dims each, 16 parts' maxima and sums at once.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kvc_join_kernel(KvcAttn a) {
    constexpr int N = HD / 16;
    const int l = threadIdx.x & 15;
    const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4;
    if (id >= (int64_t)a.c.batch * a.max_rows * a.heads) return;        // 16 lanes leave together
    const int qh = (int)(id % a.heads), r = (int)(id / a.heads % a.max_rows), b = (int)(id / a.heads / a.max_rows);
    int r0, count, n;
    kvc_rows(a, b, r0, count, n);
    if (r >= count) return;
    const int group = (int)a.group.d, cols = count * group, col0 = (r * group + qh % group) / a.tile_cols * a.tile_cols;
    const KvcSpan span = kvc_span(a, a.ch, count, n, col0, min(cols, col0 + a.tile_cols));
    const int parts = kvc_parts(a, span);
    if (parts == 1) return;                                 // a single part went to its place
    const int64_t row = r0 + r, at = (row * a.heads + qh) * a.splits;
    float best = -INFINITY;
    for (int s = l; s < parts; s += 16) best = fmaxf(best, a.part_ml[at + s].x);
    best = row16_max(best);
    const float base = kvc_base(best);
    float total = 0.f, acc[N] = {};
    for (int s0 = 0; s0 < parts; s0 += 16) {
        float scale = 0.f;
        if (s0 + l < parts) {
            const float2 ml = a.part_ml[at + s0 + l];
            scale = kvc_weight(a, ml.x, base);
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
    if (l == 0 && a.lse) a.lse[row * a.heads + qh] = kvc_lse(a, best, total);
}
