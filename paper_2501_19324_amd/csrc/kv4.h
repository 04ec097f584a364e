// A paged KV cache held in 4 bits: writing and reading entries, attention, eviction.
//
// Page [kv head][HD * 17 bytes], 16 tokens.  Keys: quarter q of the head dimension, token t, HD/8 bytes: lane l = 16 q + t of a wave loads its
// part of the page as one vector, the A operand of the products q.K (rows: tokens) after the conversion to bf16.  Values: lane l = 16 c + m
// loads for tokens 4 c .. + 3 the dims m and m + 16 of every group of 32: byte [group][token % 4] holds that pair, so the conversion (one scale for both values of a
// byte) sees one token and one group at a time.  Four tokens' pairs are transposed by byte permutes into the A operands of the products
// V^T P^T (rows: dims), whose contraction order (tokens 4 c + i of one page, then of the next) is the layout in which the matrix instruction
// leaves the scores: the probabilities go from one product into the other without leaving their lanes.
// A byte belongs to one token: an entry is written without reading its neighbours.  (The moves of an eviction own the pages that they write to, and write the values
// of such a page back whole.)
#pragma once
#include "q4.h"

#define KV4_PAGE 16
#define KV4_CHUNK 64        // tokens a wave takes at once

struct Kv4Cache {
    uint8_t* pool;
    const int* table;       // [batch][max_pages]
    int* kv_len;            // [batch]
    int n_pages, hkv, batch, max_pages;
};
__device__ __forceinline__ int64_t kv4_block(int hd) { return (int64_t)hd * 17; }
// address of a (page, head) block; a table entry outside the pool gives null
__device__ __forceinline__ uint8_t* kv4_page(const Kv4Cache& c, int hd, int seq, int page, int head) {
    const int p = c.table[(int64_t)seq * c.max_pages + page];
    return (unsigned)p < (unsigned)c.n_pages ? c.pool + ((int64_t)p * c.hkv + head) * kv4_block(hd) : nullptr;
}
// places of one entry's bytes inside its block
__device__ __forceinline__ int kv4_key_at(int hd, int t, int dim) { return dim / (hd / 4) * 2 * hd + t * (hd / 8) + dim % (hd / 4) / 2; }
__device__ __forceinline__ int kv4_val_at(int hd, int t, int g, int m) { return 8 * hd + (t >> 2) * 2 * hd + m * (hd / 8) + g * 4 + (t & 3); }
__device__ __forceinline__ int kv4_key_scale_at(int hd, int t, int g) { return 16 * hd + g * 16 + t; }
__device__ __forceinline__ int kv4_val_scale_at(int hd, int t, int g) { return 16 * hd + hd / 2 + ((t >> 2) * (hd / 32) + g) * 4 + (t & 3); }

struct Kv4Book {            // per entry: accumulated attention weight, position; either may be null
    float* scores;
    int* pos;
    int64_t score_b, score_h, pos_b, pos_h;
};

// consecutive values at any address
__device__ __forceinline__ void kv4_load4(const float* p, float o[4]) {
    const f32x4_t v = *reinterpret_cast<const f32x4_any_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = v[i];
}
__device__ __forceinline__ void kv4_load4(const bf16_t* p, float o[4]) {
    const u32x2_t v = *reinterpret_cast<const u32x2_any_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __uint_as_float(i & 1 ? v[i / 2] & 0xFFFF0000u : v[i / 2] << 16);
}
__device__ __forceinline__ void kv4_load8(const float* p, float o[8]) { kv4_load4(p, o); kv4_load4(p + 4, o + 4); }
__device__ __forceinline__ void kv4_load8(const bf16_t* p, float o[8]) {
    const u32x4_t v = *reinterpret_cast<const u32x4_any_t*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = __uint_as_float(i & 1 ? v[i / 2] & 0xFFFF0000u : v[i / 2] << 16);
}
// scale byte and codes of a group of 32 held by four neighbouring lanes, eight values each: x[i], x[i + 4] share byte i where PAIRED,
// x[2 i], x[2 i + 1] otherwise
template <bool PAIRED> __device__ __forceinline__ uint32_t kv4_encode8(const float x[8], int& scale_byte) {
    float amax = 0.f;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(x[i])), bad |= !q4_finite(x[i]);
    amax = fmaxf(amax, __uint_as_float(dpp_move<0xB1>(__float_as_uint(amax))));
    amax = fmaxf(amax, __uint_as_float(dpp_move<0x4E>(__float_as_uint(amax))));
    uint32_t any = bad;
    any |= dpp_move<0xB1>(any);
    any |= dpp_move<0x4E>(any);
    scale_byte = any ? Q4_NAN : q4_scale_byte(amax);
    const float scale = __uint_as_float((uint32_t)scale_byte << 23);
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) codes |= (PAIRED ? q4_encode2(x[i], x[i + 4], scale) : q4_encode2(x[2 * i], x[2 * i + 1], scale)) << (8 * i);
    return any ? 0u : codes;
}

// ---- entries in: four lanes take one group of 32 dims of one (row, head), keys and values.  What a lane has to wait for in turn (row numbers,
// then the table, then the stores) is a chain of latencies: keys and values are requested before it, eight of each to a lane.
// Four rows lie side by side in a wave: where they are four tokens of a page that share their values' dwords (pieces of prompts), the lanes exchange bytes and store whole
// dwords.  7936 rows of 8 heads in fp32 (75 MB): 17 us, 21.5 byte by byte, 37 with two values to a lane, requested behind the chain.
struct Kv4Line { int row, h, g, l, r, first; };
__device__ __forceinline__ Kv4Line kv4_line(int hkv, int groups) {
    const uint32_t item = (blockIdx.x * 256 + threadIdx.x) >> 2, four = item / groups;       // [row / 4][head][row % 4][group]
    Kv4Line t;
    t.l = threadIdx.x & 3, t.g = (int)(item % groups), t.r = (int)(four & 3);
    t.h = (int)((four >> 2) % hkv), t.row = (int)((four >> 2) / hkv * 4) + t.r;
    t.first = (threadIdx.x & 63) - t.r * 4 * groups;        // the lane of row % 4 = 0
    return t;
}
// all four rows exist (`is`) and their slots share the values' dwords; every lane of the wave takes part
__device__ __forceinline__ bool kv4_together(const Kv4Line& t, int groups, bool is, int b, int s) {
    const int b0 = __shfl(b, t.first), s0 = __shfl(s, t.first);
    const uint64_t fits = __ballot(is && b == b0 && s == s0 + t.r && (s0 & 3) == 0), four = 1ull | 1ull << 4 * groups | 1ull << 8 * groups | 1ull << 12 * groups;
    return ((fits >> t.first) & four) == four;
}
// byte i of row r's lane <-> byte r of row i's lane
__device__ __forceinline__ uint32_t kv4_exchange(const Kv4Line& t, int groups, uint32_t x) {
    uint32_t y = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) y |= (((uint32_t)__shfl((int)x, t.first + i * 4 * groups) >> (8 * t.r)) & 255u) << (8 * i);
    return y;
}
template <typename T>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4Cache c, int hd, const T* __restrict__ k, int64_t k_row, int64_t k_head, const T* __restrict__ v,
                                                         int64_t v_row, int64_t v_head, const int* __restrict__ seq, const int* __restrict__ slot,
                                                         const int* __restrict__ position, int rows, Kv4Book book) {
    const int groups = hd / 32;
    const Kv4Line at = kv4_line(c.hkv, groups);
    const int l = at.l, g = at.g, h = at.h, row = at.row;
    float kx[8] = {}, vx[8] = {};
    int b = -1, s = -1;
    if (row < rows) {
        b = seq[row], s = slot[row];
        const T* kr = k + row * k_row + h * k_head + g * 32 + 8 * l;
        const T* vr = v + row * v_row + h * v_head + g * 32 + 4 * l;
        kv4_load4(kr, kx);
        kv4_load4(kr + 4, kx + 4);
        kv4_load4(vr, vx);
        kv4_load4(vr + 16, vx + 4);
    }
    uint8_t* block = nullptr;
    if ((unsigned)b < (unsigned)c.batch && (unsigned)s < (unsigned)c.max_pages * KV4_PAGE) block = kv4_page(c, hd, b, s / KV4_PAGE, h);
    const bool together = kv4_together(at, groups, block != nullptr, b, s);
    int ke, ve;
    const uint32_t kc = kv4_encode8<false>(kx, ke), vc = kv4_encode8<true>(vx, ve), vc4 = kv4_exchange(at, groups, vc);
    if (!block) return;
    const int t = s % KV4_PAGE;
    *reinterpret_cast<uint32_t*>(block + kv4_key_at(hd, t, g * 32 + 8 * l)) = kc;
    if (together) *reinterpret_cast<uint32_t*>(block + kv4_val_at(hd, t & ~3, g, 4 * l + at.r)) = vc4;
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) block[kv4_val_at(hd, t, g, 4 * l + i)] = (uint8_t)(vc >> (8 * i));
    if (l == 0) {
        block[kv4_key_scale_at(hd, t, g)] = (uint8_t)ke;
        block[kv4_val_scale_at(hd, t, g)] = (uint8_t)ve;
        if (g == 0 && book.scores) book.scores[b * book.score_b + h * book.score_h + s] = 0.f;
        if (g == 0 && book.pos) book.pos[b * book.pos_b + h * book.pos_h + s] = position[row];
    }
}

// ---- entries out: [rows][heads][hd], contiguous; a row that names no entry of the cache gives zeros.  The lanes as above.
template <typename T> __device__ __forceinline__ void kv4_store4(T* p, const uint32_t a, const uint32_t b) {      // two pairs of bf16
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(p) = make_uint2(a, b);
    else *reinterpret_cast<float4*>(p) = make_float4(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u), __uint_as_float(b << 16), __uint_as_float(b & 0xFFFF0000u));
}
template <typename T>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Cache c, int hd, const int* __restrict__ seq, const int* __restrict__ slot, int rows,
                                                       T* __restrict__ k, T* __restrict__ v) {
    const int groups = hd / 32;
    const Kv4Line at = kv4_line(c.hkv, groups);
    const int l = at.l, g = at.g, h = at.h, row = at.row;
    const int b = row < rows ? seq[row] : -1, s = row < rows ? slot[row] : -1, t = s % KV4_PAGE;
    const uint8_t* block = nullptr;
    if ((unsigned)b < (unsigned)c.batch && (unsigned)s < (unsigned)c.max_pages * KV4_PAGE) block = kv4_page(c, hd, b, s / KV4_PAGE, h);
    const bool together = kv4_together(at, groups, block != nullptr, b, s);
    uint32_t kc = 0, vc = 0;
    int ke = 0, ve = 0;
    if (block) {
        kc = *reinterpret_cast<const uint32_t*>(block + kv4_key_at(hd, t, g * 32 + 8 * l));
        ke = block[kv4_key_scale_at(hd, t, g)];
        ve = block[kv4_val_scale_at(hd, t, g)];
        if (together) vc = *reinterpret_cast<const uint32_t*>(block + kv4_val_at(hd, t & ~3, g, 4 * l + at.r));
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) vc |= (uint32_t)block[kv4_val_at(hd, t, g, 4 * l + i)] << (8 * i);
    }
    const uint32_t vc4 = kv4_exchange(at, groups, vc);
    if (row >= rows) return;
    u32x4_t kk = {}, vv = {};
    if (block) kk = q4_decode8(kc, (uint32_t)ke << 23), vv = q4_decode8(together ? vc4 : vc, (uint32_t)ve << 23);
    const int64_t o = ((int64_t)row * c.hkv + h) * hd + g * 32;
    kv4_store4(k + o + 8 * l, kk[0], kk[1]);
    kv4_store4(k + o + 8 * l + 4, kk[2], kk[3]);
    // pairs (m, m + 16): the low halves are dims 4 l .. + 3, the high ones those 16 further on
    kv4_store4(v + o + 4 * l, __builtin_amdgcn_perm(vv[1], vv[0], 0x05040100u), __builtin_amdgcn_perm(vv[3], vv[2], 0x05040100u));
    kv4_store4(v + o + 16 + 4 * l, __builtin_amdgcn_perm(vv[1], vv[0], 0x07060302u), __builtin_amdgcn_perm(vv[3], vv[2], 0x07060302u));
}

// ---- attention
// what becomes of the weights in a launch of the attention: none are asked for; it adds them to the scores; it leaves the logarithms that they are taken with
enum { KV4_NO_WEIGHTS, KV4_WEIGHTS, KV4_LOGS };
struct Kv4Attn {
    Kv4Cache c;
    const void* q;
    int64_t q_row, q_head;
    const int* row_start;   // [batch + 1]; null: row b is sequence b's
    int total_rows, max_rows, heads, group;
    float factor;           // |scale|; 1 where q is multiplied by it
    float factor2;          // the same * log2(e): exponents are taken to the base 2; finite, never 0
    float slack;            // 8 / factor2, finite: a score may pass the running maximum by so much
    bool negative;          // scale < 0: q changes its sign instead
    bool plain;             // scale is 0, infinite or NaN: q is multiplied by it, so that -inf means "not seen" and nothing else (0 times an infinite score is NaN)
    float scale;
    void* out;
    int64_t o_row, o_head;
    float* lse;             // [rows][heads] or null
    float2* dealt;          // kv4_dealt of every row and head, for the kernels that add the weights afterwards (KV4_LOGS), or null
    int max_kv, tiles, split, splits, hd;
    bool by_length;         // the blocks of the longest sequences go first
    float* part_o;          // [rows][heads][splits][hd], unnormalised
    float2* part_ml;        // [rows][heads][splits]: maximum, sum
    Kv4Book book;
    int w_cols, w_groups;   // attention weights: the columns are dealt in groups of w_cols, at most w_groups of them
    int64_t w_slots;        // of a part below
    float* part_w;          // [w_groups][batch][kv heads][w_slots]: a group's weight of each entry
};
// rows of sequence b: the first one and how many; entries it has
__device__ __forceinline__ void kv4_rows(const Kv4Attn& a, int b, int& r0, int& count, int& n) {
    r0 = b;
    count = b < a.total_rows ? 1 : 0;
    if (a.row_start) {
        r0 = min(max(a.row_start[b], 0), a.total_rows);
        count = min(min(max(a.row_start[b + 1], r0), a.total_rows) - r0, a.max_rows);
    }
    n = min(min(max(a.c.kv_len[b], 0), a.max_kv), a.c.max_pages * KV4_PAGE);
}

// parts that the entries of a sequence make
__device__ __forceinline__ int kv4_parts(const Kv4Attn& a, int n) { return a.splits == 1 ? 1 : (n - 1) / a.split + 1; }

// Sequences of unlike lengths make blocks of unlike times; where the blocks do not all run at once the longest go first, so that the last to start are short
// (16 sequences of unlike lengths and rows, 72B heads: fp32 205 -> 173 us, bf16 147 -> 126).  The i-th sequence in that order, among every 64 together: the same for all lanes of a
// whole wave, about a microsecond at a block's start.
__device__ __forceinline__ int kv4_by_length(const Kv4Attn& a, int i) {
    if (!a.by_length) return i;
    const int lane = threadIdx.x & 63, first = i & ~63;
    const int len = first + lane < a.c.batch ? min(max(a.c.kv_len[first + lane], 0), 1 << 24) : -1;
    const int key = len * 64 + 63 - lane;                   // no two alike
    int before = 0;
#pragma unroll 8
    for (int u = 0; u < 64; ++u) before += __builtin_amdgcn_readlane(key, u) > key;
    return first + __builtin_ctzll(__ballot(before == (i & 63)));
}

template <int HD> struct Kv4Keys { typename u32vec<HD / 32>::type w[4]; uint32_t scale[4]; };
template <int HD> struct Kv4Vals { typename u32vec<HD / 32>::type w[4], scale[4]; };

// the blocks of the four pages of a chunk; bit p of `there` is clear where the table names no page of the pool
template <int HD> __device__ __forceinline__ void kv4_pages(const Kv4Cache& c, int seq, int head, int slot0, const uint8_t* page[4], int& there) {
    there = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int id = __builtin_amdgcn_readfirstlane(c.table[(int64_t)seq * c.max_pages + min(slot0 / KV4_PAGE + p, c.max_pages - 1)]);
        const bool ok = (unsigned)id < (unsigned)c.n_pages;
        there |= ok << p;
        page[p] = c.pool + ((int64_t)(ok ? id : 0) * c.hkv + head) * kv4_block(HD);
    }
}
template <int HD> __device__ __forceinline__ void kv4_load_keys(const uint8_t* const page[4], int lane, Kv4Keys<HD>& k) {
    typedef typename u32vec<HD / 32>::type V;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        k.w[p] = reinterpret_cast<const V*>(page[p])[lane];
        k.scale[p] = page[p][16 * HD + (lane >> 4) * (HD / 4) / 32 * 16 + (lane & 15)];
    }
}
template <int HD> __device__ __forceinline__ void kv4_load_vals(const uint8_t* const page[4], int lane, Kv4Vals<HD>& v) {
    typedef typename u32vec<HD / 32>::type V;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        v.w[p] = reinterpret_cast<const V*>(page[p] + 8 * HD)[lane];
        v.scale[p] = reinterpret_cast<const V*>(page[p] + 16 * HD + HD / 2)[lane >> 4];
    }
}
// what q is multiplied by, beside factor2
__device__ __forceinline__ void kv4_scale_q(const Kv4Attn& a, float x[8]) {
    if (a.negative)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = -x[i];
    if (a.plain)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= a.scale;
}
// q of one tile of 16 columns as B operands [HD/32][plane]; column c of a (sequence, kv head) is row c / group, head c % group
template <typename T, int HD, int PLANES>
__device__ __forceinline__ void kv4_load_q(const Kv4Attn& a, int r0, int count, int head, int col, int lane, u32x4_t q[HD / 32][PLANES]) {
    const int r = col / a.group, g = col % a.group;
    // a column beyond the rows repeats the last one; its results are not used
    const T* p = static_cast<const T*>(a.q) + (int64_t)(r0 + min(r, count - 1)) * a.q_row + (int64_t)(head * a.group + g) * a.q_head + (lane >> 4) * (HD / 4);
    float x[HD / 32][8];
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) kv4_load8(p + j * 8, x[j]);
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) {
        kv4_scale_q(a, x[j]);
        q4_operand<PLANES>(x[j], q[j]);
    }
}
// scores of one page: rows (tokens) 4 (lane / 16) + i, column lane % 16
template <int HD, int PLANES>
__device__ __forceinline__ f32x4_t kv4_scores(const Kv4Keys<HD>& k, int p, const u32x4_t q[HD / 32][PLANES]) {
    f32x4_t s = {};
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) {
        const u32x4_t m = q4_decode8(k.w[p][j], k.scale[p] << 23);
#pragma unroll
        for (int x = 0; x < PLANES; ++x) s = q4_mfma(m, q[j][x], s);
    }
    return s;
}
// one group's values of two pages (w: bytes, s: scale bytes of four tokens) as the A operands of its dims 0 .. 15 (lo) and 16 .. 31 (hi)
__device__ __forceinline__ void kv4_pair_operands(uint32_t w0, uint32_t s0, uint32_t w1, uint32_t s1, u32x4_t& lo, u32x4_t& hi) {
    const uint32_t w[2] = {w0, w1}, s[2] = {s0, s1};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t c0 = q4_decode2<0>(w[e], q4_scale_at<0>(s[e])), c1 = q4_decode2<1>(w[e], q4_scale_at<1>(s[e]));
        const uint32_t c2 = q4_decode2<2>(w[e], q4_scale_at<2>(s[e])), c3 = q4_decode2<3>(w[e], q4_scale_at<3>(s[e]));
        lo[2 * e] = __builtin_amdgcn_perm(c1, c0, 0x05040100u);
        lo[2 * e + 1] = __builtin_amdgcn_perm(c3, c2, 0x05040100u);
        hi[2 * e] = __builtin_amdgcn_perm(c1, c0, 0x07060302u);
        hi[2 * e + 1] = __builtin_amdgcn_perm(c3, c2, 0x07060302u);
    }
}
// the scale bytes of four tokens of which the first `left` are to be kept
__device__ __forceinline__ uint32_t kv4_keep(int left) { return left >= 4 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << (8 * left)) - 1; }
// bit 8 i + 7: byte i is 255 and i >= from
__device__ __forceinline__ uint32_t kv4_nan_marks(uint32_t s, int from) {
    const uint32_t look = from <= 0 ? 0xFFFFFFFFu : from >= 4 ? 0u : 0xFFFFFFFFu << (8 * from);
    return ((s & 0x7F7F7F7Fu) + 0x01010101u) & s & 0x80808080u & look;
}
// An entry that reads as NaN must not reach the columns that do not see it (as 0 * NaN).  Such groups among the entries from slot `safe` on
// are taken out of the product (scale byte 0), and the sums of the columns that do see the entry become NaN instead.
template <int HD>
__device__ __forceinline__ void kv4_nan_values(Kv4Vals<HD>& v, int slot0, int safe, int limit, f32x4_t (&o)[HD / 16]) {
    const int quad = (threadIdx.x & 63) >> 4;
    uint32_t any = 0;
    uint32_t marks[4][HD / 32];                             // bit 8 i + 7: token i of the quad is NaN in this group
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int from = safe - (slot0 + p * KV4_PAGE + quad * 4);
#pragma unroll
        for (int g = 0; g < HD / 32; ++g) {
            marks[p][g] = kv4_nan_marks(v.scale[p][g], from);
            any |= marks[p][g];
        }
    }
    if (!__any(any != 0)) return;
    // how many such entries each column sees: a product of marks (rows: any dim) and of what is seen, like the one of values and probabilities
    f32x4_t seen[HD / 32] = {};
#pragma unroll
    for (int p = 0; p < 4; p += 2) {
        u32x4_t mark[HD / 32];
#pragma unroll
        for (int g = 0; g < HD / 32; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t m = marks[p + e / 2][g] >> (16 * (e & 1));
                mark[g][e] = (m & 0x80u ? 0x3F80u : 0u) | (m & 0x8000u ? 0x3F800000u : 0u);
            }
        u32x4_t sees;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int slot = slot0 + (p + e / 2) * KV4_PAGE + quad * 4 + 2 * (e & 1);
            sees[e] = (slot < limit ? 0x3F80u : 0u) | (slot + 1 < limit ? 0x3F800000u : 0u);
        }
#pragma unroll
        for (int g = 0; g < HD / 32; ++g) seen[g] = q4_mfma(mark[g], sees, seen[g]);
    }
#pragma unroll
    for (int g = 0; g < HD / 32; ++g) {
        const float add = seen[g][0] > 0.f ? __uint_as_float(0x7FC00000u) : 0.f;
        o[2 * g] += add;
        o[2 * g + 1] += add;
    }
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int g = 0; g < HD / 32; ++g) v.scale[p][g] &= ~((marks[p][g] >> 7) * 255u);
}

// The weight 2^(factor2 (s - top)) of a score, or of what was gathered under another maximum.  The difference is formed first and is 0 at the maximum.  (factor2 s - fl(factor2 top) in one
// multiply-add keeps the rounding of the second product: beyond 2^31 that is 128 and more, and the weights of the largest scores themselves were 0 or infinite.)
__device__ __forceinline__ float kv4_weight(const Kv4Attn& a, float s, float base) { return __builtin_amdgcn_exp2f((s - base) * a.factor2); }
__device__ __forceinline__ float kv4_base(float top) { return top == -INFINITY ? 0.f : top; }
__device__ __forceinline__ float kv4_lse(const Kv4Attn& a, float top, float total) { return total == 0.f ? -INFINITY : kv4_base(top) * a.factor + logf(total); }
// What a column's weights are taken with: its maximum, and the logarithm to the base 2 of the sum that they are divided by (in one number, a large maximum would swallow the logarithm).  A column
// that deals out nothing, because it sees nothing or all its scores are -inf, has +inf: its weights are 0 (with -inf, the logarithm of its sum, those of the scores -inf were NaN).
__device__ __forceinline__ float2 kv4_dealt(float top, float total) { return make_float2(kv4_base(top), total == 0.f ? INFINITY : log2f(total)); }
__device__ __forceinline__ float kv4_dealt_weight(const Kv4Attn& a, float s, float2 dealt) { return __builtin_amdgcn_exp2f(__builtin_fmaf(s - dealt.x, a.factor2, -dealt.y)); }
// what a column has gathered, for the join: rows (dims) 4 quad + i of every block d of 16 dims, column lane % 16
template <typename T, int WEIGHTS>
__device__ __forceinline__ void kv4_finish(const Kv4Attn& a, int64_t row, int qh, int dim, bool first, f32x4_t acc, float top, float total, int parts) {
    if (parts > 1) {
        const int64_t at = (row * a.heads + qh) * a.splits + blockIdx.z;
        *reinterpret_cast<f32x4_t*>(a.part_o + at * a.hd + dim) = acc;
        if (first) a.part_ml[at] = make_float2(top, total);
        return;
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    T* dst = static_cast<T*>(a.out) + row * a.o_row + qh * a.o_head + dim;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2_any_t*>(dst) = u32x2_t{f2bf2(acc[0] * inv, acc[1] * inv), f2bf2(acc[2] * inv, acc[3] * inv)};
    else *reinterpret_cast<f32x4_any_t*>(dst) = acc * inv;
    if (first && a.lse) a.lse[row * a.heads + qh] = kv4_lse(a, top, total);
    if (WEIGHTS == KV4_LOGS && first) a.dealt[row * a.heads + qh] = kv4_dealt(top, total);
}

// One chunk against one tile of columns: scores q.k (masked where `whole` is false), new maximum, probabilities in place of the scores; what was gathered is scaled.
// factor2 > 0; top is a score.
template <int NB>
__device__ __forceinline__ void kv4_softmax(f32x4_t s[4], bool whole, int there, int slot0, int limit, int quad, const Kv4Attn& a, float& top, float& sum, f32x4_t o[NB]) {
    if (!whole) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int end_p = (there >> p) & 1 ? limit : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) s[p][i] = slot0 + p * KV4_PAGE + quad * 4 + i < end_p ? s[p][i] : -INFINITY;
        }
    }
    float best = -INFINITY;
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) best = fmaxf(best, s[p][i]);
    best = rows4_max(best);
    best = fmaxf(top, best);
    // The maximum moves only where a probability of some column of the tile would pass 2^8 (up to there they lose nothing in 32 bits): seldom after the first chunks.
    if (__any(best > top + a.slack)) {
        const float scale = kv4_weight(a, top, kv4_base(best));
        sum *= scale;
#pragma unroll
        for (int d = 0; d < NB; ++d) o[d] *= scale;
        top = best;
    }
    const float base = kv4_base(top);
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[p][i] = kv4_weight(a, s[p][i], base);
            sum += s[p][i];
        }
}
// Probabilities of two pages as operands: the sum of two bf16 numbers (16 bits) where the result is rounded to bf16, of three (all 24 bits) where it is fp32.
template <int PP> __device__ __forceinline__ void kv4_weights(const f32x4_t s0, const f32x4_t s1, u32x4_t w[PP]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = i < 2 ? s0[2 * i] : s1[2 * i - 4], y = i < 2 ? s0[2 * i + 1] : s1[2 * i - 3];
        if constexpr (PP == 2) {
            uint32_t hi, lo;
            split2(x, y, hi, lo);
            w[0][i] = hi;
            w[1][i] = lo;
        } else {
            // cut as in q4_cut3; a probability is at most 2^8 (the maximum moves in steps) and its rounding, or NaN, whose first part is NaN
            const float x1 = x - __uint_as_float(__float_as_uint(x) & 0xFFFF0000u), y1 = y - __uint_as_float(__float_as_uint(y) & 0xFFFF0000u);
            const float x2 = x1 - __uint_as_float(__float_as_uint(x1) & 0xFFFF0000u), y2 = y1 - __uint_as_float(__float_as_uint(y1) & 0xFFFF0000u);
            w[0][i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
            w[1][i] = __builtin_amdgcn_perm(__float_as_uint(y1), __float_as_uint(x1), 0x07060302u);
            w[2][i] = __builtin_amdgcn_perm(__float_as_uint(y2), __float_as_uint(x2), 0x07060302u);
        }
    }
}

// weights of the slots from `slot` on, of which the column sees those below `end`
__device__ __forceinline__ void kv4_seen_weights(f32x4_t& w, int slot, int end) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = slot + i < end ? w[i] : 0.f;
}
// Attention weights of a chunk's entries (rows of the scores) from one tile of columns, whose sums are known: `dealt` is their kv4_dealt, (0, +inf) for a
// column that does not exist.  WHOLE: every column sees every entry.
template <int HD, int PLANES>
__device__ __forceinline__ void kv4_add_weights(const Kv4Keys<HD>& k, const u32x4_t q[HD / 32][PLANES], bool whole, int there, int slot0, int limit, const Kv4Attn& a,
                                                float2 dealt, f32x4_t weight[4]) {
    const int quad = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const f32x4_t s = kv4_scores<HD, PLANES>(k, p, q);
        f32x4_t w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = kv4_dealt_weight(a, s[i], dealt);
        if (!whole) kv4_seen_weights(w, slot0 + p * KV4_PAGE + quad * 4, (there >> p) & 1 ? limit : 0);
        weight[p] += w;
    }
}
// Each of the 16 lanes of a quad keeps one of its 16 entries: entry 4 p + i.  Its place among the scores, or -1
__device__ __forceinline__ int kv4_score_slot(int slot0, int n, int there) {
    const int lane = threadIdx.x & 63, slot = slot0 + (lane & 12) * 4 + (lane >> 4) * 4 + (lane & 3);
    return slot < n && ((there >> ((lane & 15) >> 2)) & 1) ? slot : -1;
}
// One step of the sum over 16 lanes of 2 N values each: lanes whose numbers differ in a bit (CTRL pairs them) keep N values each and give the other N away
template <int CTRL, int N> __device__ __forceinline__ void kv4_halve(float v[16], bool upper) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float keep = upper ? v[j + N] : v[j], give = upper ? v[j] : v[j + N];
        v[j] = keep + __uint_as_float(dpp_move<CTRL>(__float_as_uint(give)));
    }
}
// sum over the 16 columns of each entry, for the lane that keeps it: 15 additions instead of the 64 of a sum of every entry for every lane
__device__ __forceinline__ float kv4_sum_weights(const f32x4_t weight[4]) {
    const int l = threadIdx.x;
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = weight[e / 4][e % 4];
    kv4_halve<0x140, 8>(v, l & 8);       // row_mirror: the lane 15 - l
    kv4_halve<0x141, 4>(v, l & 4);       // row_half_mirror: 7 - l of its half
    kv4_halve<0x4E, 2>(v, l & 2);        // quad_perm [2,3,0,1]
    kv4_halve<0xB1, 1>(v, l & 1);        // quad_perm [1,0,3,2]
    return v[0];
}

// Few columns (single tokens, verification of a few): a block owns a tile of 16 columns of one (sequence, kv head) and one part of its entries, of which
// its waves take chunks of 64 in turn, each with its own running maximum and sum; they are joined in LDS.  The next chunk's bytes are requested before
// this one is worked on, the table entries one chunk earlier still.  A second tile reads the entries again, from L2 (with
// both tiles in one wave's registers 28 columns of 64 sequences took a quarter longer).
// 256 sequences of 4096 .. 8192 entries, 7B heads: 859 MB in 163 .. 167 us, 5.2 TB/s, what a copy reaches (8 us more in the order of the sequences); 480 vector
// and 48 matrix instructions per chunk keep a SIMD busy for two thirds of that.  Without the requests ahead, or with them dropped for a third wave per SIMD, it
// took 5 and 10 % longer.  At 128 dims the fp32 instances spill 5 of 256 registers.
// KV4_WEIGHTS: the tile is the only one and its entries are not split, so the block knows the sums of its columns and adds the weights itself, with the keys
// once more.  Against two launches: 64 x 4 of 64 .. 512 entries 12.5 us and 16.9, of 128 .. 5120 47 and 47 (fp32 57 and 61; 256 blocks, so the longest sequence
// decides); where the blocks go in rounds the weights' own, finer blocks are ahead (256 x 4 of 512 .. 4096: 118 and 104).
template <typename T, int HD, int PLANES, int WEIGHTS>
__global__ __launch_bounds__(512, 2) void kv4_attn_kernel(Kv4Attn a) {
    constexpr int G = HD / 32, PP = PLANES == 1 ? 2 : 3, WAVES = 8;
    __shared__ __align__(16) float lds_o[WAVES][G * 2][64][4];
    __shared__ float lds_ml[WAVES][2][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, quad = lane >> 4;
    const int b = kv4_by_length(a, blockIdx.x / a.c.hkv), head = blockIdx.x % a.c.hkv, col0 = blockIdx.y * 16, col = col0 + (lane & 15);
    int r0, count, n;
    kv4_rows(a, b, r0, count, n);
    const int cols = count * a.group, parts = kv4_parts(a, n);
    if (col0 >= cols || (int)blockIdx.z >= parts) return;
    const int begin = blockIdx.z * a.split, end = min(begin + a.split, n - (count - 1 - (min(cols, col0 + 16) - 1) / a.group));
    const int safe = min(end, n - (count - 1 - col0 / a.group));      // below: every column sees every entry
    const int limit = min(end, col < cols ? n - (count - 1 - col / a.group) : 0);      // entries seen by the column's row: slots below
    const int step = waves * KV4_CHUNK;

    Kv4Keys<HD> k[2];
    Kv4Vals<HD> v[2];
    const uint8_t* page[2][4];
    int there[2];
    int slot0 = begin + wave * KV4_CHUNK;
    u32x4_t q[G][PLANES];
    f32x4_t o[2 * G] = {};
    float top = -INFINITY, sum = 0.f;
    auto work = [&](Kv4Keys<HD>& k_, Kv4Vals<HD>& v_, int there_) {
        const bool whole = slot0 + KV4_CHUNK <= safe && there_ == 15;
        if (!whole) {
            // Values that are not there, or not seen by all columns: what lies behind the last entry may read as NaN, and 0 * NaN is NaN.
            // Their scales are cleared.
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const uint32_t keep = kv4_keep((there_ >> p) & 1 ? end - (slot0 + p * KV4_PAGE + quad * 4) : 0);
#pragma unroll
                for (int g = 0; g < G; ++g) v_.scale[p][g] &= keep;
            }
            if (slot0 + KV4_CHUNK > safe) kv4_nan_values<HD>(v_, slot0, safe, limit, o);
        }
        f32x4_t s[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) s[p] = kv4_scores<HD, PLANES>(k_, p, q);
        kv4_softmax<2 * G>(s, whole, there_, slot0, limit, quad, a, top, sum, o);
#pragma unroll
        for (int p = 0; p < 4; p += 2) {
            u32x4_t w[PP];
            kv4_weights<PP>(s[p], s[p + 1], w);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                u32x4_t lo, hi;
                kv4_pair_operands(v_.w[p][g], v_.scale[p][g], v_.w[p + 1][g], v_.scale[p + 1][g], lo, hi);
#pragma unroll
                for (int x = 0; x < PP; ++x) {
                    o[2 * g] = q4_mfma(lo, w[x], o[2 * g]);
                    o[2 * g + 1] = q4_mfma(hi, w[x], o[2 * g + 1]);
                }
            }
        }
    };
    kv4_pages<HD>(a.c, b, head, slot0, page[0], there[0]);
    kv4_load_keys<HD>(page[0], lane, k[0]);
    kv4_load_vals<HD>(page[0], lane, v[0]);
    kv4_pages<HD>(a.c, b, head, slot0 + step, page[1], there[1]);
    kv4_load_q<T, HD, PLANES>(a, r0, count, head, col, lane, q);
    while (slot0 < end) {
        kv4_load_keys<HD>(page[1], lane, k[1]);
        kv4_load_vals<HD>(page[1], lane, v[1]);
        const int there1 = there[1];
        kv4_pages<HD>(a.c, b, head, slot0 + 2 * step, page[0], there[1]);
        work(k[0], v[0], there[0]);
        slot0 += step;
        if (slot0 >= end) break;
        kv4_load_keys<HD>(page[0], lane, k[0]);
        kv4_load_vals<HD>(page[0], lane, v[0]);
        there[0] = there[1];
        kv4_pages<HD>(a.c, b, head, slot0 + 2 * step, page[1], there[1]);
        work(k[1], v[1], there1);
        slot0 += step;
    }
    sum = rows4_sum(sum);
    if (quad == 0) lds_ml[wave][0][lane] = top, lds_ml[wave][1][lane] = sum;
#pragma unroll
    for (int d = 0; d < 2 * G; ++d) *reinterpret_cast<f32x4_t*>(lds_o[wave][d][lane]) = o[d];
    __syncthreads();
    for (int d = wave; d < 2 * G; d += waves) {
        const int c = lane & 15;
        float best = -INFINITY, total = 0.f;
        for (int w = 0; w < waves; ++w) best = fmaxf(best, lds_ml[w][0][c]);
        const float base = kv4_base(best);
        f32x4_t acc = {};
        for (int w = 0; w < waves; ++w) {
            const float scale = kv4_weight(a, lds_ml[w][0][c], base);
            total += scale * lds_ml[w][1][c];
            acc += scale * *reinterpret_cast<const f32x4_t*>(lds_o[w][d][lane]);
        }
        if (col < cols) kv4_finish<T, WEIGHTS>(a, r0 + col / a.group, head * a.group + col % a.group, d * 16 + quad * 4, d == 0 && quad == 0, acc, best, total, parts);
    }
    if constexpr (WEIGHTS == KV4_WEIGHTS) {
        float best = -INFINITY, total = 0.f;
        for (int w = 0; w < waves; ++w) best = fmaxf(best, lds_ml[w][0][lane & 15]);
        const float base = kv4_base(best);
        for (int w = 0; w < waves; ++w) total += kv4_weight(a, lds_ml[w][0][lane & 15], base) * lds_ml[w][1][lane & 15];
        const float2 dealt = kv4_dealt(best, col < cols ? total : 0.f);
        float* scores = a.book.scores + b * a.book.score_b + head * a.book.score_h;
        slot0 = begin + wave * KV4_CHUNK;
        kv4_pages<HD>(a.c, b, head, slot0, page[0], there[0]);
        kv4_load_keys<HD>(page[0], lane, k[0]);
        kv4_pages<HD>(a.c, b, head, slot0 + step, page[1], there[1]);
        for (; slot0 < end; slot0 += step) {
            kv4_load_keys<HD>(page[1], lane, k[1]);
            const int slot = kv4_score_slot(slot0, end, there[0]), there1 = there[1];
            const float before = slot >= 0 ? scores[slot] : 0.f;
            kv4_pages<HD>(a.c, b, head, slot0 + 2 * step, page[1], there[1]);
            f32x4_t weight[4] = {};
            kv4_add_weights<HD, PLANES>(k[0], q, slot0 + KV4_CHUNK <= safe && there[0] == 15, there[0], slot0, limit, a, dealt, weight);
            const float sum_ = kv4_sum_weights(weight);
            if (slot >= 0) scores[slot] = before + sum_;
            k[0] = k[1];
            there[0] = there1;
        }
    }
}

// Many columns (steps and prompts): a block of four waves owns four tiles of columns of one (sequence, kv head) and one part of its entries.  All its waves
// need every key and value, so a chunk is decoded once for the block, into operands in LDS, a share by each wave; the next chunk's bytes are on their way in the meantime.
// Several blocks per CU cover each other's waits: 16 sequences of 17 .. 128 rows and 512 .. 2560 entries, 72B heads, fp32: 131 .. 138 us, by which rows meet which
// lengths, 0.95 executed PFLOP/s (three bf16 parts of q and of the weights) of the 1.22 that a plain product reaches; bf16 102 .. 106 us.  (4 % more in fp32 with the sums of a
// tile one after the other, 18 % in the order of the sequences.)  Two tiles to a wave, for half the reads of LDS, take two waves a SIMD: fp32 26 %, bf16 7 % more.
// The fp32 instance at 128 dims spills 10 of 168 registers, reloaded in every chunk.
template <typename T, int HD, int PLANES, int WEIGHTS>
__global__ __launch_bounds__(256, 3) void kv4_attn_many_kernel(Kv4Attn a) {
    constexpr int G = HD / 32, PP = PLANES == 1 ? 2 : 3, NW = 4, COLS = 16 * NW;
    typedef typename u32vec<G>::type V;
    __shared__ u32x4_t lds_k[4 * G][64], lds_v[4 * G][64];              // keys [page][j], values [pair of pages][block of 16 dims]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quad = lane >> 4;
    const int id = blockIdx.x, head = id % a.c.hkv, col0 = id / a.c.hkv % a.tiles * COLS;
    const int b = kv4_by_length(a, id / a.c.hkv / a.tiles);
    int r0, count, n;
    kv4_rows(a, b, r0, count, n);
    const int cols = count * a.group, parts = kv4_parts(a, n);
    if (col0 >= cols || (int)blockIdx.z >= parts) return;
    const int begin = blockIdx.z * a.split, end = min(begin + a.split, n - (count - 1 - (min(cols, col0 + COLS) - 1) / a.group));
    const int safe = min(end, n - (count - 1 - col0 / a.group));
    const bool mine = col0 + wave * 16 < cols;              // some of this wave's columns exist
    const int col = col0 + wave * 16 + (lane & 15);
    const int limit = min(end, col < cols ? n - (count - 1 - col / a.group) : 0);
    u32x4_t q[G][PLANES];
    f32x4_t o[2 * G] = {};
    float top = -INFINITY, sum = 0.f;
    kv4_load_q<T, HD, PLANES>(a, r0, count, head, col, lane, q);
    // this wave's share of a chunk: its page's keys; the values of VS of the 2 G (pair of pages, group)
    constexpr int VS = 2 * G > NW ? 2 * G / NW : 1;
    const bool has_v = wave * VS < 2 * G;
    const int pair = min(wave * VS, 2 * G - 1) / G * 2, g0 = wave * VS % G;
    V raw_k;
    uint32_t raw_ks, raw_v[2][VS], raw_vs[2][VS];
    int there;
    auto request = [&](int slot0) {
        const uint8_t* page[4];
        kv4_pages<HD>(a.c, b, head, slot0, page, there);
        const uint8_t *pk = page[0], *pv[2] = {page[0], page[1]};
#pragma unroll
        for (int p = 1; p < 4; ++p) pk = wave == p ? page[p] : pk;
        if (pair) pv[0] = page[2], pv[1] = page[3];
        raw_k = reinterpret_cast<const V*>(pk)[lane];
        raw_ks = pk[16 * HD + quad * (HD / 4) / 32 * 16 + (lane & 15)];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t* v = reinterpret_cast<const uint32_t*>(pv[e] + 8 * HD) + lane * G + g0;
            const uint32_t* s = reinterpret_cast<const uint32_t*>(pv[e] + 16 * HD + HD / 2) + quad * G + g0;
#pragma unroll
            for (int g = 0; g < VS; ++g) raw_v[e][g] = v[g], raw_vs[e][g] = s[g];
        }
    };
    auto decode = [&](int slot0) {
#pragma unroll
        for (int j = 0; j < G; ++j) lds_k[wave * G + j][lane] = q4_decode8(raw_k[j], raw_ks << 23);
        if (!has_v) return;
        if (slot0 + KV4_CHUNK > safe || there != 15) {
            // as in the kernel above: what is not there, and NaN that not every column sees, is taken out of the product
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int first = slot0 + (pair + e) * KV4_PAGE + quad * 4;
                const uint32_t keep = kv4_keep((there >> (pair + e)) & 1 ? end - first : 0);
#pragma unroll
                for (int g = 0; g < VS; ++g) raw_vs[e][g] &= keep, raw_vs[e][g] &= ~((kv4_nan_marks(raw_vs[e][g], safe - first) >> 7) * 255u);
            }
        }
#pragma unroll
        for (int g = 0; g < VS; ++g) {
            u32x4_t lo, hi;
            kv4_pair_operands(raw_v[0][g], raw_vs[0][g], raw_v[1][g], raw_vs[1][g], lo, hi);
            lds_v[pair * G + 2 * (g0 + g)][lane] = lo;
            lds_v[pair * G + 2 * (g0 + g) + 1][lane] = hi;
        }
    };
    if (begin < end) request(begin);
    for (int slot0 = begin; slot0 < end; slot0 += KV4_CHUNK) {
        decode(slot0);
        const int there0 = there;
        __syncthreads();
        request(min(slot0 + KV4_CHUNK, end - 1));
        if (mine) {
            if (slot0 + KV4_CHUNK > safe) {                 // a NaN that some of the columns see
                const uint8_t* page[4];
                int there_;
                Kv4Vals<HD> v;
                kv4_pages<HD>(a.c, b, head, slot0, page, there_);
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    v.scale[p] = reinterpret_cast<const V*>(page[p] + 16 * HD + HD / 2)[quad];
                    const uint32_t keep = kv4_keep((there_ >> p) & 1 ? end - (slot0 + p * KV4_PAGE + quad * 4) : 0);
#pragma unroll
                    for (int g = 0; g < G; ++g) v.scale[p][g] &= keep;
                }
                kv4_nan_values<HD>(v, slot0, safe, limit, o);
            }
            // four sums side by side: a matrix instruction that waits for the one before it leaves the unit idle
            f32x4_t s[4] = {};
            u32x4_t k[2][4];
#pragma unroll
            for (int p = 0; p < 4; ++p) k[0][p] = lds_k[p * G][lane];
#pragma unroll
            for (int j = 0; j < G; ++j) {
                if (j + 1 < G)
#pragma unroll
                    for (int p = 0; p < 4; ++p) k[(j + 1) & 1][p] = lds_k[p * G + j + 1][lane];
#pragma unroll
                for (int x = 0; x < PLANES; ++x)
#pragma unroll
                    for (int p = 0; p < 4; ++p) s[p] = q4_mfma(k[j & 1][p], q[j][x], s[p]);
            }
            constexpr int AT = G == 1 ? 2 : 4, STEPS = 4 * G / AT;       // values: operands of a pair of pages, then those of the other
            u32x4_t v[2][AT];
#pragma unroll
            for (int d = 0; d < AT; ++d) v[0][d] = lds_v[d][lane];
            kv4_softmax<2 * G>(s, slot0 + KV4_CHUNK <= safe && there0 == 15, there0, slot0, limit, quad, a, top, sum, o);
            u32x4_t w[PP];
#pragma unroll
            for (int t = 0; t < STEPS; ++t) {
                if (t == 0) kv4_weights<PP>(s[0], s[1], w);
                if (t == STEPS / 2) kv4_weights<PP>(s[2], s[3], w);
                if (t + 1 < STEPS)
#pragma unroll
                    for (int d = 0; d < AT; ++d) v[(t + 1) & 1][d] = lds_v[(t + 1) * AT + d][lane];
#pragma unroll
                for (int x = 0; x < PP; ++x)
#pragma unroll
                    for (int d = 0; d < AT; ++d) o[(t * AT + d) % (2 * G)] = q4_mfma(v[t & 1][d], w[x], o[(t * AT + d) % (2 * G)]);
            }
        }
        __syncthreads();
    }
    sum = rows4_sum(sum);
    if (col >= cols) return;
#pragma unroll
    for (int d = 0; d < 2 * G; ++d)
        kv4_finish<T, WEIGHTS>(a, r0 + col / a.group, head * a.group + col % a.group, d * 16 + quad * 4, d == 0 && quad == 0, o[d], top, sum, parts);
}

// Joins the parts of the entries: 16 lanes per (row, head), HD/16 dims each.  The lanes read 16 parts' maxima and sums at once (one after the other they
// were a chain of latencies, 6 us for a handful of rows).
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_join_kernel(Kv4Attn a) {
    constexpr int N = HD / 16;
    const int l = threadIdx.x & 15;
    const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4;
    if (id >= (int64_t)a.c.batch * a.max_rows * a.heads) return;        // 16 lanes leave together
    const int qh = (int)(id % a.heads), r = (int)(id / a.heads % a.max_rows), b = (int)(id / a.heads / a.max_rows);
    int r0, count, n;
    kv4_rows(a, b, r0, count, n);
    const int parts = kv4_parts(a, n);
    if (r >= count || parts == 1) return;                   // a single part went to its place
    // (a row that sees nothing of the last part has an empty one there)
    const int64_t row = r0 + r, at = (row * a.heads + qh) * a.splits;
    float best = -INFINITY;
    for (int s = l; s < parts; s += 16) best = fmaxf(best, a.part_ml[at + s].x);
    best = row16_max(best);
    const float base = kv4_base(best);
    float total = 0.f, acc[N] = {};
    for (int s0 = 0; s0 < parts; s0 += 16) {
        float scale = 0.f;
        if (s0 + l < parts) {
            const float2 ml = a.part_ml[at + s0 + l];
            scale = kv4_weight(a, ml.x, base);
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
    if (l == 0 && a.lse) a.lse[row * a.heads + qh] = kv4_lse(a, best, total);
    if (l == 0 && a.dealt) a.dealt[row * a.heads + qh] = kv4_dealt(best, total);
}

// Attention weight per entry, added to the accumulated one: the scores are computed a second time (keys are half of the cache; storing a
// group's probabilities would move as many bytes), now with the final sum of every row.  A wave owns chunks of 64 entries of one (sequence, kv head): no atomics, one order.
template <typename T, int HD, int PLANES>
__global__ __launch_bounds__(256) void kv4_weight_kernel(Kv4Attn a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15;
    const int b = blockIdx.x / a.c.hkv, head = blockIdx.x % a.c.hkv;
    int r0, count, n;
    kv4_rows(a, b, r0, count, n);
    const int cols = count * a.group, step = gridDim.y * 4 * KV4_CHUNK;
    const int safe = n - (count - 1);                       // every row sees the slots below
    int slot0 = (blockIdx.y * 4 + wave) * KV4_CHUNK;
    if (slot0 >= n || cols == 0) return;
    const uint8_t* page[4];
    int there, next;
    Kv4Keys<HD> k, k1;
    u32x4_t q[HD / 32][PLANES];
    kv4_pages<HD>(a.c, b, head, slot0, page, there);
    kv4_load_keys<HD>(page, lane, k);
    const int limit = col < cols ? n - (count - 1 - col / a.group) : 0;
    const float2 dealt = col < cols ? a.dealt[(int64_t)(r0 + col / a.group) * a.heads + head * a.group + col % a.group] : kv4_dealt(0.f, 0.f);
    kv4_load_q<T, HD, PLANES>(a, r0, count, head, col, lane, q);
    float* scores = a.book.scores + b * a.book.score_b + head * a.book.score_h;
    for (; slot0 < n; slot0 += step) {
        kv4_pages<HD>(a.c, b, head, slot0 + step, page, next);
        kv4_load_keys<HD>(page, lane, k1);
        const int slot = kv4_score_slot(slot0, n, there);
        const float before = slot >= 0 ? scores[slot] : 0.f;
        f32x4_t weight[4] = {};
        kv4_add_weights<HD, PLANES>(k, q, slot0 + KV4_CHUNK <= safe && there == 15, there, slot0, limit, a, dealt, weight);
        const float mine = kv4_sum_weights(weight);
        if (slot >= 0) scores[slot] = before + mine;
        k = k1;
        there = next;
    }
}

// The same for more than one tile of columns: a wave keeps its chunk's keys decoded and goes over the tiles, whose q the block cuts into operands in LDS, one
// (tile, 32 dims) by each wave, the next ones while these are worked on.  Where blocks are few or unlike the columns are dealt in groups, whose weights the next
// kernel adds up.  16 sequences of 17 .. 128 rows and 512 .. 2560 entries, 72B heads, fp32: 99 .. 115 us and 5 for the sum, bf16 61 .. 69 and 5; 19 and 12 us
// more in one group; three times as long with every wave cutting q for itself, chunk by chunk.  Some 232 vector instructions a tile and chunk beside 48 matrix
// instructions; three waves a SIMD (two: 15 % more), for which the fp32 instance at 128 dims spills 3 registers.
template <typename T, int HD, int PLANES>
__global__ __launch_bounds__(256, 3) void kv4_weight_many_kernel(Kv4Attn a) {
    constexpr int G = HD / 32, TILES = 4 / G;
    __shared__ u32x4_t lds_q[2][4][PLANES][64];             // [buffer][tile * G + 32 dims]
    __shared__ float2 lds_dealt[2][TILES][16];
    __shared__ int lds_limit[2][TILES][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quad = lane >> 4;
    const int b = blockIdx.x / a.c.hkv, head = blockIdx.x % a.c.hkv;
    int r0, count, n;
    kv4_rows(a, b, r0, count, n);
    const int begin = blockIdx.z * a.w_cols, cols = min(count * a.group, begin + a.w_cols), safe = n - (count - 1);
    if (begin >= cols) return;
    float* scores = a.book.scores + b * a.book.score_b + head * a.book.score_h;
    // this lane's column of the tile that its wave cuts: its row, its head of the group, and where q and its kv4_dealt lie
    const int first = begin + wave / G * 16 + (lane & 15), rows_on = 16 * TILES / a.group, heads_on = 16 * TILES % a.group;
    int col, head_at, limit, buf = 0;
    const T* at;
    const float2* from;
    float raw[8] = {};
    float2 dealt;
    auto request = [&]() {                                  // a column beyond the last one keeps the values of the one before it; it sees nothing
        const bool is = col < cols;
        if (is) kv4_load8(at, raw);
        dealt = is ? *from : kv4_dealt(0.f, 0.f);
    };
    auto advance = [&]() {
        const bool over = (head_at += heads_on) >= a.group;
        const int rows = rows_on + over, heads = heads_on - (over ? a.group : 0);
        head_at -= over ? a.group : 0;
        col += 16 * TILES;
        limit = col < cols ? limit + rows : 0;
        at += rows * a.q_row + heads * a.q_head;
        from += (int64_t)rows * a.heads + heads;
    };
    for (int base = blockIdx.y * 4 * KV4_CHUNK; base < n; base += gridDim.y * 4 * KV4_CHUNK) {      // the same for all waves: they meet below
        const int slot0 = base + wave * KV4_CHUNK;
        const uint8_t* page[4];
        int there;
        Kv4Keys<HD> raw_k;
        u32x4_t k[4][G];
        col = first, head_at = first % a.group;
        limit = col < cols ? n - (count - 1 - col / a.group) : 0;
        at = static_cast<const T*>(a.q) + (int64_t)(r0 + col / a.group) * a.q_row + (int64_t)(head * a.group + head_at) * a.q_head + quad * (HD / 4) + wave % G * 8;
        from = a.dealt + (int64_t)(r0 + col / a.group) * a.heads + head * a.group + head_at;
        request();
        kv4_pages<HD>(a.c, b, head, slot0, page, there);
        kv4_load_keys<HD>(page, lane, raw_k);
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int j = 0; j < G; ++j) k[p][j] = q4_decode8(raw_k.w[p][j], raw_k.scale[p] << 23);
        const bool whole = slot0 + KV4_CHUNK <= safe && there == 15;
        f32x4_t weight[4] = {};
        for (int c0 = begin; c0 < cols; c0 += 16 * TILES, buf ^= 1) {
            // the readers of this buffer's last contents have passed the barrier of the step in between
            u32x4_t o[PLANES];
            kv4_scale_q(a, raw);
            q4_operand<PLANES>(raw, o);
#pragma unroll
            for (int x = 0; x < PLANES; ++x) lds_q[buf][wave][x][lane] = o[x];
            if (wave % G == 0 && quad == 0) lds_dealt[buf][wave / G][lane] = dealt, lds_limit[buf][wave / G][lane] = limit;
            __syncthreads();
            advance();
            request();
            if (slot0 >= n) continue;
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                if (c0 + t * 16 >= cols) break;
                const float2 of = lds_dealt[buf][t][lane & 15];
                f32x4_t s[4] = {};
#pragma unroll
                for (int j = 0; j < G; ++j)
#pragma unroll
                    for (int x = 0; x < PLANES; ++x) {
                        const u32x4_t q = lds_q[buf][t * G + j][x][lane];
#pragma unroll
                        for (int p = 0; p < 4; ++p) s[p] = q4_mfma(k[p][j], q, s[p]);
                    }
                const int sees = lds_limit[buf][t][lane & 15];
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    f32x4_t w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = kv4_dealt_weight(a, s[p][i], of);
                    if (!whole) kv4_seen_weights(w, slot0 + p * KV4_PAGE + quad * 4, (there >> p) & 1 ? sees : 0);
                    weight[p] += w;
                }
            }
        }
        const float mine = kv4_sum_weights(weight);
        if (a.w_groups == 1) {
            const int slot = kv4_score_slot(slot0, n, there);
            if (slot >= 0) scores[slot] += mine;
        } else {
            const int slot = kv4_score_slot(slot0, n, 15);
            if (slot >= 0) a.part_w[((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * a.w_slots + slot] = kv4_score_slot(slot0, n, there) >= 0 ? mine : -0.f;
        }
    }
}
// adds the groups' weights to the scores, in the order of the groups
__global__ __launch_bounds__(256) void kv4_weight_sum_kernel(Kv4Attn a) {
    const int b = blockIdx.x / a.c.hkv, head = blockIdx.x % a.c.hkv;
    int r0, count, n;
    kv4_rows(a, b, r0, count, n);
    const int groups = (count * a.group + a.w_cols - 1) / a.w_cols;
    if (groups == 0) return;
    float* scores = a.book.scores + b * a.book.score_b + head * a.book.score_h;
    for (int64_t s = (int64_t)blockIdx.y * 256 + threadIdx.x; s < n; s += (int64_t)gridDim.y * 256) {
        float sum = scores[s];
        for (int g = 0; g < groups; ++g) sum += a.part_w[((int64_t)g * gridDim.x + blockIdx.x) * a.w_slots + s];
        scores[s] = sum;
    }
}

// ---- eviction
struct Kv4Evict {
    Kv4Cache c;
    Kv4Book book;
    int budget, recent;
    int* plan;              // [batch][hkv]: entries moved, entries before, 0, 0; for each slot below the budget its rank among the freed ones
                            // or -1; the kept slots above it in order (at most `moves`)
    int moves;
    __host__ __device__ int64_t list_words() const { return 4 + (int64_t)((budget + 3) & ~3) + moves; }
};
// Scores as whole numbers of the same order; protected entries above all, NaN as -inf, both zeros alike
__device__ __forceinline__ uint32_t kv4_rank_key(float score, bool safe) {
    if (safe) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(score != score ? -INFINITY : score + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// Exclusive sums over the 1024 threads of a block of two counts, and the totals; `part` is 2 x 16 words of LDS, free again after the next barrier.
__device__ __forceinline__ void kv4_block_scan(int& a, int& b, int& all_a, int& all_b, int (*part)[16]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = a, y = b;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int p = __shfl_up(x, d), q = __shfl_up(y, d);
        if (lane >= d) x += p, y += q;
    }
    if (lane == 63) part[0][wave] = x, part[1][wave] = y;
    __syncthreads();
    a = x - a, b = y - b, all_a = all_b = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        const int p = part[0][w], q = part[1][w];
        if (w < wave) a += p, b += q;
        all_a += p, all_b += q;
    }
}

// One block per (sequence, kv head).  The key of the budget-th entry comes from a radix selection, eight bits a pass from the top, that ends
// as soon as a bin is kept whole (two or three passes for scores that differ).  Then every thread takes a run of consecutive slots: one sum over the block
// ranks the ties, a second one the freed slots below the budget and the kept entries above it, which are the moves.
// CACHED: the keys stay in LDS (up to 16384 slots); longer lists are read again by every pass.
template <bool CACHED>
__global__ __launch_bounds__(1024) void kv4_select_kernel(Kv4Evict a, int hkv) {
    extern __shared__ uint32_t kv4_keys[];
    __shared__ __align__(16) int hist[256][8], part[2][2][16], found[3], newest_w[16];     // eight lanes' counts of a bin side by side
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = blockIdx.x / hkv, h = blockIdx.x % hkv;
    int* plan = a.plan + blockIdx.x * a.list_words();
    int *place = plan + 4, *from = place + ((a.budget + 3) & ~3);
    const int n = min(max(a.c.kv_len[b], 0), a.c.max_pages * KV4_PAGE);
    if (tid == 0) plan[0] = 0, plan[1] = n;
    if (n <= a.budget) return;
    const float* score = a.book.scores + b * a.book.score_b + h * a.book.score_h;
    const int* pos = a.book.pos + b * a.book.pos_b + h * a.book.pos_h;
    // protected: position > newest - recent, in 64 bits (positions may be any int32)
    int64_t bound = INT64_MAX;
    if (a.recent > 0) {
        int newest = INT32_MIN;
        for (int s = tid; s < n; s += 1024) {
            const int x = pos[s];
            if constexpr (CACHED) kv4_keys[s] = (uint32_t)x;
            newest = max(newest, x);
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) newest = max(newest, __shfl_xor(newest, d));
        if (lane == 0) newest_w[wave] = newest;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 16; ++w) newest = max(newest, newest_w[w]);
        bound = (int64_t)newest - a.recent;
    }
    if constexpr (CACHED) {
        for (int s = tid; s < n; s += 1024) kv4_keys[s] = kv4_rank_key(score[s], a.recent > 0 && (int)kv4_keys[s] > bound);
    }
    // Protected entries are above all others, and alike, until there are more of them than the budget: the selection then ends at their key, and a second
    // one ranks them by their scores, above all others (0).
    bool crowded = false;
    auto rank_of = [&](int s) {
        const bool safe = a.recent > 0 && pos[s] > bound;
        return crowded && !safe ? 0u : kv4_rank_key(score[s], safe && !crowded);
    };
    auto key_of = [&](int s) { return CACHED ? kv4_keys[s] : rank_of(s); };
    uint32_t key;
    int need;                                               // entries still to be kept among those that agree with `key` so far
    for (;;) {
        key = 0, need = a.budget;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 2048; i += 1024) hist[i >> 3][i & 7] = 0;
            __syncthreads();
            const uint32_t above = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
            for (int s = tid; s < n; s += 1024) {
                const uint32_t u = key_of(s);
                if ((u & above) == key) atomicAdd(&hist[(u >> shift) & 255][lane & 7], 1);
            }
            __syncthreads();
            if (wave == 0) {                                // lane l: bins 255 - 4 l .. 252 - 4 l, from the top
                int c[4], mine = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int4 x = *reinterpret_cast<const int4*>(hist[255 - 4 * lane - i]), y = *reinterpret_cast<const int4*>(&hist[255 - 4 * lane - i][4]);
                    c[i] = x.x + x.y + x.z + x.w + y.x + y.y + y.z + y.w;
                    mine += c[i];
                }
                int before = mine;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) { const int x = __shfl_up(before, d); if (lane >= d) before += x; }
                before -= mine;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (before < need && before + c[i] >= need) found[0] = 255 - 4 * lane - i, found[1] = need - before, found[2] = c[i];
                    before += c[i];
                }
            }
            __syncthreads();
            key |= (uint32_t)found[0] << shift;
            need = found[1];
            if (need == found[2]) {                         // the bin is kept whole: every key from `key` on
                key -= 1, need = 0;                         // (key > 0: not every entry is kept)
                break;
            }
        }
        if (key != 0xFFFFFFFFu || crowded) break;           // (no score has the key of the protected)
        crowded = true;
        if constexpr (CACHED) {
            for (int s = tid; s < n; s += 1024) kv4_keys[s] = rank_of(s);
        }
    }
    // keep: keys above, and the first `need` of those equal to it
    const int run = (n + 1023) / 1024, s0 = min(tid * run, n), s1 = min(s0 + run, n);
    int ties = 0, none = 0, all_a, all_b;
    if (need > 0) {
        for (int s = s0; s < s1; ++s) ties += key_of(s) == key;
        kv4_block_scan(ties, none, all_a, all_b, part[0]);
    }
    int holes = 0, extras = 0, rank = ties;
    for (int s = s0; s < s1; ++s) {
        const uint32_t u = key_of(s);
        const bool keep = u > key || (u == key && rank++ < need);
        holes += s < a.budget && !keep;
        extras += s >= a.budget && keep;
    }
    kv4_block_scan(holes, extras, all_a, all_b, part[1]);
    rank = ties;
    for (int s = s0; s < s1; ++s) {
        const uint32_t u = key_of(s);
        const bool keep = u > key || (u == key && rank++ < need);
        if (s < a.budget) place[s] = keep ? -1 : holes++;
        else if (keep) from[extras++] = s;
    }
    if (tid == 0) plan[0] = all_a;
}

// The moves, page by page of the target slots: a wave brings the new entries of a page together and writes its values back whole, because the
// bytes of one token lie four apart.  64 sequences x 4 heads, 225000 moves: 24 us, 33 entry by entry with four byte stores to a lane, 30 with two pages
// to a wave (fewer waves per SIMD); bound by the lines that it touches, about 150 MB through L2.
template <int HD>
__global__ __launch_bounds__(256) void kv4_move_kernel(Kv4Evict a, int hkv) {
    constexpr int G = HD / 32;
    typedef typename u32vec<G>::type V;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 15, quad = lane >> 4;
    const int b = blockIdx.x / hkv, h = blockIdx.x % hkv;
    const int* plan = a.plan + blockIdx.x * a.list_words();
    const int *place = plan + 4, *from_list = place + ((a.budget + 3) & ~3);
    const int count = plan[0];
    if (blockIdx.y == 0 && h == 0 && threadIdx.x == 0) a.c.kv_len[b] = min(plan[1], a.budget);
    if (count == 0) return;
    float* score = a.book.scores + b * a.book.score_b + h * a.book.score_h;
    int* pos = a.book.pos + b * a.book.pos_b + h * a.book.pos_h;
    for (int page = blockIdx.y * 4 + wave; page * KV4_PAGE < a.budget; page += gridDim.y * 4) {
        // lane: token l of the page (for keys, scales, score and position), the same in every quad
        const int to = page * KV4_PAGE + l, rank = to < a.budget ? place[to] : -1;
        if (!__any(rank >= 0)) continue;
        const int from = rank >= 0 ? from_list[rank] : -1;
        uint8_t* dst = kv4_page(a.c, HD, b, page, h);
        const uint8_t* src = from >= 0 ? kv4_page(a.c, HD, b, from / KV4_PAGE, h) : nullptr;
        const int t0 = from >= 0 ? from % KV4_PAGE : 0;
        if (quad == 0 && from >= 0) {
            const float s = score[from];
            const int p = pos[from];
            score[to] = s;
            pos[to] = p;
        }
        const bool moved = src && dst;
        if (!__any(moved)) continue;
        V k = {}, v = {}, v0[4] = {};
        int ks = 0, vs = 0, tv[4];
        if (moved) {
            k = reinterpret_cast<const V*>(src)[quad * 16 + t0];
            if (quad < G) ks = src[kv4_key_scale_at(HD, t0, quad)], vs = src[kv4_val_scale_at(HD, t0, quad)];
        }
        // values: this lane holds dim l of every group for the tokens 4 quad + i; the sources' addresses come from the lanes of those tokens
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int who = quad * 4 + i;
            const uint64_t at = moved ? reinterpret_cast<uint64_t>(src) : 0;
            const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)at, who), hi = (uint32_t)__shfl((int)(uint32_t)(at >> 32), who);
            const uint8_t* p = reinterpret_cast<const uint8_t*>(((uint64_t)hi << 32) | lo);
            const int t = __shfl(t0, who);
            tv[i] = p ? t & 3 : -1;
            if (p) v0[i] = reinterpret_cast<const V*>(p + 8 * HD)[(t >> 2) * 16 + l];
        }
        const bool writes = tv[0] >= 0 || tv[1] >= 0 || tv[2] >= 0 || tv[3] >= 0;
        if (writes) v = reinterpret_cast<const V*>(dst + 8 * HD)[lane];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (tv[i] >= 0)
#pragma unroll
                for (int g = 0; g < G; ++g) v[g] = (v[g] & ~(255u << (8 * i))) | (((v0[i][g] >> (8 * tv[i])) & 255u) << (8 * i));
        if (moved) {
            reinterpret_cast<V*>(dst)[lane] = k;
            if (quad < G) dst[kv4_key_scale_at(HD, l, quad)] = (uint8_t)ks, dst[kv4_val_scale_at(HD, l, quad)] = (uint8_t)vs;
        }
        if (writes) reinterpret_cast<V*>(dst + 8 * HD)[lane] = v;
    }
}
