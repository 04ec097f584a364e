// Entry points of include/rsd_ops.h for the paged bf16 / fp32 cache: argument checks, launch shapes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "rsd_ops.h"
#include "ops_host.h"
#include "kvc.h"
#include "kvc_attn.h"

namespace {

int check_cache(const rsd_kv_cache* c, const char* what) {
    if (!c || !c->pool || !c->table || !c->kv_len) return fail(RSD_EINVAL, "%s: null cache array", what);
    if (!is_type(c->dtype)) return fail(RSD_EINVAL, "%s: cache type %d", what, c->dtype);
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return fail(RSD_EINVAL, "%s: head_dim %d (32, 64 or 128)", what, c->head_dim);
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->batch < 1 || c->max_pages < 1 || c->max_pages > INT32_MAX / (2 * KVC_PAGE))
        return fail(RSD_EINVAL, "%s: pages %d, kv heads %d, batch %d, pages per sequence %d", what, c->n_pages, c->n_kv_heads, c->batch, c->max_pages);
    if ((int64_t)c->batch * c->n_kv_heads > 1 << 20) return fail(RSD_EINVAL, "%s: batch %d x %d kv heads", what, c->batch, c->n_kv_heads);
    if (!aligned(c->pool, 16)) return fail(RSD_EINVAL, "%s: the pool is not 16-byte aligned", what);
    return RSD_OK;
}
KvcCache dev_cache(const rsd_kv_cache* c) { return KvcCache{static_cast<char*>(c->pool), c->table, c->kv_len, c->n_pages, c->n_kv_heads, c->batch, c->max_pages}; }
// activations of `dtype` over the cache
int check_types(const rsd_kv_cache* c, int32_t dtype, const char* what) {
    if (!is_type(dtype) || (dtype == RSD_BF16 && c->dtype == RSD_F32)) return fail(RSD_EINVAL, "%s: activations of type %d over a cache of type %d", what, dtype, c->dtype);
    return RSD_OK;
}

// ---- norms and rotation, entries in

// the bytes from the first to the last element of pieces of head_dim at i * row + j * head
typedef __int128 wide;
struct Bytes { wide from, to; };
Bytes bytes_of(const void* p, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t len, size_t size) {
    const wide a = (wide)(n0 - 1) * s0, b = (wide)(n1 - 1) * s1, at = (wide)reinterpret_cast<uintptr_t>(p);
    return {at + (std::min<wide>(a, 0) + std::min<wide>(b, 0)) * (int64_t)size, at + (std::max<wide>(a, 0) + std::max<wide>(b, 0) + len) * (int64_t)size};
}
Bytes bytes_of(const void* p, int64_t bytes) { return bytes_of(p, 1, 0, 1, 0, bytes, 1); }
bool meet(Bytes a, Bytes b) { return a.from < b.to && b.from < a.to; }
Bytes pool_of(const rsd_kv_cache* c) {
    const int64_t page = 2ll * KVC_PAGE * c->head_dim * c->n_kv_heads;
    return bytes_of(c->pool, c->n_pages, page, 1, 0, page, size_of(c->dtype));
}
// whether an array meets the pool, the table or (where it is used) kv_len
bool meets_cache(Bytes a, const rsd_kv_cache* c, bool lengths) {
    return meet(a, pool_of(c)) || meet(a, bytes_of(c->table, 4ll * c->batch * c->max_pages)) || (lengths && meet(a, bytes_of(c->kv_len, 4ll * c->batch)));
}

struct RowArgs {
    const rsd_heads *q, *k;
    const void* v;
    int64_t v_row, v_head;
    const int32_t *position, *seq, *slot;
    const rsd_rope* rope;
    float eps;
    int32_t rows, head_dim, dtype;
};
// heads that are written to `out` (keys that go into a cache are not)
int check_heads(const rsd_heads* h, const RowArgs& a, bool writes, const char* name, const char* what) {
    if (!h->x || (writes && !h->out)) return fail(RSD_EINVAL, "%s: null array of %s", what, name);
    if (h->n_heads < 1) return fail(RSD_EINVAL, "%s: %d heads of %s", what, h->n_heads, name);
    const size_t size = size_of(a.dtype);
    if (!aligned(h->x, size) || !aligned(h->weight, size) || (writes && !aligned(h->out, size))) return fail(RSD_EINVAL, "%s: an array of %s is not aligned to its type", what, name);
    if (!writes) return RSD_OK;
    if (pieces_overlap(a.rows, h->out_row, h->n_heads, h->out_head, a.head_dim))
        return fail(RSD_EINVAL, "%s: rows of the out of %s overlap (strides %lld, %lld)", what, name, (long long)h->out_row, (long long)h->out_head);
    // a thread has read its values before it writes them to the same place
    const bool same = h->out == h->x && (a.rows == 1 || h->out_row == h->row) && (h->n_heads == 1 || h->out_head == h->head);
    if (!same && share_memory({h->x, h->row, h->head, a.head_dim}, {h->out, h->out_row, h->out_head, a.head_dim}, a.rows, h->n_heads, size))
        return fail(RSD_EINVAL, "%s: the out of %s shares memory with %s", what, name, name);
    return RSD_OK;
}
// Whether heads a and heads b of the same rows share an element: views side by side in the rows of one buffer do not
bool heads_meet(const void* pa, int64_t ra, int64_t ha, int na, const void* pb, int64_t rb, int64_t hb, int nb, const RowArgs& g) {
    const size_t size = size_of(g.dtype);
    const Bytes a = bytes_of(pa, 1, 0, na, ha, g.head_dim, size), b = bytes_of(pb, 1, 0, nb, hb, g.head_dim, size);      // of row 0
    if (!meet(bytes_of(pa, g.rows, ra, na, ha, g.head_dim, size), bytes_of(pb, g.rows, rb, nb, hb, g.head_dim, size))) return false;
    if (ra != rb || ra == 0) return true;
    // one stride of rows: a row's part of a lies between a.from and a.to, b's between b.from and b.to, both modulo the stride
    const wide step = (ra < 0 ? -(wide)ra : (wide)ra) * (int64_t)size, la = a.to - a.from, lb = b.to - b.from;
    wide d = (b.from - a.from) % step;
    if (d < 0) d += step;
    return !(d >= la && d + lb <= step);
}
int check_rows(const RowArgs& a, bool cached, const char* what) {
    if (!is_type(a.dtype)) return fail(RSD_EINVAL, "%s: type %d", what, a.dtype);
    if (a.rows < 1) return fail(RSD_EINVAL, "%s: %d rows", what, a.rows);
    if (!(a.eps >= 0.f) || std::isinf(a.eps)) return fail(RSD_EINVAL, "%s: eps %g", what, a.eps);
    if (a.q)
        if (int rc = check_heads(a.q, a, true, "q", what)) return rc;
    if (a.k)
        if (int rc = check_heads(a.k, a, !cached, "k", what)) return rc;
    const int64_t heads = (a.q ? a.q->n_heads : 0) + (a.k ? (int64_t)a.k->n_heads * (cached ? 2 : 1) : 0);
    if (heads * a.rows > 1 << 26) return fail(RSD_EINVAL, "%s: %d rows of %lld heads are too many", what, a.rows, (long long)heads);
    if (a.rope) {
        if (!a.rope->freq || !a.position) return fail(RSD_EINVAL, "%s: a rotation without %s", what, a.position ? "frequencies" : "positions");
        if (a.rope->rot_dim < 2 || a.rope->rot_dim > a.head_dim || a.rope->rot_dim % 2) return fail(RSD_EINVAL, "%s: %d of %d dimensions turn", what, a.rope->rot_dim, a.head_dim);
        if (!aligned(a.rope->freq, 8)) return fail(RSD_EINVAL, "%s: the frequencies are not aligned to their type", what);
    }
    // what is written and what else is read or written
    const rsd_heads *q = a.q, *k = a.k;
    if (q && k) {
        if (heads_meet(q->out, q->out_row, q->out_head, q->n_heads, k->x, k->row, k->head, k->n_heads, a)) return fail(RSD_EINVAL, "%s: the out of q shares memory with k", what);
        if (!cached && heads_meet(k->out, k->out_row, k->out_head, k->n_heads, q->x, q->row, q->head, q->n_heads, a)) return fail(RSD_EINVAL, "%s: the out of k shares memory with q", what);
        if (!cached && heads_meet(k->out, k->out_row, k->out_head, k->n_heads, q->out, q->out_row, q->out_head, q->n_heads, a))
            return fail(RSD_EINVAL, "%s: the out of k shares memory with that of q", what);
    }
    if (q && cached && heads_meet(q->out, q->out_row, q->out_head, q->n_heads, a.v, a.v_row, a.v_head, k->n_heads, a)) return fail(RSD_EINVAL, "%s: the out of q shares memory with v", what);
    const size_t size = size_of(a.dtype);
    for (int i = 0; i < 2; ++i) {
        const rsd_heads* h = i ? k : q;
        if (!h || (i && cached)) continue;
        const Bytes out = bytes_of(h->out, a.rows, h->out_row, h->n_heads, h->out_head, a.head_dim, size);
        auto small = [&](const void* p, int64_t n) { return p && n && meet(out, bytes_of(p, n)); };
        if (small(q ? q->weight : nullptr, a.head_dim * size) || small(k ? k->weight : nullptr, a.head_dim * size) || small(a.rope ? a.position : nullptr, 4ll * a.rows) ||
            small(a.seq, 4ll * a.rows) || small(a.slot, 4ll * a.rows) || small(a.rope ? a.rope->freq : nullptr, a.rope ? 4ll * a.rope->rot_dim : 0))
            return fail(RSD_EINVAL, "%s: the out of %s shares memory with weights, positions, frequencies, sequences or slots", what, i ? "k" : "q");
    }
    return RSD_OK;
}
// Whether something that an append reads lies in the pool that it writes
int check_pool(const rsd_kv_cache* c, const RowArgs& a) {
    const Bytes pool = pool_of(c);
    const size_t size = size_of(a.dtype);
    auto heads = [&](const void* p, int64_t row, int64_t head, int n) { return meet(pool, bytes_of(p, a.rows, row, n, head, a.head_dim, size)); };
    auto array = [&](const void* p, int64_t n) { return p && meet(pool, bytes_of(p, n)); };
    const char* name = nullptr;
    if (heads(a.k->x, a.k->row, a.k->head, a.k->n_heads)) name = "k";
    else if (heads(a.v, a.v_row, a.v_head, a.k->n_heads)) name = "v";
    else if (a.q && heads(a.q->x, a.q->row, a.q->head, a.q->n_heads)) name = "q";
    else if (array(a.k->weight, a.head_dim * size) || array(a.q ? a.q->weight : nullptr, a.head_dim * size)) name = "a weight";
    else if (array(a.seq, 4ll * a.rows) || array(a.slot, 4ll * a.rows)) name = "seq or slot";
    else if (a.rope && (array(a.position, 4ll * a.rows) || array(a.rope->freq, 4ll * a.rope->rot_dim))) name = "position or freq";
    else if (array(c->table, 4ll * c->batch * c->max_pages)) name = "the table";
    return name ? fail(RSD_EINVAL, "append: %s lies in the pool", name) : RSD_OK;
}
KvcHeads dev_heads(const rsd_heads* h) { return h ? KvcHeads{h->x, h->out, h->weight, h->row, h->head, h->out_row, h->out_head, h->n_heads} : KvcHeads{}; }
KvcRows dev_rows(const RowArgs& a, const KvcCache& c) {
    KvcRows r{dev_heads(a.q), dev_heads(a.k), a.v, a.v_row, a.v_head, a.position, a.seq, a.slot, nullptr, 0, 1.f, a.eps, a.rows, 0, c};
    if (a.rope) r.freq = a.rope->freq, r.rot_dim = a.rope->rot_dim, r.magnitude = a.rope->magnitude;
    return r;
}
template <typename T, typename C, int HD, bool CACHE> void rows_run(const RowArgs& a, KvcRows r, Launches& l) {
    r.value_blocks = CACHE ? (int)(ceil_div(a.rows, KvcValueBlock<C, HD>::ROWS) * ceil_div(r.k.n, KvcValueBlock<C, HD>::HEADS)) : 0;
    const unsigned grid = (unsigned)(r.value_blocks + ceil_div((int64_t)a.rows * (r.q.n + r.k.n), 256 / (HD / 16)));
    if (a.rope && a.rope->interleaved) l.run(kvc_rows_kernel<T, C, HD, true, false, CACHE>, grid, 256, 0, r);
    else if (r.rot_dim % 16 == 0) l.run(kvc_rows_kernel<T, C, HD, false, false, CACHE>, grid, 256, 0, r);
    else l.run(kvc_rows_kernel<T, C, HD, false, true, CACHE>, grid, 256, 0, r);
}
template <typename T> void rope_run(const RowArgs& a, const KvcRows& r, Launches& l) {
    if (a.head_dim == 32) rows_run<T, T, 32, false>(a, r, l);
    else if (a.head_dim == 64) rows_run<T, T, 64, false>(a, r, l);
    else if (a.head_dim == 128) rows_run<T, T, 128, false>(a, r, l);
    else rows_run<T, T, 256, false>(a, r, l);
}
template <typename T, typename C> void append_run(const RowArgs& a, const KvcRows& r, Launches& l) {
    if (a.head_dim == 32) rows_run<T, C, 32, true>(a, r, l);
    else if (a.head_dim == 64) rows_run<T, C, 64, true>(a, r, l);
    else rows_run<T, C, 128, true>(a, r, l);
}

// ---- attention

struct AttnPlan {
    int lists, tiles, tile_cols, ch, waves, split, splits;
    bool many, by_length, packed;
    uint64_t o_bytes, ml_bytes;
    uint64_t bytes() const { return o_bytes + ml_bytes; }
};
// a window that no row reaches past is none
int window_of(const rsd_kv_cache* c, const rsd_kv_attn* a) { return a->window >= std::min<int64_t>(a->max_kv, (int64_t)c->max_pages * KVC_PAGE) ? 0 : a->window; }

// Which kernel, which tiles, how the entries are split: by the sizes that the host knows.  Measured with 28 heads over 4 of 128, bf16, where nothing else is said, in us:
//  - the kernel of few columns takes up to two tiles of 16 (21 columns, 4 sequences of 2048 entries: 13.3, the other 17.0; 8, 32 of 128 .. 5120: 18 and 24, 38 and 51; fp32 activations 19 and 31, 40 and 54; of 64 such
//    sequences the longest decide: 81 and 72), but one tile where the lists of entries alone fill the card (21 columns, 128, 256 of 2048: 113 and 97, 221 and 191), and all over an fp32 cache (16 x 16 heads of 64, 17 .. 128 rows: 43 and 63).
//  - 128 columns to a block instead of 64 where rows see 768 entries and more before their own (2048 rows of 8192: 305 and 348, with a window of 2000 107 and 113; 16 x 128 of 1024: 56 and 60; against that 2048 of 2048: 71 and 58,
//    64 x 128 of 300: 88 and 84) and there are 384 such blocks with their parts (512 rows of 8192: 104 and 111; against that 4 x 128 of 2048: 47 and 41, 256 of 8192: 64 and 63).
//  - a part's sums are 4 bytes an element written and read, beside the join's launch.  Many columns are split up to 512 blocks (16 x 128 of 1024: 58 whole, 79 in two; 256 x 8 of 2048: 200 whole, 246 in two;
//    256 of 8192: 219 whole, 65 in eight), up to 48 columns for 768 (64 x 5 of 128 .. 5120: 97 whole, 76 in three, 88 in four; where all have 5120 the three cost: 117 whole, 142), no part under 512 or 1024 entries.
//    Few columns for 256 blocks, no part under 768 (one sequence of 1279: 10.2 whole, 11.1 in two; of 2500: 15.0 whole, 12.2 in three; of 8000: 39 whole, 15.8 in ten; 16 of 8000: 67 whole, 45 .. 48 in two to four).
//  - few columns: eight waves up to 256 blocks (one sequence of 896 .. 1279: 10.2, 11.9 with four) and for long lists (256 of 4096 .. 8192: 535 and 558), else four (window 1024: 101, 105 with eight; heads of 64: 49 and 54).
//  - where sequences have unlike numbers of rows, blocks without columns go behind the others (16 of 17 .. 128 rows, 72B heads, fp32, window 1000: 103 and 111; 32 of 5 .. 128 rows of 300 .. 4096: 133 and 146;
//    16 x 16 heads of 64, fp32: 43 and 46; where all have the same it costs a block's start 0.5 us: 64 x 128 of 300: 87 and 83).
//  - the longest lists first, from the point where the blocks are more than the card holds at once (64 x 5 of 128 .. 5120: 76 and 87; 256 of 4096 .. 8192: 534 and 555).
AttnPlan attn_plan(const rsd_kv_cache* c, const rsd_kv_attn* a) {
    AttnPlan p{};
    const int group = a->n_heads / c->n_kv_heads, window = window_of(c, a);
    const int64_t cols = (int64_t)a->max_rows * group, max_kv = std::min<int64_t>(a->max_kv, (int64_t)c->max_pages * KVC_PAGE);
    p.lists = c->batch * c->n_kv_heads;
    p.many = c->dtype == RSD_BF16 && (cols > 32 || (cols > 16 && p.lists >= 512));
    p.tile_cols = 16;
    if (p.many) {
        p.tile_cols = 64;
        const int64_t base = (int64_t)p.lists * ceil_div(cols, 128), parts = std::max<int64_t>(1, std::min(512 / base, max_kv / 1024));
        if (a->dtype == RSD_BF16 && cols > 64 && max_kv - a->max_rows >= 768 && base * parts >= 384) p.tile_cols = 128;
    }
    p.tiles = (int)ceil_div(cols, p.tile_cols);
    // slots of a chunk, or of a step of the kernel for many columns
    p.ch = (c->dtype == RSD_F32 ? 1 : 2) * KVC_PAGE * (p.many && (a->dtype == RSD_F32 || p.tile_cols == 128) ? 2 : 1);
    const int ch = p.ch;
    int64_t chunks = std::max<int64_t>(1, ceil_div(max_kv, ch));
    if (window) {
        const int64_t rows = std::min<int64_t>(a->max_rows, (p.tile_cols + group - 2) / group + 1);      // that share a tile
        chunks = std::min(chunks, ceil_div(std::min<int64_t>(a->sinks, max_kv), ch) + ceil_div((int64_t)window + rows - 1, ch) + 1);
    }
    const int64_t base = (int64_t)p.lists * p.tiles;
    int64_t parts;
    if (p.many) {
        p.waves = 4;
        parts = p.tile_cols == 128 ? std::min(512 / base, chunks * ch / 1024) : std::min((cols <= 48 ? 768 : 512) / base, chunks * ch / 512);
    } else {
        parts = std::max<int64_t>(1, std::min(256 / base, chunks * ch / 768));
        p.waves = (int)std::min<int64_t>(base * parts <= 256 || (chunks * ch >= 1536 * parts && base < 1 << 21) ? 8 : 4, chunks);
    }
    p.split = (int)ceil_div(chunks, std::max<int64_t>(1, parts));
    p.splits = (int)ceil_div(chunks, p.split);
    p.by_length = c->batch > 1 && base * p.splits * p.waves > 2048;
    p.packed = p.tiles > 1 && a->rows < (int64_t)c->batch * a->max_rows && c->batch <= 64 && p.lists >= 8;
    const uint64_t lines = (uint64_t)a->rows * a->n_heads;
    p.o_bytes = p.splits > 1 ? up256(lines * p.splits * c->head_dim * 4) : 0;
    p.ml_bytes = p.splits > 1 ? up256(lines * p.splits * 8) : 0;
    return p;
}
int check_attn(const rsd_kv_cache* c, const rsd_kv_attn* a) {
    if (int rc = check_cache(c, "attention")) return rc;
    if (!a) return fail(RSD_EINVAL, "attention: null arguments");
    if (int rc = check_types(c, a->dtype, "attention")) return rc;
    if (a->rows < 1 || a->max_rows < 1 || a->max_kv < 0) return fail(RSD_EINVAL, "attention: rows %d, at most %d a sequence, entries %d", a->rows, a->max_rows, a->max_kv);
    if (a->n_heads < 1 || a->n_heads % c->n_kv_heads) return fail(RSD_EINVAL, "attention: %d heads over %d kv heads", a->n_heads, c->n_kv_heads);
    if (a->window < 0 || a->sinks < 0) return fail(RSD_EINVAL, "attention: window %d, sinks %d", a->window, a->sinks);
    if (!a->row_start && a->max_rows != 1) return fail(RSD_EINVAL, "attention: max_rows %d without row_start", a->max_rows);
    if ((int64_t)a->max_rows * a->n_heads > INT32_MAX / 16 || c->batch * (int64_t)c->n_kv_heads * ceil_div((int64_t)a->max_rows * (a->n_heads / c->n_kv_heads), 64) > 1 << 20)
        return fail(RSD_EINVAL, "attention: %d rows x %d heads x %d sequences", a->max_rows, a->n_heads, c->batch);
    return RSD_OK;
}
template <typename T, typename C, int HD> void attn_run(const KvcAttn& k, const AttnPlan& p, Launches& l) {
    const unsigned grid = (unsigned)kvc_blocks(p.lists, p.tiles, p.splits);
    if (!p.many) l.run(kvc_attn_few_kernel<T, C, HD>, grid, 64 * p.waves, 0, k);
    else if constexpr (sizeof(C) == 2) {
        if (p.tile_cols == 64) l.run(kvc_attn_many_kernel<T, C, HD, 1>, grid, 256, 0, k);
        else if constexpr (sizeof(T) == 2) l.run(kvc_attn_many_kernel<T, C, HD, 2>, grid, 256, 0, k);
    }
    if (p.splits > 1) l.run(kvc_join_kernel<T, HD>, (unsigned)ceil_div((int64_t)k.c.batch * k.max_rows * k.heads, 16), 256, 0, k);
}
template <typename T, typename C> void attn_run(const KvcAttn& k, const AttnPlan& p, int hd, Launches& l) {
    if (hd == 32) attn_run<T, C, 32>(k, p, l);
    else if (hd == 64) attn_run<T, C, 64>(k, p, l);
    else attn_run<T, C, 128>(k, p, l);
}

}  // namespace

extern "C" int rsd_rope_frequencies(double theta, int32_t rot_dim, int32_t kind, double factor, double original, double low, double high, double* freq) {
    if (!freq) return fail(RSD_EINVAL, "rope_frequencies: null array");
    if (rot_dim < 2 || rot_dim % 2) return fail(RSD_EINVAL, "rope_frequencies: %d dimensions", rot_dim);
    if (!(theta > 0) || std::isinf(theta)) return fail(RSD_EINVAL, "rope_frequencies: theta %g", theta);
    if (kind < RSD_ROPE_PLAIN || kind > RSD_ROPE_PARTS) return fail(RSD_EINVAL, "rope_frequencies: kind %d", kind);
    if (kind != RSD_ROPE_PLAIN && (!(factor > 0) || std::isinf(factor))) return fail(RSD_EINVAL, "rope_frequencies: factor %g", factor);
    if (kind == RSD_ROPE_BASE && rot_dim < 4) return fail(RSD_EINVAL, "rope_frequencies: one pair has no last frequency beside its first");
    if (kind == RSD_ROPE_PARTS && (!(original > 0) || std::isinf(original) || !(high > low) || std::isinf(high) || std::isinf(low)))
        return fail(RSD_EINVAL, "rope_frequencies: original %g, low %g, high %g", original, low, high);
    const double base = kind == RSD_ROPE_BASE ? theta * std::pow(factor, rot_dim / (rot_dim - 2.)) : theta;
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double f = std::pow(base, -2. * i / rot_dim);
        if (kind == RSD_ROPE_LINEAR) freq[i] = f / factor;
        else if (kind == RSD_ROPE_PARTS) {
            const double g = std::min(1., std::max(0., (original * f / (2 * M_PI) - low) / (high - low)));
            freq[i] = f * (g + (1 - g) / factor);
        } else freq[i] = f;
    }
    return RSD_OK;
}

extern "C" int rsd_qk_rope(const rsd_heads* q, const rsd_heads* k, const int32_t* position, const rsd_rope* rope, float eps, int32_t rows, int32_t head_dim,
                           int32_t dtype, void* hip_stream) {
    if (!q && !k) return fail(RSD_EINVAL, "qk_rope: neither q nor k");
    if (head_dim != 32 && head_dim != 64 && head_dim != 128 && head_dim != 256) return fail(RSD_EINVAL, "qk_rope: head_dim %d (32, 64, 128 or 256)", head_dim);
    const RowArgs a{q, k, nullptr, 0, 0, position, nullptr, nullptr, rope, eps, rows, head_dim, dtype};
    if (int rc = check_rows(a, false, "qk_rope")) return rc;
    Launches l(hip_stream);
    const KvcRows r = dev_rows(a, KvcCache{});
    if (dtype == RSD_F32) rope_run<float>(a, r, l);
    else rope_run<bf16_t>(a, r, l);
    return l.done("qk_rope");
}

extern "C" int rsd_kv_append(const rsd_kv_cache* c, const rsd_heads* k, const void* v, int64_t v_row, int64_t v_head, const rsd_heads* q, const int32_t* seq,
                             const int32_t* slot, const int32_t* position, const rsd_rope* rope, float eps, int32_t rows, int32_t dtype, void* hip_stream) {
    if (int rc = check_cache(c, "append")) return rc;
    if (!k || !v || !seq || !slot) return fail(RSD_EINVAL, "append: null array");
    if (int rc = check_types(c, dtype, "append")) return rc;
    if (k->n_heads != c->n_kv_heads) return fail(RSD_EINVAL, "append: %d heads of k, %d of the cache", k->n_heads, c->n_kv_heads);
    if (!aligned(v, size_of(dtype))) return fail(RSD_EINVAL, "append: v is not aligned to its type");
    const RowArgs a{q, k, v, v_row, v_head, position, seq, slot, rope, eps, rows, c->head_dim, dtype};
    if (int rc = check_rows(a, true, "append")) return rc;
    if (int rc = check_pool(c, a)) return rc;
    if (q && meets_cache(bytes_of(q->out, rows, q->out_row, q->n_heads, q->out_head, c->head_dim, size_of(dtype)), c, false))
        return fail(RSD_EINVAL, "append: the out of q shares memory with the cache");
    Launches l(hip_stream);
    const KvcRows r = dev_rows(a, dev_cache(c));
    if (c->dtype == RSD_F32) append_run<float, float>(a, r, l);
    else if (dtype == RSD_F32) append_run<float, bf16_t>(a, r, l);
    else append_run<bf16_t, bf16_t>(a, r, l);
    return l.done("append");
}

extern "C" int rsd_kv_read(const rsd_kv_cache* c, const int32_t* seq, const int32_t* slot, int32_t rows, void* k, void* v, void* hip_stream) {
    if (int rc = check_cache(c, "read")) return rc;
    if (!k || !v || !seq || !slot) return fail(RSD_EINVAL, "read: null array");
    if (rows < 1) return fail(RSD_EINVAL, "read: %d rows", rows);
    if (!aligned(k, 16) || !aligned(v, 16)) return fail(RSD_EINVAL, "read: k or v is not 16-byte aligned");
    if (2ll * rows * c->n_kv_heads > 1 << 26) return fail(RSD_EINVAL, "read: %d rows are too many", rows);
    const int64_t bytes = (int64_t)rows * c->n_kv_heads * c->head_dim * (int64_t)size_of(c->dtype);
    for (const void* p : {k, v}) {
        const Bytes out = bytes_of(p, bytes);
        if (meets_cache(out, c, false) || meet(out, bytes_of(seq, 4ll * rows)) || meet(out, bytes_of(slot, 4ll * rows)) || meet(bytes_of(k, bytes), bytes_of(v, bytes)))
            return fail(RSD_EINVAL, "read: k or v shares memory with another array");
    }
    const unsigned grid = (unsigned)ceil_div(2ll * rows * c->n_kv_heads * (c->head_dim / 8), 256);
    Launches l(hip_stream);
    auto run = [&](auto zero) {
        typedef decltype(zero) C;
        const KvcCache d = dev_cache(c);
        if (c->head_dim == 32) l.run(kvc_read_kernel<C, 32>, grid, 256, 0, d, seq, slot, rows, static_cast<C*>(k), static_cast<C*>(v));
        else if (c->head_dim == 64) l.run(kvc_read_kernel<C, 64>, grid, 256, 0, d, seq, slot, rows, static_cast<C*>(k), static_cast<C*>(v));
        else l.run(kvc_read_kernel<C, 128>, grid, 256, 0, d, seq, slot, rows, static_cast<C*>(k), static_cast<C*>(v));
    };
    if (c->dtype == RSD_F32) run(float{});
    else run(bf16_t{});
    return l.done("read");
}

extern "C" uint64_t rsd_kv_attention_workspace(const rsd_kv_cache* c, const rsd_kv_attn* a) { return check_attn(c, a) ? 0 : attn_plan(c, a).bytes(); }

extern "C" int rsd_kv_attention(const rsd_kv_cache* c, const rsd_kv_attn* a, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
    if (int rc = check_attn(c, a)) return rc;
    if (!a->q || !a->out) return fail(RSD_EINVAL, "attention: null array");
    if (!aligned(a->q, size_of(a->dtype)) || !aligned(a->out, size_of(a->dtype)) || !aligned(a->lse, 4)) return fail(RSD_EINVAL, "attention: q, out or lse is not aligned to its type");
    if (pieces_overlap(a->rows, a->out_row, a->n_heads, a->out_head, c->head_dim))
        return fail(RSD_EINVAL, "attention: rows of out overlap (strides %lld, %lld)", (long long)a->out_row, (long long)a->out_head);
    // a block has read its columns of q before it writes them, and no other block reads them
    const bool same = a->out == a->q && (a->rows == 1 || a->out_row == a->q_row) && (a->n_heads == 1 || a->out_head == a->q_head);
    if (!same && share_memory({a->q, a->q_row, a->q_head, c->head_dim}, {a->out, a->out_row, a->out_head, c->head_dim}, a->rows, a->n_heads, size_of(a->dtype)))
        return fail(RSD_EINVAL, "attention: out shares memory with q");
    const AttnPlan p = attn_plan(c, a);
    const uint64_t need = p.bytes();
    if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 256))))
        return fail(RSD_EINVAL, "attention: the workspace holds %llu of %llu bytes, or is not 256-byte aligned", (unsigned long long)workspace_bytes, (unsigned long long)need);
    const size_t size = size_of(a->dtype);
    const Bytes q = bytes_of(a->q, a->rows, a->q_row, a->n_heads, a->q_head, c->head_dim, size), out = bytes_of(a->out, a->rows, a->out_row, a->n_heads, a->out_head, c->head_dim, size),
                lse = bytes_of(a->lse, a->lse ? 4ll * a->rows * a->n_heads : 0), ws = bytes_of(need ? workspace : nullptr, need);
    if (meet(out, lse) || meet(out, ws) || meet(lse, ws) || meet(q, lse) || meet(q, ws))
        return fail(RSD_EINVAL, "attention: two of q, out, lse and the workspace share memory");
    for (const Bytes& x : {out, lse, ws})
        if (meets_cache(x, c, true) || (a->row_start && meet(x, bytes_of(a->row_start, 4ll * (c->batch + 1))))) return fail(RSD_EINVAL, "attention: out, lse or the workspace shares memory with the cache or row_start");
    KvcAttn k{};
    k.c = dev_cache(c);
    k.q = a->q, k.q_row = a->q_row, k.q_head = a->q_head;
    k.row_start = a->row_start, k.total_rows = a->rows, k.max_rows = a->max_rows, k.heads = a->n_heads;
    auto divisor = [](int d) { return KvcDivisor{(uint32_t)d, d == 1 ? 0xFFFFFFFFu : (uint32_t)((1ull << 32) / (uint64_t)d + 1)}; };
    k.group = divisor(a->n_heads / c->n_kv_heads), k.by_heads = divisor(c->n_kv_heads), k.by_tiles = divisor(p.tiles);
    k.scale = a->scale;
    k.plain = !(std::fabs(a->scale) > 0.f) || std::isinf(a->scale);
    k.factor = k.plain ? 1.f : std::fabs(a->scale);
    k.factor2 = (float)std::min(k.factor * 1.4426950408889634, (double)FLT_MAX);
    k.slack = (float)std::min(8. / k.factor2, (double)FLT_MAX);
    k.negative = a->scale < 0.f;
    k.out = a->out, k.o_row = a->out_row, k.o_head = a->out_head;
    k.lse = a->lse;
    k.max_kv = std::min(a->max_kv, c->max_pages * KVC_PAGE), k.window = window_of(c, a), k.sinks = std::min(a->sinks, c->max_pages * KVC_PAGE);
    k.lists = p.lists, k.ch = p.ch, k.tiles = p.tiles, k.tile_cols = p.tile_cols, k.split = p.split, k.splits = p.splits, k.by_length = p.by_length, k.packed = p.packed;
    k.part_o = static_cast<float*>(workspace);
    k.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + p.o_bytes);
    Launches l(hip_stream);
    if (c->dtype == RSD_F32) attn_run<float, float>(k, p, c->head_dim, l);
    else if (a->dtype == RSD_F32) attn_run<float, bf16_t>(k, p, c->head_dim, l);
    else attn_run<bf16_t, bf16_t>(k, p, c->head_dim, l);
    return l.done("attention");
}
