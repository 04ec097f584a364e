// Entry points of include/rsd_ops.h: argument checks, launch shapes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <type_traits>

#include "rsd_ops.h"
#include "q4.h"
#include "w4.h"
#include "kv4.h"

namespace {

thread_local char op_error[256] = "";

int fail(int code, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(op_error, sizeof(op_error), fmt, ap);
    va_end(ap);
    return code;
}
// The launches of a call, by the status that each returns: the runtime's last error may be one that the caller has not read yet, and stays.
class Launches {
    hipStream_t st_;
    hipError_t first_ = hipSuccess;
public:
    explicit Launches(void* stream) : st_(static_cast<hipStream_t>(stream)) {}
    template <typename... P> void run(void (*kernel)(P...), dim3 grid, unsigned threads, size_t lds, std::common_type_t<P>... args) {
        if (first_ != hipSuccess) return;
        void* at[] = {&args...};
        first_ = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), at, lds, st_);
    }
    int done(const char* what) {
        if (first_ == hipSuccess) return RSD_OK;
        (void)hipGetLastError();                            // reported here
        return fail(RSD_EHIP, "%s: %s", what, hipGetErrorString(first_));
    }
};
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool is_type(int32_t t) { return t == RSD_F32 || t == RSD_BF16; }
size_t size_of(int32_t t) { return t == RSD_F32 ? 4 : 2; }
uint64_t up256(uint64_t n) { return (n + 255) & ~255ull; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t kMostBlocks = 1ll << 22;      // blocks of at most 512 threads: a launch counts threads in 32 bits per dimension

// Pieces of `len` elements at i s0 + j s1, i < n0, j < n1: whether two of them share an element.  Mostly one stride passes the other's pieces, which is seen
// at once; else every distance in the shorter dimension is set against the nearest ones in the other.
bool pieces_overlap(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t len) {
    typedef __int128 wide;
    if (n0 > n1) std::swap(n0, n1), std::swap(s0, s1);
    const wide a = s0 < 0 ? -(wide)s0 : s0, b = s1 < 0 ? -(wide)s1 : s1;      // distances count in both directions
    if (n0 == 1) return n1 > 1 && b < len;
    if (a < len || b < len) return true;
    if (b >= (n0 - 1) * a + len || a >= (n1 - 1) * b + len) return false;
    for (wide i = 1; i < n0; ++i) {
        const wide j = i * a / b;
        if ((j < n1 && i * a - j * b < len) || (j + 1 < n1 && (j + 1) * b - i * a < len)) return true;
    }
    return false;
}

// Two arrays of one type, pieces at i s0 + j s1 of each (i < n0, j < n1), of `len` elements
struct Pieces { const void* at; int64_t s0, s1, len; };
// Whether they share an element.  Views of one buffer (heads of q beside those of out) mostly have the same s0; where that differs, arrays that lie between
// each other's ends count as sharing.
bool share_memory(Pieces p, Pieces q, int64_t n0, int64_t n1, size_t size) {
    typedef __int128 wide;
    if (n0 == 1) p.s0 = q.s0 = 0;
    if (n1 == 1) p.s1 = q.s1 = 0;
    const wide d = ((wide)reinterpret_cast<uintptr_t>(q.at) - (wide)reinterpret_cast<uintptr_t>(p.at)) / (int64_t)size;
    auto low = [&](const Pieces& x) { return std::min<wide>(0, (wide)(n0 - 1) * x.s0) + std::min<wide>(0, (wide)(n1 - 1) * x.s1); };
    auto high = [&](const Pieces& x) { return std::max<wide>(0, (wide)(n0 - 1) * x.s0) + std::max<wide>(0, (wide)(n1 - 1) * x.s1) + x.len; };
    if (d + low(q) >= high(p) || d + high(q) <= low(p)) return false;
    if (p.s0 != q.s0) return true;
    const wide s0 = p.s0 < 0 ? -(wide)p.s0 : p.s0;         // distances in i count in both directions
    auto floor_div = [](wide a, wide b) { return a / b - (a % b < 0); };
    if (s0 > 0 && p.s1 >= 0 && q.s1 >= 0) {                 // side by side in every row of the buffer
        const wide from = d - floor_div(d, s0) * s0;
        if (from >= (n1 - 1) * (wide)p.s1 + p.len && from + (n1 - 1) * (wide)q.s1 + q.len <= s0) return false;
    }
    // q's piece starts `c` behind p's, and a multiple of s0: somewhere between -q.len and p.len?
    auto meet = [&](wide c) {
        return s0 == 0 ? c > -q.len && c < p.len : std::max<wide>(-floor_div(q.len - 1 + c, s0), 1 - n0) <= std::min<wide>(floor_div(p.len - 1 - c, s0), n0 - 1);
    };
    for (int64_t j = 0; j < n1; ++j)
        for (int64_t i = 0; i < n1; ++i) {
            if (p.s1 == q.s1 && i > 0 && j > 0) break;      // (only their distance counts)
            if (meet(d + (wide)j * q.s1 - (wide)i * p.s1)) return true;
        }
    return false;
}

// ---- products with 4-bit weights

struct W4Plan { int nt, kt, ks; bool few; int ntile, waves, xt, splits, tiles; uint64_t part_bytes; };

// Which kernel, and how the columns are split (by sizes and type alone; measured on both sides of each bound, times with launch):
//  - few rows (<= 16): while its blocks together read at most 64 MB of x (16 rows bf16, 3584 x 3584: 8.2 us against 12.4; 8 rows, 8192 x 29568: 35.8 against 29.4),
//    and with more than four rows while a wave has few tiles of columns: up to 80 in all (8 rows bf16, 8192 x 8192: 12.1 us against 13.6; 3584 x 18944: 21.6
//    against 12.3), up to 16 in fp32, which its waves cut into three parts each for itself (1536 x 1536: 8.4 against 12.2, 3584 x 3584: 15.5 against 12.3).
//    Four tiles of W to a block instead of two where two would give more blocks of 16 waves than CUs (8 rows, 10240 x 8192: 13.9 us against 21.2; 8192 x 8192: 12.9 against 12.5).
//  - many rows: blocks for every CU, two where a tile of x is small (64 rows, 3584 x 18944: 73 us in 2 splits, 40 in 4, 24 in 8, 19 in 16; 256 rows: 73, 44, 44, 55),
//    no split of fewer than four tiles.  From six on splits come in eights: one part of x per XCD.
W4Plan w4_plan(int rows, int n, int k, int dtype) {
    W4Plan p{};
    p.nt = (int)ceil_div(n, 16);
    p.kt = (int)ceil_div(k, 128);
    p.ks = (int)ceil_div(k, 512);
    const bool f32 = dtype == RSD_F32;
    p.few = rows <= 16 && ceil_div(p.nt, 2) * rows * k * (int64_t)size_of(dtype) <= 64 << 20 && !(rows > 4 && p.kt > (f32 ? 16 : 80));
    p.ntile = rows > 4 && k >= 8 && p.nt > 512 ? 4 : 2;
    int64_t splits = 1;
    if (!p.few) {
        p.xt = rows <= 16 || k < 8 ? 1 : rows <= 32 || f32 ? 2 : 4;
        const int64_t blocks = ceil_div(p.nt, 16) * ceil_div(rows, p.xt * 16);
        splits = std::max<int64_t>(1, std::min<int64_t>((p.xt == 4 ? 256 : 512) / blocks, p.kt / 4));
        if (splits > 5) splits = std::min<int64_t>((splits + 3) / 8 * 8, 16);
    }
    p.tiles = (int)ceil_div(p.kt, splits);
    if (!p.few) p.tiles = (p.tiles + 3) & ~3;
    p.splits = (int)ceil_div(p.kt, p.tiles);
    // waves of a few-row block: some 4096 in all, at least four, as many as take equally many tiles
    p.waves = (int)std::min<int64_t>(std::min(f32 && rows > 4 ? 8 : 16, p.kt), std::max<int64_t>(4, ceil_div(4096, ceil_div(p.nt, p.ntile))));
    p.waves = (int)ceil_div(p.kt, ceil_div(p.kt, p.waves));
    p.part_bytes = p.splits > 1 ? up256((uint64_t)p.splits * rows * w4_padded(n) * 4) : 0;
    return p;
}

template <typename T> void w4_launch(const W4Plan& p, const W4Args& a, Launches& l) {
    const bool wide = a.k >= 8;
    if (p.few) {
        const unsigned grid = (unsigned)ceil_div(p.nt, p.ntile), threads = 64 * p.waves;
        if (!wide) l.run(w4_few_kernel<T, 2, 4, false>, grid, threads, 0, a);
        else if (a.rows <= 4) l.run(w4_few_kernel<T, 2, 1, true>, grid, threads, 0, a);
        else if (p.ntile == 2) l.run(w4_few_kernel<T, 2, 4, true>, grid, threads, 0, a);
        else l.run(w4_few_kernel<T, 4, 4, true>, grid, threads, 0, a);
        return;
    }
    const unsigned grid = (unsigned)(p.splits * ceil_div(p.nt, 16) * ceil_div(a.rows, p.xt * 16));
    if (!wide) l.run(w4_many_kernel<T, 1, false>, grid, 256, 0, a);
    else if (p.xt == 1) l.run(w4_many_kernel<T, 1, true>, grid, 256, 0, a);
    else if (p.xt == 2) l.run(w4_many_kernel<T, 2, true>, grid, 256, 0, a);
    else if constexpr (sizeof(T) == 2) l.run(w4_many_kernel<T, 4, true>, grid, 256, 0, a);
}
template <typename T> void w4_run(const W4Plan& p, const W4Args& a, Launches& l) {
    w4_launch<T>(p, a, l);
    if (p.splits > 1)
        l.run(w4_sum_kernel<T>, (unsigned)ceil_div((int64_t)a.rows * (w4_padded(a.n) / 4), 256), 256, 0, a);
}

// ---- the cache

int check_cache(const rsd_kv4_cache* c, const char* what) {
    if (!c || !c->pool || !c->table || !c->kv_len) return fail(RSD_EINVAL, "%s: null cache array", what);
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return fail(RSD_EINVAL, "%s: head_dim %d (32, 64 or 128)", what, c->head_dim);
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->batch < 1 || c->max_pages < 1 || c->max_pages > INT32_MAX / (2 * KV4_PAGE))
        return fail(RSD_EINVAL, "%s: pages %d, kv heads %d, batch %d, pages per sequence %d", what, c->n_pages, c->n_kv_heads, c->batch, c->max_pages);
    if ((int64_t)c->batch * c->n_kv_heads > kMostBlocks / 4) return fail(RSD_EINVAL, "%s: batch %d x %d kv heads", what, c->batch, c->n_kv_heads);
    if (!aligned(c->pool, 16)) return fail(RSD_EINVAL, "%s: the pool is not 16-byte aligned", what);
    return RSD_OK;
}
Kv4Cache dev_cache(const rsd_kv4_cache* c) {
    return Kv4Cache{static_cast<uint8_t*>(c->pool), c->table, c->kv_len, c->n_pages, c->n_kv_heads, c->batch, c->max_pages};
}
Kv4Book dev_book(const rsd_kv4_book* b) {
    return b ? Kv4Book{b->scores, b->positions, b->score_b, b->score_h, b->position_b, b->position_h} : Kv4Book{};
}

// what is known of the entries, where it is changed: a list for each (sequence, kv head)
bool lists_overlap(const rsd_kv4_cache* c, int64_t batch_stride, int64_t head_stride) {
    return pieces_overlap(c->batch, batch_stride, c->n_kv_heads, head_stride, (int64_t)c->max_pages * KV4_PAGE);
}

struct AttnPlan {
    int tiles, waves, split, splits, w_cols, w_groups;
    bool many, by_length, fused;
    uint64_t o_bytes, ml_bytes, lse_bytes, w_bytes;
    uint64_t bytes() const { return o_bytes + ml_bytes + lse_bytes + w_bytes; }
};

// Which kernel, and how the entries are split (by the sizes that the host knows; times with launch):
//  - more than two tiles of columns share their decoded entries (64 sequences of 128 .. 5120 entries, bf16: 28 columns 42 us without, 58 with; 35 and 42 columns
//    62 either way; 56 columns 69 without, 65 with; fp32: 53 and 70, 79 and 80, 89 and 84).
//  - few columns: eight waves to a block up to 256 blocks (64 x 4 of 128 .. 5120 entries: 29 us against 33 with four), and up to 512 where lists are long
//    (128 x 4 of 512 .. 8192: 61 us against 74; 256 x 2 of 128 .. 2048: 30 against 26); else four (150 x 4: 52 against 65).
//    With fewer than 128 (sequence, kv head) pairs the entries are split for 512 blocks, down to two chunks a wave (one sequence, 2 x 8192 entries: 16 us, 26 with eight
//    chunks, 39 whole); with more, down to six (32 x 4 pairs of 8192: 31 us in two parts, 42 in three, 41 in four, 43 whole), because the parts have to be joined.
//  - many columns: up to 2048 blocks in parts of 20 chunks at least (64 x 4, 8 rows of 128 .. 5120: 65 us in four parts, 67 in seven, 120 whole; 16 x 4, 17 .. 128 rows of
//    512 .. 2560, bf16, two parts or whole, by which rows the longest sequences have: 69 or 81, 64 or 67, 72 or 72, 93 or 84), in smaller ones, down to six, only to
//    give every CU a block (40 rows of one sequence, 2 x 2048 entries: 49 us whole, 20 in parts of six).
//  - more blocks than run at once: the longest sequences first (64 x 4 x 2 tiles: 42 us against 53; 256 x 4 of 4096 .. 8192: 163 against 171); below that the order decides
//    nothing and costs 1 us.
//  - attention weights of more than one tile: the columns in groups of eight tiles at least, up to 4096 blocks of four chunks (16 x 8, 72B heads, with the attention, fp32:
//    295 us in two to four groups, 298 in eight, 314 in one).
AttnPlan attn_plan(const rsd_kv4_cache* c, const rsd_kv4_attn* a, bool scored) {
    AttnPlan p;
    const int64_t cols = (int64_t)a->max_rows * (a->n_heads / c->n_kv_heads);
    const int64_t max_kv = std::min<int64_t>(a->max_kv, (int64_t)c->max_pages * KV4_PAGE);
    const int64_t chunks = std::max<int64_t>(1, ceil_div(max_kv, KV4_CHUNK));
    p.many = cols > 32;
    p.tiles = (int)ceil_div(cols, p.many ? 64 : 16);
    const int64_t base = (int64_t)c->batch * c->n_kv_heads * p.tiles;
    int64_t parts;
    if (p.many) {
        p.waves = 4;
        parts = std::max(std::min(ceil_div(2048, base), chunks / 20), std::min(ceil_div(256, base), chunks / 6));
    } else {
        p.waves = (int)std::min<int64_t>(base <= 256 || (base <= 512 && chunks >= 48) ? 8 : 4, chunks);
        parts = std::min<int64_t>(ceil_div(512, base), chunks / (p.waves * (base < 128 ? 2 : 6)));
    }
    p.split = (int)(ceil_div(chunks, std::max<int64_t>(1, parts)) * KV4_CHUNK);
    p.splits = (int)ceil_div(chunks * KV4_CHUNK, p.split);
    p.by_length = base * p.splits * p.waves > 2048;
    const uint64_t lines = (uint64_t)a->rows * a->n_heads;
    p.o_bytes = p.splits > 1 ? up256(lines * p.splits * c->head_dim * 4) : 0;
    p.ml_bytes = p.splits > 1 ? up256(lines * p.splits * 8) : 0;
    p.fused = scored && !p.many && p.tiles == 1 && p.splits == 1;
    p.lse_bytes = scored && !p.fused ? up256(lines * 4) : 0;
    const int64_t tiles = ceil_div(cols, 16), pairs = (int64_t)c->batch * c->n_kv_heads;
    const int64_t groups = tiles == 1 ? 1 : std::max<int64_t>(1, std::min(4096 / (pairs * ceil_div(chunks, 4)), tiles / 8));
    p.w_cols = (int)(ceil_div(tiles, groups) * 16);
    p.w_groups = (int)ceil_div(tiles * 16, p.w_cols);
    p.w_bytes = scored && p.w_groups > 1 ? up256((uint64_t)(p.w_groups * pairs * chunks) * KV4_CHUNK * 4) : 0;
    return p;
}
int check_attn(const rsd_kv4_cache* c, const rsd_kv4_attn* a) {
    if (int rc = check_cache(c, "attention")) return rc;
    if (!a) return fail(RSD_EINVAL, "attention: null arguments");
    if (!is_type(a->dtype)) return fail(RSD_EINVAL, "attention: type %d", a->dtype);
    if (a->rows < 1 || a->max_rows < 1 || a->max_kv < 0) return fail(RSD_EINVAL, "attention: rows %d, at most %d a sequence, entries %d", a->rows, a->max_rows, a->max_kv);
    if (a->n_heads < 1 || a->n_heads % c->n_kv_heads) return fail(RSD_EINVAL, "attention: %d heads over %d kv heads", a->n_heads, c->n_kv_heads);
    if (!a->row_start && a->max_rows != 1) return fail(RSD_EINVAL, "attention: max_rows %d without row_start", a->max_rows);
    // columns of a (sequence, kv head) are counted in 32 bits; so are the threads of a launch: blocks of 256 for 64 columns each.  (Parts are made and joined for
    // fewer than 2048 blocks alone.)
    if ((int64_t)a->max_rows * a->n_heads > INT32_MAX / 16 || c->batch * c->n_kv_heads * ceil_div((int64_t)a->max_rows * (a->n_heads / c->n_kv_heads), 64) >= 1 << 24)
        return fail(RSD_EINVAL, "attention: %d rows x %d heads x %d sequences", a->max_rows, a->n_heads, c->batch);
    return RSD_OK;
}

template <typename T, int HD, int PLANES> void attn_run(const Kv4Attn& k, const AttnPlan& p, Launches& l) {
    const unsigned lists = (unsigned)(k.c.batch * k.c.hkv);
    const dim3 grid(lists, (unsigned)p.tiles, (unsigned)p.splits), many(lists * (unsigned)p.tiles, 1, (unsigned)p.splits);
    if (p.many && k.lse2) l.run(kv4_attn_many_kernel<T, HD, PLANES, KV4_LOGS>, many, 256, 0, k);
    else if (p.many) l.run(kv4_attn_many_kernel<T, HD, PLANES, KV4_NO_WEIGHTS>, many, 256, 0, k);
    else if (p.fused) l.run(kv4_attn_kernel<T, HD, PLANES, KV4_WEIGHTS>, grid, 64 * p.waves, 0, k);
    else if (k.lse2) l.run(kv4_attn_kernel<T, HD, PLANES, KV4_LOGS>, grid, 64 * p.waves, 0, k);
    else l.run(kv4_attn_kernel<T, HD, PLANES, KV4_NO_WEIGHTS>, grid, 64 * p.waves, 0, k);
    if (p.splits > 1)
        l.run(kv4_join_kernel<T, HD>, (unsigned)ceil_div((int64_t)k.c.batch * k.max_rows * k.heads, 16), 256, 0, k);
    if (k.book.scores && !p.fused) {
        const int64_t n = std::min<int64_t>(k.max_kv, (int64_t)k.c.max_pages * KV4_PAGE);
        const int64_t pairs = (int64_t)k.c.batch * k.c.hkv, chunks = ceil_div(n, 4 * KV4_CHUNK);
        if (n > 0 && (int64_t)k.max_rows * k.group <= 16)
            l.run(kv4_weight_kernel<T, HD, PLANES>, dim3((unsigned)pairs, (unsigned)std::min(chunks, ceil_div(1024, pairs))), 256, 0, k);
        else if (n > 0) {
            const unsigned y = (unsigned)std::min<int64_t>(chunks, 32768);
            l.run(kv4_weight_many_kernel<T, HD, PLANES>, dim3((unsigned)pairs, y, (unsigned)p.w_groups), 256, 0, k);
            if (p.w_groups > 1) l.run(kv4_weight_sum_kernel, dim3((unsigned)pairs, y), 256, 0, k);
        }
    }
}
template <typename T, int PLANES> void attn_run(const Kv4Attn& k, const AttnPlan& p, int hd, Launches& l) {
    if (hd == 32) attn_run<T, 32, PLANES>(k, p, l);
    else if (hd == 64) attn_run<T, 64, PLANES>(k, p, l);
    else attn_run<T, 128, PLANES>(k, p, l);
}
uint64_t up4(uint64_t n) { return (n + 3) & ~3ull; }
// the most entries of a list that can move, in whole vectors
int evict_moves(const rsd_kv4_cache* c, int budget) {
    return (int)up4(std::max<int64_t>(0, std::min<int64_t>(budget, (int64_t)c->max_pages * KV4_PAGE - budget)));
}

}  // namespace

extern "C" const char* rsd_op_last_error(void) { return op_error; }

extern "C" int rsd_w4_pack(const void* w, int32_t dtype, int64_t ld, int32_t n, int32_t k, void* codes, void* scales, void* hip_stream) {
    if (!w || !codes || !scales) return fail(RSD_EINVAL, "w4_pack: null array");
    if (!is_type(dtype)) return fail(RSD_EINVAL, "w4_pack: type %d", dtype);
    if (n < 1 || k < 1 || ld < k) return fail(RSD_EINVAL, "w4_pack: [%d][%d], rows %lld apart", n, k, (long long)ld);
    const int nt = (int)ceil_div(n, 16), kt = (int)ceil_div(k, 128), ks = (int)ceil_div(k, 512);
    const int64_t blocks = (int64_t)nt * ks * 16;        // 16 rows x 16 groups x 16 lanes of every 512 columns
    if (blocks > kMostBlocks) return fail(RSD_EINVAL, "w4_pack: [%d][%d] is too large", n, k);
    Launches l(hip_stream);
    if (dtype == RSD_F32)
        l.run(w4_pack_kernel<float>, (unsigned)blocks, 256, 0, static_cast<const float*>(w), ld, n, k, nt, kt, ks, static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales));
    else
        l.run(w4_pack_kernel<bf16_t>, (unsigned)blocks, 256, 0, static_cast<const bf16_t*>(w), ld, n, k, nt, kt, ks, static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales));
    return l.done("w4_pack");
}

extern "C" uint64_t rsd_w4_linear_workspace(int32_t rows, int32_t n, int32_t k, int32_t dtype) {
    if (rows < 1 || n < 1 || k < 1 || !is_type(dtype)) return 0;
    const W4Plan p = w4_plan(rows, n, k, dtype);
    return p.part_bytes;
}

extern "C" int rsd_w4_linear(const rsd_w4* w, const void* x, int64_t ldx, void* y, int64_t ldy, int32_t rows, int32_t dtype,
                             void* workspace, uint64_t workspace_bytes, void* hip_stream) {
    if (!w || !w->codes || !w->scales || !x || !y) return fail(RSD_EINVAL, "w4_linear: null array");
    if (!is_type(dtype)) return fail(RSD_EINVAL, "w4_linear: type %d", dtype);
    if (rows < 1 || w->n < 1 || w->k < 1 || ldx < w->k || ldy < w->n)
        return fail(RSD_EINVAL, "w4_linear: %d rows, [%d][%d], rows of x %lld apart, of y %lld", rows, w->n, w->k, (long long)ldx, (long long)ldy);
    if (!aligned(w->codes, 16) || !aligned(w->scales, 16)) return fail(RSD_EINVAL, "w4_linear: the weights are not 16-byte aligned");
    if (!aligned(x, size_of(dtype)) || !aligned(y, size_of(dtype))) return fail(RSD_EINVAL, "w4_linear: x or y is not aligned to its type");
    if ((int64_t)rows * w->n > kMostBlocks * 256 || rows > 1 << 20 || w->n > 1 << 26)
        return fail(RSD_EINVAL, "w4_linear: %d rows with [%d][%d] are too many", rows, w->n, w->k);
    if (share_memory({x, ldx, 0, w->k}, {y, ldy, 0, w->n}, rows, 1, size_of(dtype))) return fail(RSD_EINVAL, "w4_linear: y shares memory with x");
    const W4Plan p = w4_plan(rows, w->n, w->k, dtype);
    if (workspace_bytes < p.part_bytes || (p.part_bytes && (!workspace || !aligned(workspace, 256))))
        return fail(RSD_EINVAL, "w4_linear: the workspace holds %llu of %llu bytes, or is not 256-byte aligned",
                    (unsigned long long)workspace_bytes, (unsigned long long)p.part_bytes);
    const W4Args a{static_cast<const u32x4_t*>(w->codes), static_cast<const uint32_t*>(w->scales), w->n, w->k, p.nt, p.kt, p.ks, x, ldx, rows, y, ldy,
                   p.splits > 1 ? static_cast<float*>(workspace) : nullptr, p.tiles, p.splits};
    Launches l(hip_stream);
    if (dtype == RSD_F32) w4_run<float>(p, a, l);
    else w4_run<bf16_t>(p, a, l);
    return l.done("w4_linear");
}

extern "C" int rsd_kv4_append(const rsd_kv4_cache* c, const void* k, int64_t k_row, int64_t k_head, const void* v, int64_t v_row, int64_t v_head,
                              int32_t dtype, const int32_t* seq, const int32_t* slot, const int32_t* position, int32_t rows,
                              const rsd_kv4_book* book, void* hip_stream) {
    if (int rc = check_cache(c, "append")) return rc;
    if (!k || !v || !seq || !slot) return fail(RSD_EINVAL, "append: null array");
    if (!is_type(dtype) || rows < 1) return fail(RSD_EINVAL, "append: type %d, %d rows", dtype, rows);
    if (book && book->positions && !position) return fail(RSD_EINVAL, "append: positions are kept but none are given");
    if (!aligned(k, size_of(dtype)) || !aligned(v, size_of(dtype))) return fail(RSD_EINVAL, "append: k or v is not aligned to its type");
    const int64_t blocks = ceil_div(ceil_div(rows, 4) * 4 * c->n_kv_heads * (c->head_dim / 32), 64);
    if (blocks > kMostBlocks) return fail(RSD_EINVAL, "append: %d rows are too many", rows);
    Launches l(hip_stream);
    if (dtype == RSD_F32)
        l.run(kv4_append_kernel<float>, (unsigned)blocks, 256, 0, dev_cache(c), c->head_dim, static_cast<const float*>(k), k_row, k_head,
                                                                   static_cast<const float*>(v), v_row, v_head, seq, slot, position, rows, dev_book(book));
    else
        l.run(kv4_append_kernel<bf16_t>, (unsigned)blocks, 256, 0, dev_cache(c), c->head_dim, static_cast<const bf16_t*>(k), k_row, k_head,
                                                                    static_cast<const bf16_t*>(v), v_row, v_head, seq, slot, position, rows, dev_book(book));
    return l.done("append");
}

extern "C" int rsd_kv4_read(const rsd_kv4_cache* c, const int32_t* seq, const int32_t* slot, int32_t rows, void* k, void* v, int32_t dtype,
                            void* hip_stream) {
    if (int rc = check_cache(c, "read")) return rc;
    if (!k || !v || !seq || !slot) return fail(RSD_EINVAL, "read: null array");
    if (!is_type(dtype) || rows < 1) return fail(RSD_EINVAL, "read: type %d, %d rows", dtype, rows);
    if (!aligned(k, 16) || !aligned(v, 16)) return fail(RSD_EINVAL, "read: k or v is not 16-byte aligned");
    const int64_t blocks = ceil_div(ceil_div(rows, 4) * 4 * c->n_kv_heads * (c->head_dim / 32), 64);
    if (blocks > kMostBlocks) return fail(RSD_EINVAL, "read: %d rows are too many", rows);
    Launches l(hip_stream);
    if (dtype == RSD_F32) l.run(kv4_read_kernel<float>, (unsigned)blocks, 256, 0, dev_cache(c), c->head_dim, seq, slot, rows, static_cast<float*>(k), static_cast<float*>(v));
    else l.run(kv4_read_kernel<bf16_t>, (unsigned)blocks, 256, 0, dev_cache(c), c->head_dim, seq, slot, rows, static_cast<bf16_t*>(k), static_cast<bf16_t*>(v));
    return l.done("read");
}

extern "C" uint64_t rsd_kv4_attention_workspace(const rsd_kv4_cache* c, const rsd_kv4_attn* a, int32_t scored) {
    if (check_attn(c, a)) return 0;
    const AttnPlan p = attn_plan(c, a, scored != 0);
    return p.bytes();
}

extern "C" int rsd_kv4_attention(const rsd_kv4_cache* c, const rsd_kv4_attn* a, const rsd_kv4_book* book, void* workspace,
                                 uint64_t workspace_bytes, void* hip_stream) {
    if (int rc = check_attn(c, a)) return rc;
    if (!a->q || !a->out) return fail(RSD_EINVAL, "attention: null array");
    if (!aligned(a->q, size_of(a->dtype)) || !aligned(a->out, size_of(a->dtype))) return fail(RSD_EINVAL, "attention: q or out is not aligned to its type");
    const bool scored = book && book->scores;
    if (pieces_overlap(a->rows, a->out_row, a->n_heads, a->out_head, c->head_dim))
        return fail(RSD_EINVAL, "attention: rows of out overlap (strides %lld, %lld)", (long long)a->out_row, (long long)a->out_head);
    if (scored && lists_overlap(c, book->score_b, book->score_h))
        return fail(RSD_EINVAL, "attention: lists of scores overlap (strides %lld, %lld)", (long long)book->score_b, (long long)book->score_h);
    const AttnPlan p = attn_plan(c, a, scored);
    // A block has read its columns of q before it writes them, so out may be q itself; but weights that are added by a kernel of their own need q once more.
    const bool same = a->out == a->q && (a->rows == 1 || a->out_row == a->q_row) && (a->n_heads == 1 || a->out_head == a->q_head);
    if (same ? scored && !p.fused
             : share_memory({a->q, a->q_row, a->q_head, c->head_dim}, {a->out, a->out_row, a->out_head, c->head_dim}, a->rows, a->n_heads, size_of(a->dtype)))
        return fail(RSD_EINVAL, "attention: out shares memory with q%s", same ? ", which the weights need again" : "");
    const uint64_t need = p.bytes();
    if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 256))))
        return fail(RSD_EINVAL, "attention: the workspace holds %llu of %llu bytes, or is not 256-byte aligned", (unsigned long long)workspace_bytes, (unsigned long long)need);
    char* ws = static_cast<char*>(workspace);
    Kv4Attn k{};
    k.c = dev_cache(c);
    k.q = a->q, k.q_row = a->q_row, k.q_head = a->q_head;
    k.row_start = a->row_start, k.total_rows = a->rows, k.max_rows = a->max_rows, k.heads = a->n_heads, k.group = a->n_heads / c->n_kv_heads;
    k.scale = a->scale;
    k.plain = !(std::fabs(a->scale) > 0.f);
    k.factor2 = k.plain ? 1.f : (float)(std::fabs((double)a->scale) * 1.4426950408889634);
    k.negative = a->scale < 0.f;
    k.out = a->out, k.o_row = a->out_row, k.o_head = a->out_head;
    k.lse = a->lse;
    k.lse2 = p.lse_bytes ? reinterpret_cast<float*>(ws + p.o_bytes + p.ml_bytes) : nullptr;
    k.max_kv = a->max_kv, k.tiles = p.tiles, k.split = p.split, k.splits = p.splits, k.by_length = p.by_length, k.hd = c->head_dim;
    k.part_o = reinterpret_cast<float*>(ws);
    k.part_ml = reinterpret_cast<float2*>(ws + p.o_bytes);
    if (scored) k.book = dev_book(book);
    k.w_cols = p.w_cols, k.w_groups = p.w_groups;
    k.w_slots = ceil_div(std::min<int64_t>(a->max_kv, (int64_t)c->max_pages * KV4_PAGE), KV4_CHUNK) * KV4_CHUNK;
    k.part_w = reinterpret_cast<float*>(ws + p.o_bytes + p.ml_bytes + p.lse_bytes);
    Launches l(hip_stream);
    if (a->dtype == RSD_F32) attn_run<float, 3>(k, p, c->head_dim, l);
    else attn_run<bf16_t, 1>(k, p, c->head_dim, l);
    return l.done("attention");
}

extern "C" uint64_t rsd_kv4_evict_workspace(const rsd_kv4_cache* c, int32_t budget) {
    if (check_cache(c, "evict") || budget < 1) return 0;
    const int moves = evict_moves(c, budget);
    return moves ? up256((uint64_t)c->batch * c->n_kv_heads * (4 + up4(budget) + moves) * 4) : 0;      // (none: no list can hold more than the budget)
}

extern "C" int rsd_kv4_evict(const rsd_kv4_cache* c, const rsd_kv4_book* book, int32_t budget, int32_t recent, void* workspace,
                             uint64_t workspace_bytes, void* hip_stream) {
    if (int rc = check_cache(c, "evict")) return rc;
    if (!book || !book->scores || !book->positions) return fail(RSD_EINVAL, "evict: scores and positions are needed");
    if (budget < 1 || recent < 0 || recent > budget) return fail(RSD_EINVAL, "evict: budget %d, recent %d", budget, recent);
    if (lists_overlap(c, book->score_b, book->score_h) || lists_overlap(c, book->position_b, book->position_h))
        return fail(RSD_EINVAL, "evict: lists of scores or positions overlap (strides %lld, %lld and %lld, %lld)", (long long)book->score_b, (long long)book->score_h,
                    (long long)book->position_b, (long long)book->position_h);
    const uint64_t need = rsd_kv4_evict_workspace(c, budget);
    if (need && (workspace_bytes < need || !workspace || !aligned(workspace, 256)))
        return fail(RSD_EINVAL, "evict: the workspace holds %llu of %llu bytes, or is not 256-byte aligned", (unsigned long long)workspace_bytes, (unsigned long long)need);
    const Kv4Evict e{dev_cache(c), dev_book(book), budget, recent, static_cast<int*>(workspace), evict_moves(c, budget)};
    if (e.moves == 0) return RSD_OK;
    Launches l(hip_stream);
    const unsigned lists = (unsigned)(c->batch * c->n_kv_heads);
    const int64_t slots = (int64_t)c->max_pages * KV4_PAGE;
    if (slots <= 16384) l.run(kv4_select_kernel<true>, lists, 1024, (size_t)slots * 4, e, c->n_kv_heads);
    else l.run(kv4_select_kernel<false>, lists, 1024, 0, e, c->n_kv_heads);
    // four pages to a block at a time; at most 64 blocks to a list, which then go on with the next 256
    const dim3 grid(lists, (unsigned)std::min<int64_t>(64, ceil_div(ceil_div(budget, KV4_PAGE), 4)));
    if (c->head_dim == 32) l.run(kv4_move_kernel<32>, grid, 256, 0, e, c->n_kv_heads);
    else if (c->head_dim == 64) l.run(kv4_move_kernel<64>, grid, 256, 0, e, c->n_kv_heads);
    else l.run(kv4_move_kernel<128>, grid, 256, 0, e, c->n_kv_heads);
    return l.done("evict");
}
