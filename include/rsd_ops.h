/*
 * rsd_ops.h - operators of a decode step whose memory is 4 bits wide, on AMD MI355X (gfx950): products with 4-bit
 * weights, a paged 4-bit KV cache (writing, reading, attention), and eviction from that cache by accumulated attention
 * weight.
 *
 * Conventions
 *  - "dev" pointers are device addresses.  Calls enqueue their kernels on hip_stream (a hipStream_t, NULL: the default
 *    stream) and return; they allocate nothing and do not synchronise, so they may be recorded into a HIP graph.
 *    Device memory that a call needs beside its arguments is a workspace of the caller's, 256-byte aligned, of at least the size the
 *    matching ..._workspace function returns for the same sizes (0: none).  It is free again once the stream has passed the
 *    call; calls that may run at the same time need one each.
 *  - Strides count elements.  The innermost dimension of every array is contiguous.  Rows of q, k and v may overlap; rows of an array that a call
 *    writes to may not: the products, the attention and the eviction refuse such arrays.
 *  - Every entry point returns RSD_OK (0), RSD_EINVAL (bad shape or argument; nothing was enqueued) or RSD_EHIP;
 *    rsd_op_last_error() is the text of the calling thread's last failure.  Nothing aborts or throws.
 *  - Values that live on the device (lengths, tables, row numbers) cannot be checked before the launch.  The kernels check them: a
 *    length is cut to what its table can hold, and a table entry, sequence or slot outside its range stands for no entry
 *    (nothing is written, attention does not see it, reading gives zeros).
 *  - Data types: RSD_F32, RSD_BF16 (rsd.h).
 *
 * The 4-bit format.  32 consecutive values along the contracted axis (columns of a weight row; the head dimension of a
 * key or value) form a group with one scale 2^(s - 127), a byte s.  A value is 4 bits: a sign and one of 0, .5, 1, 1.5, 2, 3,
 * 4, 6 (two exponent bits, one fraction bit).  The scale is the least power of two 2^e with max|x| <= 7 * 2^e, e within -125 .. 125;
 * x / 2^e is rounded to the nearest value, ties to the even code, at most 6.  A group that holds a NaN or an infinity gets s = 255 and
 * reads as NaN.  Two values share a byte, the first in the low half.
 */
#ifndef RSD_OPS_H
#define RSD_OPS_H

#include <stdint.h>
#include "rsd.h"

#ifdef __cplusplus
extern "C" {
#endif

const char *rsd_op_last_error(void);

/* ---- products with 4-bit weights ----
 * A matrix W [n][k] in tiles of 16 rows x 128 columns, zero beyond n and k (NT = ceil(n/16), KT = ceil(k/128), KS = ceil(k/512)):
 *   codes  dev [NT][KT][4 groups][16 rows][16 bytes]     the 32 values of group g of a row
 *   scales dev [NT][KS][4 groups][16 rows][4 tiles]      scale byte of column tile 4 * ks + i
 * Both 16-byte aligned. */
typedef struct rsd_w4 {
    const void *codes, *scales;
    int32_t n, k;
} rsd_w4;

/* w dev [n][k], rows ld >= k elements apart, to codes and scales (dev, sizes as above).  NT * KS up to 2^18. */
int rsd_w4_pack(const void *w, int32_t dtype, int64_t ld, int32_t n, int32_t k, void *codes, void *scales, void *hip_stream);

/* y[r][i] = sum_j x[r][j] W[i][j] for rows of x, any number >= 1.  x dev [rows][k] (rows ldx apart) and y dev [rows][n] (rows ldy apart)
 * are of one type and share no memory; rows up to 2^20, n up to 2^26, rows * n up to 2^30.  Products are exact and summed in fp32 (an fp32 x enters with all its 24 bits); y is rounded once.  The order of the
 * sum depends on the sizes only. */
uint64_t rsd_w4_linear_workspace(int32_t rows, int32_t n, int32_t k, int32_t dtype);
int rsd_w4_linear(const rsd_w4 *w, const void *x, int64_t ldx, void *y, int64_t ldy, int32_t rows, int32_t dtype,
                  void *workspace, uint64_t workspace_bytes, void *hip_stream);

/* ---- a paged KV cache in 4 bits ----
 * Pages of 16 tokens: pool dev [n_pages][n_kv_heads][17 * head_dim bytes], 16-byte aligned; table dev [batch][max_pages]
 * (page of each sequence's 16 tokens, -1: none; pages may not be shared by sequences that write); kv_len dev [batch], the entries of each
 * sequence.  head_dim 32, 64 or 128.  Entries keep no order that matters: attention sees them as a set, except that the rows
 * of one call see the newest entries one by one.  Keys are stored as they are scored (rotated before they are written).
 * Inside a (page, kv head), G = head_dim / 32, token t of 16:
 *   key codes    [4 quarters of the head dimension][16 t][head_dim / 8 bytes]
 *   value codes  [t / 4][dim % 16][G][t % 4]: a byte holds dims m and m + 16 of its group
 *   key scales   [G][16 t]
 *   value scales [t / 4][G][t % 4]
 * Sizes: batch * n_kv_heads up to 2^20, max_pages up to 2^26 - 1; rows of a call that writes or reads entries (in whole fours) * n_kv_heads * head_dim / 32 up to
 * 2^28. */
typedef struct rsd_kv4_cache {
    void *pool;
    const int32_t *table;
    int32_t *kv_len;
    int32_t n_pages, n_kv_heads, head_dim, batch, max_pages;
} rsd_kv4_cache;

/* What is known of each entry beside its key and value, dev arrays [batch][n_kv_heads][slots] with slots >= 16 * max_pages: the
 * attention weight it has received and the position of its token.  Strides of the first two dimensions. */
typedef struct rsd_kv4_book {
    float *scores;
    int32_t *positions;
    int64_t score_b, score_h, position_b, position_h;
} rsd_kv4_book;

/* Writes entries: row i (keys and values [n_kv_heads][head_dim], dev, row and head strides) becomes slot[i] of sequence seq[i] (dev int32
 * [rows]; the pairs must differ).  kv_len is neither read nor changed.  With book (may be NULL; either array may be NULL) the entry's
 * score becomes 0 and its position position[i] (dev int32 [rows], needed with book->positions). */
int rsd_kv4_append(const rsd_kv4_cache *c, const void *k, int64_t k_row, int64_t k_head, const void *v, int64_t v_row,
                   int64_t v_head, int32_t dtype, const int32_t *seq, const int32_t *slot, const int32_t *position,
                   int32_t rows, const rsd_kv4_book *book, void *hip_stream);

/* Reads entries back: k, v dev [rows][n_kv_heads][head_dim], contiguous, the values the cache holds (exact in both types). */
int rsd_kv4_read(const rsd_kv4_cache *c, const int32_t *seq, const int32_t *slot, int32_t rows, void *k, void *v,
                 int32_t dtype, void *hip_stream);

/* Attention of new tokens over the cache (their own entries included).  Sequence b has the rows row_start[b] .. row_start[b + 1] - 1 (dev
 * [batch + 1]; NULL: row b alone), at most max_rows of them (further ones are not computed), and n = min(kv_len[b], max_kv) entries.  Row j of its q rows sees the entries in
 * slots < n - (q - 1 - j).  q, out dev [rows][n_heads][head_dim] with row and head strides; head h reads kv head h / (n_heads /
 * n_kv_heads).  out = softmax(scale q.K) V; a row that sees nothing, or scores -inf with all that it sees, gives 0.  lse (dev [rows][n_heads] or NULL) = log of
 * the sum of exp(scale q.k), -inf for such rows, which deal out no weight either.  With scores in book (NULL: none) every entry's score grows by the softmax weights it received, summed over the rows
 * and the heads of its group.  Sizes: batch * n_kv_heads * (max_rows * n_heads / n_kv_heads in
 * whole 64s) below 2^30, max_rows * n_heads below 2^27.  out may be q itself where no scores are given, and shares no memory with it else. */
typedef struct rsd_kv4_attn {
    const void *q;
    void *out;
    float *lse;
    int64_t q_row, q_head, out_row, out_head;
    const int32_t *row_start;
    int32_t rows, max_rows, n_heads, max_kv, dtype;
    float scale;
} rsd_kv4_attn;
uint64_t rsd_kv4_attention_workspace(const rsd_kv4_cache *c, const rsd_kv4_attn *a, int32_t scored);
int rsd_kv4_attention(const rsd_kv4_cache *c, const rsd_kv4_attn *a, const rsd_kv4_book *book, void *workspace,
                      uint64_t workspace_bytes, void *hip_stream);

/* Eviction: of the entries of every (sequence, kv head) that has more than `budget`, keeps the ones whose position is
 * within `recent` of the newest, then those of the highest score (NaN: lowest), ties to the lower slot, `budget` in all.  Positions may repeat: where more than
 * `budget` entries are that new, those of the highest score among them stay.  Kept entries in slots
 * >= budget move, with score and position, into the slots freed below it: the i-th of them in slot order into the i-th
 * freed one.  kv_len becomes min(kv_len, budget); what lies behind it is left as it was.  0 <= recent <= budget, budget >= 1; book with both
 * arrays.  Every slot below kv_len needs its page here: entries without one are ranked like the others, but there is nothing to move, and what moves to a slot without one is
 * lost. */
uint64_t rsd_kv4_evict_workspace(const rsd_kv4_cache *c, int32_t budget);
int rsd_kv4_evict(const rsd_kv4_cache *c, const rsd_kv4_book *book, int32_t budget, int32_t recent, void *workspace,
                  uint64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif
