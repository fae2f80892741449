/*
 * dart_cache.h -- paged key/value cache of the target model and the tree
 * attention that reads it (GB300, sm_103a).
 *
 * dart_tree_attention (include/dart_verify.h) takes one contiguous bf16
 * context of one length.  Here sequences of different lengths share a pool of
 * pages, in bf16, 8 or 4 bits, and the pass has the row of the last verified
 * token (the root of the draft tree) beside the tree's nodes, so that with no
 * nodes it is the decoding of single tokens.
 *
 *   K, V pools   [num_pages][Hkv][page_size][dh], bf16, e4m3 or e2m1 (two
 *                codes a byte, the even element's in its low half)
 *   their scales [num_pages][Hkv][page_size] fp32 (e4m3 and e2m1), >= 0
 *   their blocks [num_pages][Hkv][page_size][dh / 16] e4m3 (e2m1 only), >= 0:
 *                an element stands for code * scale, or code * block * scale
 *                with the block scale of its 16 elements.  K is stored
 *                rotated (RoPE)
 *   page_table   [nseq][max_pages] int32: token p of sequence s is slot
 *                p % page_size of page page_table[s][p / page_size]
 *   lens         [nseq] int32: tokens of each sequence in the cache
 *
 * Rows of a pass, R = B + 1 per sequence: row 0 is the last verified token,
 * at position lens[s]; row 1 + i is tree node i, at lens[s] + depths[s][i].
 * The tree arrays are those of dart_prune_and_emit (include/dart.h).
 *
 * Conventions: DEVICE pointers of the current device, asynchronous on
 * `stream` (a cudaStream_t, NULL = legacy default stream), return 0 or a
 * negative dart_status code of include/dart.h; argument errors are detected
 * on the host before anything is enqueued.  Lengths and page numbers are read
 * on the device (a captured graph can be replayed for other ones): a length
 * outside [0, max_pages * page_size] counts as the nearer end, and no page
 * outside [0, num_pages) is accessed -- its use sets value 4 in *status (a
 * device int the caller zeroes; may be NULL) and leaves the results of that
 * sequence unspecified.  What a call reads must not change before the stream
 * has reached its end.
 */
#ifndef DART_CACHE_H
#define DART_CACHE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DART_KV_BF16 0
#define DART_KV_E4M3 1
#define DART_KV_E2M1 2

typedef struct {
    int num_pages; /* pages in the pool, >= 1 */
    int page_size; /* tokens per page: 16, 32, 64 or 128 */
    int Hkv;       /* kv heads, >= 1 */
    int dh;        /* head dimension; 128 */
    int dtype;     /* DART_KV_BF16, DART_KV_E4M3 or DART_KV_E2M1 */
    void *k, *v;   /* the pools, 16-byte aligned */
    float *k_scale, *v_scale; /* 16-byte aligned; NULL for bf16 */
    void *k_block, *v_block;  /* e2m1: the block scales, 16-byte aligned; not looked at for other types */
} dart_kv_cache;

/* Writes n_rows[s] (clamped to [0, R]) tokens of every sequence into its
 * pages, at positions lens[s], lens[s] + 1, ...: token i comes from row
 * rows[s * R + i] of the R given ones, or from row i if rows is NULL (a row
 * outside [0, R) is skipped and sets value 4 in *status).
 *   k, v   bf16: row r of sequence s at element (s * R + r) * stride, its Hkv
 *          heads of dh elements one after the other; stride (a multiple of
 *          8, >= Hkv * dh) makes slices of a fused projection possible
 * K is rotated at the token's position p (rotate-half form, angles to 2^-26 +
 * p 2^-54 of a turn) in fp32.  bf16 pools hold the rounded values; e4m3 pools
 * scale = max |x| / 448 of the token's head (at least 2^-120; 1 if it is all
 * zero) and x / scale, quotients rounded to fp32 and then to e4m3.  A NaN stays
 * one in its place (in K in its rotated pair), an infinity makes the whole head
 * NaN when it is read.
 * e2m1 pools: a row's scale is a power of two, 2^-10 times the one at or below
 * its largest magnitude (at least 2^-120; 1 if it is all zero), so that x /
 * scale is exact; a block scale is its 16 elements' largest magnitude / scale /
 * 6 rounded to e4m3 (at most 352; it may be 0), and a code x / scale / block
 * rounded to e2m1, both to nearest, ties to even, magnitudes above 6 to 6.
 * What is rounded of K is its rotation at frequencies of 53 bits, to 2^-44 of a
 * pair's length (against exact frequencies p 2^-52.6 more): where the one in fp32
 * leaves a scale or a code open, it is formed again.
 * A NaN or an infinity makes its block (in K, that of its rotated pair too)
 * NaN when it is read and counts for no scale.
 * Positions past max_pages * page_size are not written
 * and set value 4 in *status.  No other
 * slot changes; lens is not advanced.  Two tokens of one call must not fall on
 * one slot (two sequences that share a page and both write in it). */
int dart_cache_append(const dart_kv_cache *cache, int nseq, int max_pages, const int32_t *page_table,
                      const int32_t *lens, int R, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                      const int32_t *rows, const int32_t *n_rows, float rope_theta, int *status, void *stream);

/* Gives tokens of the cache back: tokens lens[s] .. lens[s] + n_rows[s] - 1
 * (n_rows clamped to [0, R]) of every sequence as rows 0, 1, ... of sequence s
 * of k and v (bf16, rows with strides as in dart_cache_append): code * block *
 * scale rounded to fp32 and then to bf16, K as it is stored (rotated).  Rows from n_rows[s] on
 * and what lies between rows are not written; a position past max_pages *
 * page_size or a page outside [0, num_pages) leaves its row as it was and sets
 * value 4 in *status. */
int dart_cache_read(const dart_kv_cache *cache, int nseq, int max_pages, const int32_t *page_table,
                    const int32_t *lens, int R, void *k, int64_t k_stride, void *v, int64_t v_stride,
                    const int32_t *n_rows, int *status, void *stream);

/* Copies whole pages, keys and values with their scales: the first *count
 * (clamped to [0, max_pairs]) pairs (from, to) of pairs [max_pairs][2], as
 * dart_page_pool_reserve and dart_page_pool_compact leave them.  No page may be
 * the `to` of two pairs, or the `to` of one and the `from` of another.  A pair
 * with a page outside [0, num_pages) is skipped and sets value 4 in *status. */
int dart_cache_copy_pages(const dart_kv_cache *cache, const int32_t *pairs, int max_pairs, const int32_t *count,
                          int *status, void *stream);

/* ---- who holds which page --------------------------------------------------
 *
 * The pages of a cache (or of several that share a table, one for each layer)
 * and the sequences that hold them; sequences may share pages.  All of it is
 * device memory, so that the calls need no host step and can be captured:
 *   refs  [num_pages]         sequences that hold each page; 0: a free page
 *   table [nseq][max_pages]   the page tables: entries [0, held[s]) of row s are
 *                             pages, what stands behind them is not looked at
 *   held  [nseq]              pages of each sequence
 * A fresh pool is all zeros.  page_table of the other calls is `table`, lens
 * are the caller's.  Held counts are clamped to [0, max_pages], lengths to [0,
 * max_pages * page_size].  A table entry that should be a page and lies outside
 * [0, num_pages) sets value 4 in *status and counts for nothing.  Results do not
 * depend on the order in which threads run.  One call at a time works on a
 * pool: calls on different streams have to be ordered by events.
 * `workspace`: dart_page_pool_workspace bytes, 256-byte aligned, in use until
 * the stream reaches the call's end; nothing is kept in it between calls. */
typedef struct {
    int num_pages; /* >= 1 */
    int page_size; /* tokens per page: 16, 32, 64 or 128 */
    int nseq;      /* sequences, >= 1 */
    int max_pages; /* row length of table, >= 1; nseq * max_pages and max_pages * page_size <= 2^30 */
    int32_t *refs; /* 16-byte aligned */
    int32_t *table;
    int32_t *held;
} dart_page_pool;

size_t dart_page_pool_workspace(const dart_page_pool *pool); /* 0: invalid */

/* Sequences become continuations of others, all at once from the state before
 * the call: parents[s] = s leaves sequence s as it is; p != s makes it a copy of
 * sequence p (it gives its pages back and holds the first ceil(lens[p] /
 * page_size) of p's instead, lens[s] = lens[p]); -1 ends it (it gives its
 * pages back, lens[s] = 0).  Any other value leaves s as it is and sets value
 * 4 in *status.  lens [nseq] is changed in place. */
int dart_page_pool_select(const dart_page_pool *pool, const int32_t *parents, int32_t *lens, void *workspace,
                          size_t workspace_bytes, int *status, void *stream);

/* Room for n_rows[s] more tokens from position lens[s] on, on pages that no
 * other sequence holds: of the pages that these tokens fall on, the ones that
 * sequence s does not have yet or shares are replaced by free ones, lowest
 * numbers first in the order of sequences and then positions.  Where a shared
 * page has tokens before lens[s], the pair (it, its replacement) is listed in
 * pairs [max_pairs][2] (max_pairs >= nseq), in the order of sequences, for
 * dart_cache_copy_pages, which has to come before the pages' next use; *count is
 * their number.  Two sequences that share a page and are both given room in it
 * get a copy each.  A sequence that the table's row or the free pages do not
 * suffice for (and, for the free pages, every later one that needs some) is
 * left as it is and sets value 8 in *status.  n_rows[s] <= 0 asks for nothing.
 * A sequence without room must not be written to: its table still has the pages
 * that it shares, and behind those numbers that may be other sequences' pages.
 * dart_page_pool_reserve_rows says so on the device: granted[s] is n_rows[s] where
 * there is room, else 0 (also where n_rows[s] < 0); it is what dart_cache_append
 * takes as n_rows and what the caller's lens grow by (or the smaller of it and the
 * rows that are kept).  granted may be n_rows itself. */
int dart_page_pool_reserve(const dart_page_pool *pool, const int32_t *lens, const int32_t *n_rows, int32_t *pairs,
                           int max_pairs, int32_t *count, void *workspace, size_t workspace_bytes, int *status,
                           void *stream);
int dart_page_pool_reserve_rows(const dart_page_pool *pool, const int32_t *lens, const int32_t *n_rows,
                                int32_t *granted, int32_t *pairs, int max_pairs, int32_t *count, void *workspace,
                                size_t workspace_bytes, int *status, void *stream);

/* Gives back every page behind the first ceil(lens[s] / page_size) of sequence s. */
int dart_page_pool_trim(const dart_page_pool *pool, const int32_t *lens, int *status, void *stream);

/* Moves the pages in use to the front: with n of them, those with numbers >= n
 * go to the free numbers below n, both in ascending order; refs and table
 * follow, and pairs [max_pairs][2] (max_pairs >= num_pages / 2), *count list
 * the moves for dart_cache_copy_pages, which has to come before the pages'
 * next use. */
int dart_page_pool_compact(const dart_page_pool *pool, int32_t *pairs, int max_pairs, int32_t *count, void *workspace,
                           size_t workspace_bytes, int *status, void *stream);

typedef struct {
    int nseq;         /* sequences, >= 1 */
    int B;            /* tree nodes per sequence, 0..1024; R = B + 1 rows */
    int max_pages;    /* row length of page_table, >= 1 */
    int Hq;           /* query heads; Hq / Hkv in {1, 2, 4, 8, 16} */
    float rope_theta; /* RoPE base, > 1 */
    float scale;      /* softmax scale, > 0 */
} dart_paged_attn_config;

/* Device workspace (bytes) of dart_paged_attention; 0 on an invalid
 * configuration.  For large trees over e4m3 or e2m1 pages (five tiles of 128 query
 * rows a kv head and more) it has room for the f16 form of max_pages pages a
 * sequence, whatever the lengths are: 512 bytes a token and kv head, where the
 * pages themselves take 264 or 152.  Where that would be more than 4 GB it has
 * none, and every query tile converts the pages for itself. */
size_t dart_paged_attention_workspace(const dart_paged_attn_config *cfg, const dart_kv_cache *cache);

/* One tree-attention layer over the cache:
 *   q    = RoPE(Q[s][r][h], position of r)
 *   keys = cache tokens 0 .. lens[s] - 1 of kv head g = h / (Hq / Hkv),
 *          RoPE(k[s][j][g], position of j) for row j = 0 and, where bit j - 1
 *          of mask[s][r - 1] is set, for row j <= r (ancestors come before
 *          their descendants: bits of rows > r are ignored, in every row);
 *          row 0 sees itself and the cache alone
 *   out[s][r][h] = softmax(scale * q . keys) . values;  rows > n_nodes[s]: 0
 * Layouts (bf16 unless stated): q [nseq * R] rows of Hq * dh, k and v
 * [nseq * R] rows of Hkv * dh, each with a stride between rows (elements, a
 * multiple of 8); out [nseq][R][Hq][dh], dense; depths [nseq][B] int32, mask
 * [nseq][B][ceil(B / 64)] uint64, n_nodes [nseq] int32 (all three may be NULL
 * if B = 0).  Nothing is written to the cache: dart_cache_append writes the
 * rows that the pass keeps.  Every key and value in use must be finite;
 * slots past lens[s] and rows past n_nodes[s] may hold anything.
 * Over pages of codes values are weighed in f16, so those that lie far (2^-20
 * and beyond) below the largest of their head and sequence keep fewer bits; rows
 * of zeros (e2m1: whose block scales are all 0) count for nothing there, whatever
 * their scale is.
 *   workspace: 256-byte aligned, used by this call only until the stream
 *   reaches its end (no state is kept between calls); two calls that may run
 *   at the same time need one each.
 * Value 1 in *status: a bounded device wait gave up and `out` is
 * unspecified.  DART_ERR_UNSUPPORTED: the device is not sm_103a. */
int dart_paged_attention(const dart_paged_attn_config *cfg, const dart_kv_cache *cache, const int32_t *page_table,
                         const int32_t *lens, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                         const void *v, int64_t v_stride, const int32_t *depths, const uint64_t *mask,
                         const int32_t *n_nodes, void *out, void *workspace, size_t workspace_bytes, int *status,
                         void *stream);

/* Test hook of dart_paged_attention's bounded waits, in a library compiled with
 * -DDART_DEBUG: calls made from now on take the wait that softmax warp `warp` of
 * each CTA of the 128-row tiles ends its part number `part` with for one that gave
 * up (negative: none).  Nothing waits longer: the call ends with value 1 in
 * *status.  Other builds: DART_ERR_UNSUPPORTED, unless both are negative. */
int dart_test_paged_wait(int warp, int part);

#ifdef __cplusplus
}
#endif

#endif /* DART_CACHE_H */
