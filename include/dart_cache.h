/*
 * dart_cache.h -- paged key/value cache of the target model and the tree
 * attention that reads it (GB300, sm_103a).
 *
 * dart_tree_attention (include/dart_verify.h) takes one contiguous bf16
 * context of one length.  Here sequences of different lengths share a pool of
 * pages, in bf16 or in 8 bits, and the pass has the row of the last verified
 * token (the root of the draft tree) beside the tree's nodes, so that with no
 * nodes it is the decoding of single tokens.
 *
 *   K, V pools   [num_pages][Hkv][page_size][dh], bf16 or e4m3
 *   their scales [num_pages][Hkv][page_size] fp32 (e4m3 only): an element
 *                stands for code * scale; K is stored rotated (RoPE)
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

typedef struct {
    int num_pages; /* pages in the pool, >= 1 */
    int page_size; /* tokens per page: 16, 32, 64 or 128 */
    int Hkv;       /* kv heads, >= 1 */
    int dh;        /* head dimension; 128 */
    int dtype;     /* DART_KV_BF16 or DART_KV_E4M3 */
    void *k, *v;   /* the pools, 16-byte aligned */
    float *k_scale, *v_scale; /* 16-byte aligned; NULL for bf16 */
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
 * NaN when it is read.  Positions past max_pages * page_size are not written
 * and set value 4 in *status.  No other
 * slot changes; lens is not advanced.  Two tokens of one call must not fall on
 * one slot (two sequences that share a page and both write in it). */
int dart_cache_append(const dart_kv_cache *cache, int nseq, int max_pages, const int32_t *page_table,
                      const int32_t *lens, int R, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                      const int32_t *rows, const int32_t *n_rows, float rope_theta, int *status, void *stream);

typedef struct {
    int nseq;         /* sequences, >= 1 */
    int B;            /* tree nodes per sequence, 0..1024; R = B + 1 rows */
    int max_pages;    /* row length of page_table, >= 1 */
    int Hq;           /* query heads; Hq / Hkv in {1, 2, 4, 8, 16} */
    float rope_theta; /* RoPE base, > 1 */
    float scale;      /* softmax scale, > 0 */
} dart_paged_attn_config;

/* Device workspace (bytes) of dart_paged_attention; 0 on an invalid
 * configuration.  For large trees over e4m3 pages it has room for the f16 form
 * of max_pages pages a sequence, where that takes at most 4 GB. */
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

#ifdef __cplusplus
}
#endif

#endif /* DART_CACHE_H */
