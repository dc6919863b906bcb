/*
 * attn_paged.h -- C ABI of the paged key/value cache: appending to it and attention over it.  Same library, status
 * codes and conventions as attn.h (device pointers of the caller, kernels enqueued on `hip_stream`, nothing allocated
 * or synchronised, arguments checked on the host before anything is launched).
 *
 * The batch is packed: sequence b has the rows q_start[b] .. q_start[b+1]-1 of Q, O, K and V, n_b of them (none is
 * allowed), and kv_lens[b] = L_b keys in the cache, its new rows among them: they are its last ones.  Row i of
 * sequence b therefore has the position p = L_b - n_b + i.  q_start, kv_lens and the page table are int32 in DEVICE
 * memory, so that a captured graph serves whatever they hold when it is replayed.  Rows from q_start[B] on belong to
 * nobody: they are neither read nor written.
 *
 * A cache is [pages][Hkv][page_size][D] by the strides cache_stride_p, cache_stride_h, cache_stride_s (elements, D
 * contiguous); position p of sequence b lies in page page_table[b][p / page_size], slot p % page_size.  It holds
 *   - 16-bit elements of the tensors' type, or
 *   - e4m3 codes (8 bits: OCP float8 with 4 exponent and 3 mantissa bits, largest value 448) where k_scale and v_scale
 *     are given: fp32 [pages][Hkv], contiguous, the value of a code is code * scale[page][head].  The attention takes
 *     any scale that is 0 or a positive normal number; attn_paged_append writes powers of two.  A code times
 *     its scale lies in the range of the tensors' type.
 *
 * What device memory holds is not checked on the host.  The kernels stay inside their buffers whatever it is:
 *   - L_b counts as within 0 .. table_width * page_size, row ranges as within 0 .. T;
 *   - a page id outside 0 .. pages-1 is no page: nothing is written there, and its keys are not seen;
 *   - a row at a negative position (L_b < n_b) is not appended, and under a causal mask sees nothing.
 * Slots from L_b on are never read as values: they may hold anything.  Values in the cache up to L_b, in Q, K and V
 * are finite.
 */
#ifndef MI355_ATTN_PAGED_H
#define MI355_ATTN_PAGED_H

#include "attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int32_t T;            /* rows of Q, O, K, V (0: nothing is done)                                        */
    int32_t B;            /* sequences (0: nothing is done)                                                 */
    int32_t Hq, Hkv;      /* Hkv divides Hq; query heads h * Hq/Hkv .. share K/V head h                     */
    int32_t D;            /* a multiple of 8 (of 16 with an e4m3 cache), at most 256                        */
    int32_t pages;        /* pages of the cache                                                             */
    int32_t page_size;    /* keys of a page: a power of two, 16 .. 4096                                     */
    int32_t table_width;  /* entries of a row of the page table; table_width * page_size is at most 2^30    */
    int32_t table_stride; /* distance of its rows in entries, table_width at least                          */
    int32_t max_q;        /* attention: no sequence has more rows than this (1: decoding).  Rows of a sequence
                             that has more are left as they were.  T is always right.                       */
    int32_t causal;       /* attention: row at position p sees keys 0 .. p; otherwise all L_b               */
    int32_t rot;          /* append: columns that are rotated, 0 or a multiple of 8 up to D                 */
    int32_t table_rows;   /* append: rows of cos_table and sin_table, table_width * page_size at least      */
    float scale;          /* attention: as in attn.h                                                        */
    int64_t q_stride_t, q_stride_h;    /* Q                                                                 */
    int64_t out_stride_t, out_stride_h; /* O, Q_rot                                                         */
    int64_t kv_stride_t, kv_stride_h;  /* append: K, V                                                      */
    int64_t cache_stride_p, cache_stride_h, cache_stride_s;
                          /* strides are multiples of 16 bytes, pointers 16-byte aligned; a page's rows of one
                             head lie within 2^30 bytes                                                     */
} attn_paged_params_t;

/* Fills p for contiguous tensors Q [T][Hq][D], K, V [T][Hkv][D] and caches [pages][Hkv][page_size][D]; max_q = T,
 * rot = 0. */
void attn_paged_params_contiguous(attn_paged_params_t *p, int32_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t D,
                                  int32_t pages, int32_t page_size, int32_t table_width, float scale, int32_t causal);

/*
 * Appends the batch's rows of K and V, all bf16 (attn_paged_append_f16: fp16), to the caches, in place.
 *   rot > 0: columns j and j + rot/2 (j < rot/2) of a K row at position p, and of the Q row of the same token, are
 *     rotated by row p of cos_table, sin_table, fp32 [table_rows][rot/2]:
 *         y_j = x_j c_j - x_{j+rot/2} s_j        y_{j+rot/2} = x_{j+rot/2} c_j + x_j s_j
 *     in fp32; the other columns stay.  rot = 0: K is stored as it comes (tables NULL).
 *   Q, Q_rot: may both be NULL; otherwise the rotated (rot = 0: copied) rows are written to Q_rot, which may be Q
 *     (with Q's strides).  Rows at negative positions, or past the page table's, are not written.
 *   16-bit cache: the fp32 values, rounded once.  k_scale, v_scale NULL.
 *   e4m3 cache: of each page and head that gets rows, the scale becomes
 *         s = max(old scale if the page has older keys of the sequence, s_new),
 *         s_new = the least power of two, 2^-100 at least, with max |new values| <= 448 s_new,
 *     the new values are stored as round(x / s), and where s is larger than the old scale the older keys as
 *     round(code * (old scale / s)): by a power of two, which only moves their exponent (codes that fall below 2^-6
 *     are rounded).  A page belongs to one sequence: pages that two sequences of a batch append to are not
 *     supported (read by several they may be).
 * Nothing is read from slots behind the new rows; they keep what they hold.
 */
int attn_paged_append(const void *K, const void *V, const void *Q, void *Q_rot, const float *cos_table,
                      const float *sin_table, void *K_cache, void *V_cache, float *k_scale, float *v_scale,
                      const int32_t *page_table, const int32_t *q_start, const int32_t *kv_lens,
                      const attn_paged_params_t *p, void *hip_stream);
int attn_paged_append_f16(const void *K, const void *V, const void *Q, void *Q_rot, const float *cos_table,
                          const float *sin_table, void *K_cache, void *V_cache, float *k_scale, float *v_scale,
                          const int32_t *page_table, const int32_t *q_start, const int32_t *kv_lens,
                          const attn_paged_params_t *p, void *hip_stream);

/*
 * Attention of the batch's rows over the cache: O (of Q's type) and LSE, fp32 [T][Hq] contiguous, natural
 * logarithm.  A row that sees no key gets O = 0 and LSE = -infinity.
 * (T Hq/Hkv / 128 + B) Hkv (table_width page_size / 32 + 16), what spreading the work counts with, has to be an int32:
 * with 32 query and 8 K/V heads, a prompt of half a million tokens in one call.
 *   workspace: NULL (every row's keys are worked through by one work-group), or 256-byte aligned and of at least
 *     attn_fwd_paged_workspace_bytes: work over many keys is then spread over the whole chip.  Its contents are not
 *     read before they are written.
 */
size_t attn_fwd_paged_workspace_bytes(const attn_paged_params_t *p);
int attn_fwd_paged(const void *Q, const void *K_cache, const void *V_cache, const float *k_scale, const float *v_scale,
                   const int32_t *page_table, const int32_t *q_start, const int32_t *kv_lens, void *O, float *LSE,
                   void *workspace, size_t workspace_bytes, const attn_paged_params_t *p, void *hip_stream);
int attn_fwd_paged_f16(const void *Q, const void *K_cache, const void *V_cache, const float *k_scale,
                       const float *v_scale, const int32_t *page_table, const int32_t *q_start, const int32_t *kv_lens,
                       void *O, float *LSE, void *workspace, size_t workspace_bytes, const attn_paged_params_t *p,
                       void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif
