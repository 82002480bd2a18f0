/*
 * flame_kvq.h - C ABI of the paged key/value cache in 8 or 4 bits: keys and values are quantised as they are written (flame_kvq_append), read back as rows of the
 * element type (flame_kvq_read), and attended over as they lie (flame_kvq_extend, flame_kvq_decode, flame_kvq_shared).
 *
 * Everything that flame_kv.h says holds here too: configurations, rows, page tables, offsets, faults, workspaces, streams, what a row sees, what becomes of a row that sees nothing.
 * A history takes 33/64 (f8) or 17/64 (f4) of the bytes that it has as bf16, and decoding, which reads it once, as much less time.
 *
 * What is stored.  The features of a head go in blocks of 32 that share a scale 2^e; a feature x is a code c with the value c 2^e.
 *     form   codes                                        largest   e is the least with           e at least (fp16 / others)   |value - x| at most
 *     F8     e4m3: a byte, sign, 4 exponent, 3 fraction   448       max |x| 2^-e <= 464           -15 / -117                   max(2^-4 |x|, 2^-10 2^e)
 *     F4     e2m1: half a byte, sign, 2, 1                6         max |x| 2^-e < 7              -23 / -125                   max(2^-2 |x|, 2^-2 2^e)
 * so that no code of a block rounds beyond the largest one, and every value is exact in the element type.  c is x 2^-e rounded to nearest, halves to the even code; a rotated key is
 * rounded this once, from fp32.  |x| beyond 61440 (fp16 f8), 49152 (fp16 f4), 240 2^120 (f8) or 1.5 2^127 (f4), whose value could round to an infinity, is taken as that.  A block that holds an infinity or NaN is NaN as
 * a whole (its scale's byte is 255).  A cache is written and read under one element type (dtype): the limits above go by it.
 *
 * Attention is that of flame_kv.h on a cache that holds these values.
 */
#ifndef FLAME_KVQ_H
#define FLAME_KVQ_H

#include "flame_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { FLAME_KVQ_F8 = 1, FLAME_KVQ_F4 = 2 } flame_kvq_form;

/* As flame_kv_cache, with strides in BYTES of codes, not negative, each a multiple of what a head's row takes (head_dim bytes in F8, head_dim / 2 in F4), pools 16-byte aligned.  Features 2j and 2j + 1
 * are the lower and upper half of byte j in F4.  The scale of the 32 features whose codes begin at byte x of k is byte x / 32 (F8) or x / 16 (F4) of k_scales, e + 127; v alike.
 * Scales are 4-byte aligned. */
typedef struct {
  int32_t form;              /* flame_kvq_form */
  void *k, *v;               /* device pools of n_pages pages */
  void *k_scales, *v_scales; /* device */
  int64_t page_stride, slot_stride, head_stride;
  int32_t n_pages, page_size;
  const int32_t *page_table;
  int64_t table_stride;
  int32_t pages_per_seq;
} flame_kvq_cache;

/* flame_kv_append into such a cache.  The same call gives the same bits.  Of two new tokens in one slot every code and every scale there is one or the other's, and not always of the same one. */
int flame_kvq_append(const flame_kv_config *cfg, const flame_kvq_cache *cache, const flame_kv_rows *k, const flame_kv_rows *v, const flame_kv_rows *q, const flame_kv_rows *q_out,
                     const flame_kv_rotation *rotation, const int32_t *offsets, const int32_t *kv_lens, int32_t n_seqs, int64_t n_tokens, int32_t *faults, void *stream);

/* Keys and values of tokens back from the cache, as values of the element type (exact; keys as they were written, rotated).
 *   k, v         rows [n_tokens][n_kv_heads], written: rows offsets[b]..offsets[b+1] are the tokens of sequence b up to its kv_lens[b]-th, as flame_kvq_append takes them
 * A token at a position below 0 or beyond the table's row, or in no page of the pool, is not written (faults as in flame_kv_append). */
int flame_kvq_read(const flame_kv_config *cfg, const flame_kvq_cache *cache, const int32_t *offsets, const int32_t *kv_lens, int32_t n_seqs, int64_t n_tokens, const flame_kv_rows *k,
                   const flame_kv_rows *v, int32_t *faults, void *stream);

/* flame_kv_extend, flame_kv_decode and flame_kv_shared over such a cache, with the workspaces of those (flame_kv_workspace_bytes, flame_kv_shared_workspace_bytes). */
int flame_kvq_extend(const flame_kv_config *cfg, const flame_kvq_cache *cache, const flame_kv_rows *q, const int32_t *q_offsets, const int32_t *kv_lens, int32_t n_seqs, int64_t n_tokens,
                     const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults, void *stream);
int flame_kvq_decode(const flame_kv_config *cfg, const flame_kvq_cache *cache, const flame_kv_rows *q, const int32_t *kv_lens, int32_t n_seqs, const flame_kv_rows *out, void *workspace,
                     int64_t workspace_bytes, int32_t *faults, void *stream);
int flame_kvq_shared(const flame_kv_config *cfg, const flame_kvq_cache *cache, const flame_kv_rows *q, const int32_t *q_offsets, const int32_t *kv_lens, const flame_kv_groups *groups,
                     int32_t n_seqs, int64_t n_tokens, const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults, void *stream);

/* The message of the last failing flame_kvq_* call on this thread is that of flame_kv_last_error. */

#ifdef __cplusplus
}
#endif
#endif /* FLAME_KVQ_H */
