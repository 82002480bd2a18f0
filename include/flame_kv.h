/*
 * flame_kv.h - C ABI of softmax attention on a paged key/value cache, for histories that grow.
 *
 * flame_gr_prefill and flame_gr_score of flame_gr.h keep the keys and values of a batch of histories in one piece
 * inside a handle, until the next prefill.  The calls here work on a cache that the caller owns and that lives as long as its
 * users do: a pool of pages, and for every sequence a row of a page table that says which pages hold its tokens.
 * A token that arrives costs one row of keys and values (flame_kv_append) and one row of attention against what is there
 * (flame_kv_decode, or flame_kv_extend for several new tokens at once); flame_kv_prompt attends within whole sequences that
 * are in no cache.  They are plain functions, like flame_climber_head: no handle, no allocation, kernels enqueued on the
 * caller's stream and nothing else, so that each may be captured into a HIP graph and replayed while the device arrays
 * (lengths, page table, rows) change between replays.
 *
 * Attention.  Query head h (0..n_q_heads-1) reads key/value head h / (n_q_heads / n_kv_heads).  With n keys and m queries of a
 * sequence, query row i is the token at position n - m + i and sees the keys at positions 0..n-m+i:
 *     O_i = sum over c <= n-m+i of w_c V_c,    w = softmax over those c of scale <Q_i, K_c>.
 * A query row that sees no key (more queries than keys), or whose logits are all -infinity, has an output of zeros, whatever the values.  Keys and values that a
 * row does not see have no influence on it, whatever they hold (infinities and NaN too); a NaN that another row sees makes it NaN,
 * whatever its weight.
 *
 * Rotation.  The first rot_dim features of a key or query at position p are taken in pairs (a, b) - feature j with feature
 * j + rot_dim/2, or neighbours 2j and 2j + 1 - and pair j turns by the angle p * frequencies[j]:
 *     a' = a cos - b sin,   b' = a sin + b cos.
 * The angle is reduced in 64-bit fixed point: to the error of a small angle, position p adds at most p 2^-61 of a revolution (times the revolutions per position,
 * where the frequency is more than one), 2^-30 at position 2^31.
 *
 * Arithmetic.  Products of 16-bit operands are exact and added up in fp32; softmax maxima and sums are fp32; its weights are rounded to the
 * element type for the product with the values (bf16, f16: matrix operands; f32: not rounded; an f16 weight is off by half a step or by 2^-32 of the row's
 * largest); outputs are rounded once.  The sums over the keys are divided by the sum of the weights at the end, and until then a weight may be up to 2^8: of n
 * keys, values beyond 2^120 / n may give infinities (fp32 and bf16; no fp16 value gets there).  An infinite value may give a NaN where its weight is below 2^-126
 * (f16: 2^-32) of the row's largest.
 *
 * Conventions
 *   - Every function returns 0 or a negative flame_gr_status; flame_kv_last_error has the message.  On error
 *     nothing is enqueued.
 *   - "device" pointers are memory of the current HIP device, 16-byte aligned for rows of features.  Strides are in elements and
 *     multiples of 16 bytes; the features of a head lie side by side.
 *   - offsets, lengths and page tables are DEVICE arrays (int32), so that a captured call follows them.  They are read by the
 *     kernels, which check what they address by: an entry out of range makes no access, and is reported in *faults (device int32,
 *     may be NULL), into which the kernels OR the FLAME_KV_FAULT_* bits they meet.  The caller clears it.
 *   - Device buffers stay alive and unmodified until the stream has passed the call.  Outputs must not overlap inputs (q_out may be q).
 *   - Rows ahead of the first sequence and behind the last one (row < offsets[0], offsets[n_seqs] <= row < n_tokens) are neither read nor written: a batch
 *     may be padded.
 */
#ifndef FLAME_KV_H
#define FLAME_KV_H

#include <stdint.h>

#include "flame_gr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of queries, keys, values, cache and outputs (the first two as in flame_gr_dtype). */
typedef enum { FLAME_KV_F32 = 0, FLAME_KV_BF16 = 1, FLAME_KV_F16 = 2 } flame_kv_dtype;

typedef enum {
  FLAME_KV_FAULT_PAGE = 1,   /* a page-table entry outside [0, n_pages): its tokens are not written, its keys not seen */
  FLAME_KV_FAULT_LENGTH = 2, /* a length below 0 or beyond the table's row (taken as the nearest that fits), or an appended token at a position below 0 or
                                beyond it (not written to the cache; below 0 its query is not written either) */
  FLAME_KV_FAULT_OFFSET = 4  /* offsets that decrease, are below 0 or end behind the rows.  Of up to 64 sequences, those before the first offset that decreases or is below 0 have
                                their results, as far as there are rows, and no other row is written.  Of more, which rows of the batch are written is not defined. */
} flame_kv_fault;

typedef struct {
  int32_t dtype;      /* flame_kv_dtype */
  int32_t n_q_heads;  /* a multiple of n_kv_heads */
  int32_t n_kv_heads; /* >= 1 */
  int32_t head_dim;   /* 32, 64 or 128 (else UNSUPPORTED) */
  float scale;        /* of the logits, >= 0; 0 selects 1 / sqrt(head_dim) */
} flame_kv_config;

/* Rows of heads: element (row, head, feature) at data + row * row_stride + head * head_stride + feature. */
typedef struct {
  void *data;          /* device; not written where the call says input */
  int64_t row_stride;
  int64_t head_stride;
} flame_kv_rows;

/* Token t of sequence b lies in page page_table[b * table_stride + t / page_size], slot t % page_size. */
typedef struct {
  void *k, *v;               /* device pools of n_pages pages; both with the strides below */
  int64_t page_stride, slot_stride, head_stride;
  int32_t n_pages, page_size; /* page_size: any, 1..65536 */
  const int32_t *page_table; /* device [n_seqs][table_stride], the first pages_per_seq entries of a row in use */
  int64_t table_stride;
  int32_t pages_per_seq;     /* pages_per_seq * page_size: up to 2^31 - 65536 */
} flame_kv_cache;

typedef struct {
  int32_t rot_dim;            /* features that turn: a multiple of 16 up to head_dim */
  int32_t interleaved;        /* 0: pairs (j, j + rot_dim/2); 1: pairs (2j, 2j + 1) */
  const double *frequencies;  /* HOST [rot_dim/2], radians per position; read during the call */
} flame_kv_rotation;

/* Keys and values of new tokens into the cache; keys, and queries if given, rotated on the way.
 *   k, v         rows [n_tokens][n_kv_heads], packed: rows offsets[b]..offsets[b+1] are the newest of sequence b
 *   q, q_out     rows [n_tokens][n_q_heads], both or neither NULL: q_out = rotated q (may be q)
 *   rotation     NULL: none
 *   offsets      device [n_seqs+1]
 *   kv_lens      device [n_seqs]: tokens of each sequence WITH the new ones; row j of its m new rows has position kv_lens[b] - m + j
 * Every value written is the rounding of one expression: the same call gives the same bits.  Of two new tokens in one slot (a page
 * that two sequences share) every value there is one or the other's. */
int flame_kv_append(const flame_kv_config *cfg, const flame_kv_cache *cache, const flame_kv_rows *k, const flame_kv_rows *v, const flame_kv_rows *q,
                    const flame_kv_rows *q_out, const flame_kv_rotation *rotation, const int32_t *offsets, const int32_t *kv_lens, int32_t n_seqs,
                    int64_t n_tokens, int32_t *faults, void *stream);

/* Causal attention within packed sequences that are in no cache.
 *   q, out       rows [n_tokens][n_q_heads], sequence b at q_offsets[b]..q_offsets[b+1]
 *   k, v         rows [n_keys][n_kv_heads], sequence b at k_offsets[b]..k_offsets[b+1]
 *   k_offsets    device [n_seqs+1], or NULL: q_offsets */
int flame_kv_prompt(const flame_kv_config *cfg, const flame_kv_rows *q, const flame_kv_rows *k, const flame_kv_rows *v, const int32_t *q_offsets,
                    const int32_t *k_offsets, int32_t n_seqs, int64_t n_tokens, int64_t n_keys, const flame_kv_rows *out, int32_t *faults, void *stream);

/* Causal attention of the newest tokens of every sequence over its cache (which holds them already: flame_kv_append first).
 *   q, out       rows [n_tokens][n_q_heads], sequence b at q_offsets[b]..q_offsets[b+1]
 *   kv_lens      device [n_seqs]: tokens in the cache
 *   workspace    device, 16-byte aligned, of flame_kv_workspace_bytes bytes for these sequences and rows or for more.  It holds nothing between
 *                calls; two calls that overlap in time need one each. */
int flame_kv_extend(const flame_kv_config *cfg, const flame_kv_cache *cache, const flame_kv_rows *q, const int32_t *q_offsets, const int32_t *kv_lens,
                    int32_t n_seqs, int64_t n_tokens, const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults, void *stream);

/* Attention of one new token of every sequence over its cache: row b of q and out [n_seqs][n_q_heads] belongs to sequence b.
 * A sequence of length 0 has an output of zeros.  Workspace: as of n_seqs rows. */
int flame_kv_decode(const flame_kv_config *cfg, const flame_kv_cache *cache, const flame_kv_rows *q, const int32_t *kv_lens, int32_t n_seqs,
                    const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults, void *stream);

/* Groups of sequences that begin with the same tokens: sequences group_offsets[g]..group_offsets[g+1] share the first tokens of the first of them. */
typedef struct {
  const int32_t *group_offsets; /* device [n_groups+1], from 0 to n_seqs */
  const int32_t *prefix_lens;   /* device [n_seqs]: so many first tokens of a sequence are those of its group's first sequence, whose own entry is the largest of the group */
  int32_t n_groups;
} flame_kv_groups;

/* Attention of the newest tokens of every sequence over its cache, as flame_kv_extend (q_offsets NULL: one new token each, row b of sequence b, as flame_kv_decode), for sequences that
 * share long beginnings: what a group shares is read once for all rows of the group, where the table row of its first sequence says (which names the group's prefix_lens tokens, whatever
 * that sequence's own length).  Keys from prefix_lens[b] on are sequence b's own, where its own row of the table says; entries of that row for pages of shared tokens alone are not read.
 * kv_lens count both.  A shared history may end within a page, a sequence within the shared history (its rows see their own positions, as ever), and a sequence may leave the history
 * earlier than others do (its prefix_lens is less).  The outputs are those of flame_kv_extend on tables that say the same; sums are cut differently, so the last bits may differ.
 *   faults       FLAME_KV_FAULT_LENGTH also for a prefix_lens below 0, beyond the table's row, or beyond that of the group's first sequence (tokens from there on are not seen);
 *                FLAME_KV_FAULT_OFFSET also for group_offsets that decrease, are below 0, or do not go from 0 to n_seqs: a sequence that is in no group, or of up to 64 groups in one
 *                behind offsets that are none, sees its own tokens alone.  (Of more groups, which rows see what is not defined.)
 *   workspace    of flame_kv_shared_workspace_bytes bytes for these numbers or larger ones; as in flame_kv_extend
 * n_tokens is below 2^24.
 * Made for few new rows of many sequences.  A sequence's own keys are read again for every 16 of its rows (new tokens times the query heads of a key head): long pieces behind a history are faster by flame_kv_extend on
 * tables that name its pages for each (16 x 400 new behind 4 histories of 2000..8000, 32/8 heads of 128, f8: 1085 us here, 892 there).  And in a call of more than some 400 row tiles ((n_tokens G / 128 + n_groups) key heads,
 * G query heads to a key head) a history is not cut along its keys, so that one much longer than the others takes its time alone. */
int flame_kv_shared(const flame_kv_config *cfg, const flame_kv_cache *cache, const flame_kv_rows *q, const int32_t *q_offsets, const int32_t *kv_lens, const flame_kv_groups *groups,
                    int32_t n_seqs, int64_t n_tokens, const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults, void *stream);

/* HOST arithmetic: a workspace for every flame_kv_shared (and flame_kvq_shared) of this configuration with up to so many groups, sequences and query rows. */
int flame_kv_shared_workspace_bytes(const flame_kv_config *cfg, int32_t n_groups, int32_t n_seqs, int64_t n_tokens, int64_t *bytes);

/* HOST arithmetic: a workspace for every flame_kv_extend and flame_kv_decode of this configuration with up to so many sequences and query rows:
 * a program asks once, for its largest batch. */
int flame_kv_workspace_bytes(const flame_kv_config *cfg, int32_t n_seqs, int64_t n_tokens, int64_t *bytes);

/* HOST arithmetic: the geometric frequencies base^(-2j / rot_dim), j = 0..rot_dim/2-1, into out [rot_dim/2]. */
int flame_kv_rotation_frequencies(int32_t rot_dim, double base, double *out);

/* Message of the last failing flame_kv_* call on this thread ("" if none). */
const char *flame_kv_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FLAME_KV_H */
