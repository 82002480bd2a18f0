// C entries of the operators on a paged key/value cache (include/flame_kv.h): checks of arguments, byte strides, launches.
#include <algorithm>
#include <cmath>

#include "kv.h"

using namespace flame;

namespace {

thread_local const char *g_kv_error = "";

int bad(const char *message, int code = FLAME_GR_INVALID_ARGUMENT) {
  g_kv_error = message;
  return code;
}

int done(hipError_t e) {
  if (e == hipSuccess) return FLAME_GR_OK;
  return bad(hipGetErrorString(e), FLAME_GR_HIP_ERROR);
}

// A grid dimension may have 2^32 - 1 threads.  Attention on row tiles has two of them per row and head, and 256 per sequence and head; the join of split attention has up to 2^22,
// and 256 per 64 rows and heads where those are more than 2^20.
// The join of shared histories has 256 for a row and up to 8, 16 or 32 heads.
constexpr int64_t kMaxRowHeads = (int64_t)1 << 25, kMaxSequenceHeads = ((int64_t)1 << 23) - 1, kMaxSharedRows = (int64_t)1 << 24;
constexpr int64_t kSmallCache = 1024;                          // tokens that a sequence has room for, up to which its keys are not split over the chip
constexpr int64_t kMaxKeys = ((int64_t)1 << 31) - 65536;     // of a sequence: room for a tile's end behind them in 32 bits
// Limits of kv_route, for the workspace of every call up to a size: rows times heads of an extend that is split, parts of a row tile's keys, and workgroups of a launch whose keys are cut.
constexpr int64_t kFlashRows = 128, kSharedPlaces = 512;         // rows of a tile (kv_flash.h); workgroups over shared histories
constexpr int64_t kSplitRowHeads = 16384, kMostParts = 64, kPartWorkgroups = 400;

int64_t element(int32_t dtype) { return dtype == FLAME_KV_F32 ? 4 : 2; }
bool aligned(const void *p) { return ((uintptr_t)p & 15) == 0; }

int check_config(const flame_kv_config *c) {
  if (!c) return bad("the configuration is NULL");
  if (c->dtype < FLAME_KV_F32 || c->dtype > FLAME_KV_F16) return bad("dtype must be a flame_kv_dtype");
  if (c->n_kv_heads < 1 || c->n_q_heads < 1 || c->n_q_heads % c->n_kv_heads) return bad("n_q_heads must be a positive multiple of n_kv_heads");
  if (c->n_q_heads > 4096) return bad("more than 4096 heads", FLAME_GR_UNSUPPORTED);
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return bad("head_dim must be 32, 64 or 128", FLAME_GR_UNSUPPORTED);
  if (!(c->scale >= 0.f) || !std::isfinite(c->scale)) return bad("scale must be finite and not negative");
  return FLAME_GR_OK;
}

int check_batch(const flame_kv_config *c, int32_t n_seqs, int64_t n_rows) {
  if (n_seqs < 0 || (int64_t)n_seqs * c->n_q_heads > kMaxSequenceHeads) return bad("sequences times heads must be in [0, 2^23)");
  if (n_rows < 0 || n_rows > kMaxRowHeads / c->n_q_heads) return bad("rows times heads must be in [0, 2^25]");
  return FLAME_GR_OK;
}

int take_rows(const flame_kv_config *c, const flame_kv_rows *r, KvRows *out) {
  if (!r || !r->data) return bad("rows are NULL");
  const int64_t size = element(c->dtype);
  if (!aligned(r->data) || (r->row_stride * size) % 16 || (r->head_stride * size) % 16) return bad("rows must be 16-byte aligned, with strides of multiples of 16 bytes");
  *out = KvRows{(char *)r->data, r->row_stride * size, r->head_stride * size};
  return FLAME_GR_OK;
}

int take_pages(const flame_kv_config *c, const flame_kv_cache *cache, KvPages *out) {
  if (!cache) return bad("the cache is NULL");
  if (!cache->k || !cache->v || !cache->page_table) return bad("a pointer of the cache is NULL");
  if (cache->n_pages < 1 || cache->page_size < 1 || cache->page_size > 65536) return bad("n_pages must be positive and page_size in [1, 65536]");
  if (cache->pages_per_seq < 1 || (int64_t)cache->pages_per_seq * cache->page_size > kMaxKeys) return bad("pages_per_seq must be positive, and a sequence within 2^31 - 65536 tokens");
  const int64_t size = element(c->dtype);
  if (!aligned(cache->k) || !aligned(cache->v) || (cache->page_stride * size) % 16 || (cache->slot_stride * size) % 16 || (cache->head_stride * size) % 16)
    return bad("the cache must be 16-byte aligned, with strides of multiples of 16 bytes");
  *out = KvPages{(char *)cache->k, (char *)cache->v, cache->page_stride * size, cache->slot_stride * size, cache->head_stride * size, cache->n_pages, 0, 0, 0,
                 cache->page_table, cache->table_stride, cache->pages_per_seq * cache->page_size};
  kv_set_page_size(out, cache->page_size);
  return FLAME_GR_OK;
}

// of a quantised cache: strides are bytes of codes
int take_pages(const flame_kv_config *c, const flame_kvq_cache *cache, KvPages *out, KvScales *scales) {
  if (!cache) return bad("the cache is NULL");
  if (cache->form != FLAME_KVQ_F8 && cache->form != FLAME_KVQ_F4) return bad("form must be a flame_kvq_form");
  if (!cache->k || !cache->v || !cache->k_scales || !cache->v_scales || !cache->page_table) return bad("a pointer of the cache is NULL");
  if (cache->n_pages < 1 || cache->page_size < 1 || cache->page_size > 65536) return bad("n_pages must be positive and page_size in [1, 65536]");
  if (cache->pages_per_seq < 1 || (int64_t)cache->pages_per_seq * cache->page_size > kMaxKeys) return bad("pages_per_seq must be positive, and a sequence within 2^31 - 65536 tokens");
  const int64_t row = cache->form == FLAME_KVQ_F8 ? c->head_dim : c->head_dim / 2;
  if (!aligned(cache->k) || !aligned(cache->v) || ((uintptr_t)cache->k_scales & 3) || ((uintptr_t)cache->v_scales & 3)) return bad("pools must be 16-byte and scales 4-byte aligned");
  if (cache->page_stride % row || cache->slot_stride % row || cache->head_stride % row) return bad("the strides of a quantised cache must be multiples of a head's bytes");
  if (cache->page_stride < 0 || cache->slot_stride < 0 || cache->head_stride < 0) return bad("the strides of a quantised cache must not be negative");
  *out = KvPages{(char *)cache->k, (char *)cache->v, cache->page_stride, cache->slot_stride, cache->head_stride, cache->n_pages, 0, 0, 0,
                 cache->page_table, cache->table_stride, cache->pages_per_seq * cache->page_size};
  kv_set_page_size(out, cache->page_size);
  *scales = KvScales{(char *)cache->k_scales, (char *)cache->v_scales, cache->form};
  return FLAME_GR_OK;
}

int take_rotation(const flame_kv_config *c, const flame_kv_rotation *r, KvRotation *out) {
  *out = KvRotation{};
  if (!r) return FLAME_GR_OK;
  if (r->rot_dim < 16 || r->rot_dim % 16 || r->rot_dim > c->head_dim) return bad("rot_dim must be a multiple of 16 up to head_dim");
  if (!r->frequencies) return bad("the frequencies are NULL");
  out->pairs = r->rot_dim / 2;
  out->interleaved = r->interleaved != 0;
  for (int j = 0; j < out->pairs; ++j) {
    if (!std::isfinite(r->frequencies[j])) return bad("a frequency is not finite");
    // revolutions per position, of which only the fraction turns anything
    const long double turns = (long double)r->frequencies[j] * (1.0L / 6.283185307179586476925286766559005768L);
    const long double fraction = turns >= 0.0L && turns < 1.0L ? turns : turns - floorl(turns);
    out->turns[j] = fraction < 1.0L ? (uint64_t)(fraction * 0x1p64L) : 0;
  }
  return FLAME_GR_OK;
}

void take_heads(const flame_kv_config *c, KvAttention *a) {
  a->n_q_heads = c->n_q_heads;
  a->n_kv_heads = c->n_kv_heads;
  a->head_dim = c->head_dim;
  a->dtype = c->dtype;
  a->scale = c->scale == 0.f ? 1.f / std::sqrt((float)c->head_dim) : c->scale;
}

// What a call of this size needs over any cache: one of little room may go by another route than a large one.
int64_t workspace_bytes_for(const flame_kv_config &c, int32_t n_seqs, int64_t n_rows, bool decode) {
  return std::max(kv_route(c, n_seqs, n_rows, true, decode, kMaxKeys).workspace, kv_route(c, n_seqs, n_rows, true, decode, kSmallCache).workspace);
}

// What any call of up to this many sequences and rows may need, over any cache: a bound that only grows with either.  Decoding splits the rows of one per sequence, an extend up to
// kSplitRowHeads.  In parts, kv_route cuts keys into up to kMostParts, and into at most 1024 / likely: with s sequences of r rows (of a key head) and kp wavefronts to 32 of them, likely is
// s ceil(r kp / 128) key heads, and there are fewer than s (r + 1) key heads rows times heads; r + 1 <= 129 ceil(r kp / 128), so that parts times rows times heads stay below 1024 * 129.
// (Without rows to a whole sequence, r = 0, they stay below kMostParts kPartWorkgroups, which is less.)
int64_t workspace_bound(const flame_kv_config &c, int32_t n_seqs, int64_t n_rows) {
  if (n_seqs == 0 || n_rows == 0) return 0;
  const int64_t heads = n_rows * c.n_q_heads;
  static_assert(kMostParts * kPartWorkgroups <= 1024 * 129, "what a sequence of less than a row may need");
  const int64_t split = kv_split_workspace_bytes(c.head_dim, std::max(std::min((int64_t)n_seqs, n_rows) * c.n_q_heads, std::min(heads, kSplitRowHeads)));
  const int64_t parts = std::min(kMostParts * heads, (int64_t)1024 * 129) * (c.head_dim + 2) * 4;
  return std::max(split, parts);
}

int attend_cache(const flame_kv_config *cfg, const flame_kv_cache *cache, const flame_kv_rows *q, const int32_t *offsets, const int32_t *kv_lens, int32_t n_seqs, int64_t n_rows,
                 const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults, void *stream) {
  KvAttention a{};
  if (int rc = take_rows(cfg, q, &a.q)) return rc;
  if (int rc = take_rows(cfg, out, &a.out)) return rc;
  if (int rc = take_pages(cfg, cache, &a.pages)) return rc;
  if (!kv_lens) return bad("kv_lens is NULL");
  const KvRoute route = kv_route(*cfg, n_seqs, n_rows, true, offsets == nullptr, a.pages.capacity);
  const int64_t need = workspace_bytes_for(*cfg, n_seqs, n_rows, offsets == nullptr);
  if (need > 0 && (!workspace || !aligned(workspace))) return bad("the workspace is NULL or not 16-byte aligned");
  if (workspace_bytes < need) return bad("the workspace is smaller than this call needs (flame_kv_workspace_bytes)", FLAME_GR_CAPACITY_EXCEEDED);
  a.batch = KvBatch{offsets, kv_lens, n_seqs, n_rows, faults};
  take_heads(cfg, &a);
  if (route.split) return done(launch_kv_split(a, workspace, (hipStream_t)stream));
  a.splits = route.splits;
  a.parts = (float *)workspace;
  return done(launch_kv_attention(a, route.wavefronts, (hipStream_t)stream));
}

// The same over a quantised cache, and with shared histories (groups; the cache is then either).
int attend_quantised(const flame_kv_config *cfg, const flame_kvq_cache *cache, const flame_kv_rows *q, const int32_t *offsets, const int32_t *kv_lens, int32_t n_seqs, int64_t n_rows,
                     const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults, void *stream) {
  KvAttention a{};
  KvScales scales;
  if (int rc = take_rows(cfg, q, &a.q)) return rc;
  if (int rc = take_rows(cfg, out, &a.out)) return rc;
  if (int rc = take_pages(cfg, cache, &a.pages, &scales)) return rc;
  if (!kv_lens) return bad("kv_lens is NULL");
  const bool decode = offsets == nullptr;
  const KvRoute route = kvq_route(*cfg, n_seqs, n_rows, decode, a.pages.capacity);
  const int64_t need = std::max(kvq_route(*cfg, n_seqs, n_rows, decode, kMaxKeys).workspace, kvq_route(*cfg, n_seqs, n_rows, decode, kSmallCache).workspace);
  if (need > 0 && (!workspace || !aligned(workspace))) return bad("the workspace is NULL or not 16-byte aligned");
  if (workspace_bytes < need) return bad("the workspace is smaller than this call needs (flame_kv_workspace_bytes)", FLAME_GR_CAPACITY_EXCEEDED);
  a.batch = KvBatch{offsets, kv_lens, n_seqs, n_rows, faults};
  take_heads(cfg, &a);
  a.form = scales.form;
  a.k_scales = scales.k;
  a.v_scales = scales.v;
  if (route.split) return done(launch_kvq_split(a, workspace, (hipStream_t)stream));
  a.splits = route.splits;
  a.parts = (float *)workspace;
  return done((a.form == FLAME_KVQ_F8 ? launch_kvq_attention_f8 : launch_kvq_attention_f4)(a, route.wavefronts, (hipStream_t)stream));
}

// What any flame_kv_shared of up to this many groups, sequences and rows may need.  Parts of equal length: row tiles are up to rows times heads over a tile's rows and a tile for each group and key head, or
// kSharedPlaces of them, of up to 128 rows, and such a call has up to kPartWorkgroups tiles of 128 rows (and wavefronts, up to four, times as many smaller ones).  Others: as in workspace_bound, groups for sequences.
int64_t shared_workspace_bound(const flame_kv_config &c, int32_t n_seqs, int64_t n_rows) {
  if (n_seqs == 0 || n_rows == 0) return 0;
  const int64_t heads = n_rows * c.n_q_heads;
  const int64_t parts = std::max({heads, std::min(kMostParts * heads, (int64_t)1024 * 129), std::max(kSharedPlaces, 4 * kPartWorkgroups) * kFlashRows});
  return (heads + parts) * (c.head_dim + 2) * 4 + 64 * 8 + 48 + kv_split_workspace_bytes(c.head_dim, heads);
}

int check_groups(const flame_kv_config *c, int32_t n_groups, int32_t n_seqs, int64_t n_rows) {
  if (int rc = check_batch(c, n_seqs, n_rows)) return rc;
  if (n_groups < 0 || (int64_t)n_groups * c->n_q_heads > kMaxSequenceHeads) return bad("groups times heads must be in [0, 2^23)");
  if (n_rows >= kMaxSharedRows) return bad("rows of a call with shared histories must be below 2^24");
  return FLAME_GR_OK;
}

int attend_shared(const flame_kv_config *cfg, const flame_kv_cache *cache, const flame_kvq_cache *quantised, bool plain, const flame_kv_rows *q, const int32_t *offsets,
                  const int32_t *kv_lens, const flame_kv_groups *groups, int32_t n_seqs, int64_t n_rows, const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults,
                  void *stream) {
  g_kv_error = "";
  if (int rc = check_config(cfg)) return rc;
  if (!groups) return bad("the groups are NULL");
  if (int rc = check_groups(cfg, groups->n_groups, n_seqs, n_rows)) return rc;
  if (!offsets && n_rows != n_seqs) return bad("without q_offsets there is a row per sequence");
  if (n_seqs == 0 || n_rows == 0) return FLAME_GR_OK;
  KvAttention a{};
  KvScales scales{};
  if (int rc = take_rows(cfg, q, &a.q)) return rc;
  if (int rc = take_rows(cfg, out, &a.out)) return rc;
  if (int rc = plain ? take_pages(cfg, cache, &a.pages) : take_pages(cfg, quantised, &a.pages, &scales)) return rc;
  if (!kv_lens || !groups->prefix_lens || !groups->group_offsets) return bad("kv_lens, group_offsets or prefix_lens is NULL");
  const KvSharedRoute route = kv_shared_route(*cfg, groups->n_groups, n_rows, a.pages.capacity);
  const int64_t need = std::max(kv_shared_route(*cfg, groups->n_groups, n_rows, kMaxKeys).workspace, kv_shared_route(*cfg, groups->n_groups, n_rows, 1).workspace);
  if (need > 0 && (!workspace || !aligned(workspace))) return bad("the workspace is NULL or not 16-byte aligned");
  if (workspace_bytes < need) return bad("the workspace is smaller than this call needs (flame_kv_shared_workspace_bytes)", FLAME_GR_CAPACITY_EXCEEDED);
  a.batch = KvBatch{offsets, kv_lens, n_seqs, n_rows, faults};
  take_heads(cfg, &a);
  a.form = scales.form;
  a.k_scales = scales.k;
  a.v_scales = scales.v;
  a.group_offsets = groups->group_offsets;
  a.prefix_lens = groups->prefix_lens;
  a.n_groups = groups->n_groups;
  a.splits = route.splits;
  a.budget = route.budget;
  a.parts = (float *)workspace;
  a.part_rows = route.part_rows;
  a.cuts = (int2 *)((char *)workspace + route.cuts_at);
  a.own = (float *)((char *)workspace + route.own_at);
  const auto launch = plain ? launch_kv_shared_plain : a.form == FLAME_KVQ_F8 ? launch_kv_shared_f8 : launch_kv_shared_f4;
  return done(launch(a, route, (char *)workspace + route.split_at, (hipStream_t)stream));
}

}  // namespace

namespace flame {

// Decoding steps, and calls with few query rows over caches that may be long, split the keys over the chip; others run on row tiles, of which a launch of few has its keys cut
// into parts.  The host knows rows and sequences, but of the keys only what the page table has room for.
static KvRoute route_of(const flame_kv_config &c, int32_t n_seqs, int64_t n_rows, bool paged, bool decode, int64_t capacity, bool codes) {
  const bool f32 = c.dtype == FLAME_KV_F32;
  const int64_t group = c.n_q_heads / c.n_kv_heads, heads = n_rows * c.n_q_heads, rows = n_rows * group / std::max(n_seqs, 1);   // rows: of a sequence and key head
  // The split kernel reads the keys again for every 16 rows of a sequence and key head; up to there it reads them once, whatever the sequences' lengths, and carries no masked rows.
  // us split | row tiles, in parts where there are few, by rows of a sequence and key head and by rows times heads; 16-bit:
  //   up to 16 rows: 1024 (64 sequences x 2 new, 8/2 heads of 64, over 2048) 25 | 29, 2048 (16 x 4, 32/8 of 128, over 2048) 40 | 48, (over 8192) 128 | 126, 4096 (64 x 2, 32/8, over 2048) 128 | 108;
  //     of more than 64 sequences, which the row tiles do not sort by length: 6400 (200 x 4, 8/2 of 64, over 100..8192) 118 | 230, (over 2048) 62 | 54
  //   up to 32: 64 (8 new, 8/2 of 64, over 32768) 23 | 35, 256 (8 new, 32/8, over 4096) 25 | 20, (over 16384) 34 | 34, 384 (24 new, 16/16 of 128, over 16384) 45 | 50,
  //     1024 (4 x 8, 32/8, over 4096) 33 | 27, (over 16384) 81 | 70;  more: 384 (12 new, 32/8, over 16384) 51 | 36, 4096 (128 new, 32/8, over 4096) 71 | 36, (over 16384) 209 | 63
  // The lines between lose where it says so (8 new over 4096, by a fifth): the host knows what room there is, not how long the sequences are, and takes the side that loses less.
  // fp32: up to 32 rows: 2048 (16 x 4, 32/8, over 2048) 64 | 113, 16384 (64 x 8, 32/8, over 2048) 301 | 399; more: 512 (16 new, 32/8, over 4096) 36 | 55, 1024 (32 new, 32/8, over 4096) 49 | 91,
  //   (over 16384) 129 | 112, 2048 (64 new, 32/8, over 4096) 75 | 92, (over 16384) 235 | 168, 4096 (4 x 32, 32/8, over 4096) 137 | 100
  // Room for 512 tokens, bf16: 1024 (4 x 8, 32/8) 21 | 13
  // Codes are half or a quarter of the bytes, for split attention more than for row tiles; us split | row tiles, f8 (f4), 16-bit rows:
  //   up to 16 rows: 4096 (64 sequences x 2 new, 32/8 heads of 128, over 2048) 71 | 96 (51 | 88), 16384 (128 x 4) 148 | 176 (108 | 163), (256 x 2, over 1500) 174 | 303 (120 | 278),
  //     12800 (400 x 4, 8/2 of 64, over 1100) 68 | 73 (59 | 60)
  //   up to 32: 1024 (4 x 8, 32/8, over 4096) 26 | 26 (24 | 26), (over 16384) 54 | 70 (44 | 59), 8192 (32 x 8, over 2048) 69 | 76 (55 | 66), 2048 (32 x 8, 8/2 of 64, over 8192) 38 | 39 (34 | 32);
  //   more: 384 (12 new, 32/8, over 16384) 37 | 34 (31 | 33), 4096 (128 new) 48 | 32
  // At the limit, 16384 (64 x 8, 32/8, over 2000), 126 | 98 (94 | 89): it stands there for batches of unequal sequences, whose average says little and which row tiles, one long piece on few workgroups, serve worse still:
  //   63 single tokens over 2000 beside 400 new over 16384, 32/8 of 128, 439 | 511 (330 | 501), 8/2 of 64 68 | 74 (70 | 70); 400 new over 16384 beside 63 empty sequences 367 | 447 (298 | 443).
  const int64_t few = f32 ? (rows <= 32 ? kSplitRowHeads : 1024) : rows > 32 ? 0 : codes ? kSplitRowHeads : rows > 16 ? 512 : n_seqs > 64 ? 8192 : 2048;
  if (decode || (paged && capacity > kSmallCache && heads <= few)) return KvRoute{true, 1, 1, kv_split_workspace_bytes(c.head_dim, heads)};
  // Four or two wavefronts share 32 rows where that many workgroups of one wavefront per 32 rows leave places of the chip empty, or all are placed at
  // once and wait for the longest.  us with one | two | four, at that many workgroups
  // (prompts x tokens); 16-bit, 64 features: 72 (1 x 1024, 8 heads) 22 | 16 | 12, 160 (4 x 512) 14 | 11 | 10, 264 (1 x 4096) 74 | 48 | 49, 288 (4 x 1024) 23 | 18 | 23,
  //   384 (16 x 256) 11 | 12 | 17, 528 (2 x 4096) 75 | 66, 544 (4 x 2048) 41 | 45, 1152 (16 x 1024) 45 | 61 | 86
  //   128 features, 32/8 heads: 72 (1 x 256) 12 | 11 | 10, 264 (1 x 1024) 30 | 26 | 45, 520 (1 x 2048) 57 | 62 | 128;  32 features, 16 heads: 272 (1 x 2048) 32 | 20 | 22, 576 (4 x 1024) 20 | 21 | 32
  // fp32, 64 features: 136 (1 x 2048) 148 | 87 | 57, 160 (4 x 512) 42 | 27 | 30, 264 (1 x 4096) 290 | 171 | 200, 288 (4 x 1024) 79 | 52 | 70, 384 (16 x 256) 26 | 23 | 43,
  //   560 (32 x 257..640, 4 heads) 76 | 76, 596 (16 x 300..2048) 190 | 143, 1280 (32 x 512) 129 | 150
  //   128 features: 264 (1 x 1024) 145 | 95, 520 (1 x 2048) 287 | 327;  32 features: 144 (1 x 1024) 46 | 27 | 20, 320 (4 x 512) 27 | 20 | 27, 576 (4 x 1024) 53 | 60
  const int64_t four = f32 ? 150 : 160, two = f32 ? (c.head_dim == 64 ? 640 : 512) : c.head_dim == 32 ? 576 : 384;
  const bool wide = f32 && c.head_dim == 128;
  const auto workgroups = [&](int64_t kp) { return (n_rows * group * kp / 128 + n_seqs) * c.n_kv_heads; };
  KvRoute r{false, workgroups(1) <= four && !wide ? 4 : workgroups(1) <= two ? 2 : 1, 1, 0};
  // Where there is room for 1024 tokens: parts of at least 256, more than 32 of at least 512, as many as make one round of the chip's 512 places or two of them full, by the number of workgroups that sequences of equal rows would have.
  // us whole | in parts and joined (bf16, 32/8 heads of 128): 1 x 128 new over 4096 53 | 36, over 16384 217 | 63; 4 x 128 over 16384 531 | 204; 16 x 32 over 16384 469 | 275;
  // 8/2 heads of 64: 4 x 512 over 4096 50 | 50.  (25 parts in place of 16, one and a half rounds, cost 1 x 128 over 16384 26 us more.
  // Parts of 512 | 256: fp32, 32/8 heads of 128, 3 x 163 over 1277 185 | 142, 6/2 of 128 101 | 54, bf16 44 | 39; 64 parts of 256 | 32 of 512: 1 x 16 over 16384 44 | 36.
  // With room for 700 and 16 x 40 new, 8/2 of 64, whole | in parts: 13 | 19.)
  // Up to 400 workgroups: whole | in two or three parts, by workgroups(1); bf16, 32/8 heads of 128: 200 (1 x 768 over 4096) 94 | 88,
  // (over 16384) 356 | 274, 264 (1 x 1024 over 16384) 372 | 305, 352 (4 x 320 over 4096) 180 | 124, (over 16384) 769 | 438, 376 (1 x 1500 over 16384) 673 | 484, 384 (8 x 160 over 16384) 880 | 450,
  // 392 (4 x 360 over 4096) 137 | 153, (over 16384) 590 | 606, 448 (8 x 192 over 4096) 141 | 151, (over 16384) 606 | 605; 8/2 heads of 64: 188 (1 x 3000 over 4096) 49 | 56, 258 (1 x 4096 over 16384) 194 | 182,
  // 322 (1 x 5120 over 16384) 313 | 230, 382 (4 x 1500 over 16384) 372 | 273.  fp32: 200 (1 x 768 over 4096, 32/8 of 128) 576 | 481, 392 (4 x 360) 920 | 929, 448 (8 x 192) 1053 | 841 (not taken);
  // 8/2 of 64 over 16384: 322 (1 x 5120) 1536 | 1220, 382 (4 x 1500) 1779 | 1621.
  if (paged && workgroups(1) <= kPartWorkgroups && capacity >= kSmallCache) {
    const int32_t kp = rows <= 32 && !wide ? 4 : rows <= 64 ? 2 : 1;
    const int64_t likely = n_seqs * ((rows * kp + 127) / 128) * c.n_kv_heads;
    const int64_t parts = std::min({(likely > 256 ? 1024 : 512) / std::max(likely, (int64_t)1), std::min(capacity / 256, std::max((int64_t)32, capacity / 512)), kMostParts});
    if (parts > 1) r = KvRoute{false, kp, (int32_t)parts, parts * heads * (c.head_dim + 2) * 4};
  }
  return r;
}

KvRoute kv_route(const flame_kv_config &c, int32_t n_seqs, int64_t n_rows, bool paged, bool decode, int64_t capacity) { return route_of(c, n_seqs, n_rows, paged, decode, capacity, false); }
KvRoute kvq_route(const flame_kv_config &c, int32_t n_seqs, int64_t n_rows, bool decode, int64_t capacity) { return route_of(c, n_seqs, n_rows, true, decode, capacity, true); }

// The histories' rows are those of whole groups.
KvSharedRoute kv_shared_route(const flame_kv_config &c, int32_t n_groups, int64_t n_rows, int64_t capacity) {
  const int64_t group = c.n_q_heads / c.n_kv_heads, heads = n_rows * c.n_q_heads, rows = n_rows * group / std::max(n_groups, 1);
  KvSharedRoute r{};
  // Wavefronts that share 32 rows.  Four of 128 features fill a compute unit's LDS with one workgroup: us with four | two, bf16 (f8), 32/8 heads: 8 sequences over 16384 shared tokens 39 | 31 (35 | 29), 4 groups of
  // 4 over 4000-8000 47 | 46 (39 | 36).  Two | one for 64 rows: 16 over 16384 34 | 35 (31 | 33), 8 groups of 12 over 2000-12000 112 | 118
  r.wavefronts = rows <= 32 && c.head_dim < 128 ? 4 : rows <= 64 ? 2 : 1;
  r.splits = 1;
  const int64_t tile = kFlashRows / r.wavefronts;
  r.slots = n_rows * group / tile + n_groups;
  r.part_rows = n_groups > 0 ? heads : 0;
  // (Beyond kPartWorkgroups histories are not cut, whatever their lengths: one much longer than the others is then walked by one workgroup a row tile and key head.  One of 100000 tokens among others of 1000, a single
  // token each, 32/8 heads of 128, bf16: 48 groups 208 us, 56 or 64 groups 2760.)
  if (n_groups > 0 && (n_rows * group / 128 + n_groups) * c.n_kv_heads <= kPartWorkgroups && capacity >= kSmallCache) {
    if (n_groups <= 64) {
      // parts of equal length, for the chip's places
      r.splits = 0;
      r.budget = (int32_t)std::max((int64_t)1, kSharedPlaces / c.n_kv_heads);
      r.slots = std::max(r.slots, (int64_t)r.budget);
      r.part_rows = r.slots * c.n_kv_heads * tile;
    } else {
      const int64_t likely = std::max(n_groups * ((rows * r.wavefronts + 127) / 128) * c.n_kv_heads, (int64_t)1);
      r.splits = (int32_t)std::max((int64_t)1, std::min({(likely > 256 ? 1024 : 512) / likely, std::min(capacity / 256, std::max((int64_t)32, capacity / 512)), kMostParts}));
      r.part_rows = r.splits * heads;
    }
  }
  const auto up = [](int64_t n) { return (n + 15) / 16 * 16; };
  r.cuts_at = up(r.part_rows * (c.head_dim + 2) * 4);
  r.own_at = r.cuts_at + 64 * 8;
  r.split_at = up(r.own_at + heads * (c.head_dim + 2) * 4);
  r.workspace = r.split_at + kv_split_workspace_bytes(c.head_dim, heads);
  return r;
}

}  // namespace flame

extern "C" {

const char *flame_kv_last_error(void) { return g_kv_error; }

int flame_kv_rotation_frequencies(int32_t rot_dim, double base, double *out) {
  g_kv_error = "";
  if (rot_dim < 2 || rot_dim % 2 || !out) return bad("rot_dim must be positive and even, out not NULL");
  if (!(base > 0.0) || !std::isfinite(base)) return bad("base must be positive and finite");
  for (int32_t j = 0; j < rot_dim / 2; ++j) out[j] = std::pow(base, -2.0 * j / rot_dim);
  return FLAME_GR_OK;
}

int flame_kv_workspace_bytes(const flame_kv_config *cfg, int32_t n_seqs, int64_t n_tokens, int64_t *bytes) {
  g_kv_error = "";
  if (int rc = check_config(cfg)) return rc;
  if (int rc = check_batch(cfg, n_seqs, n_tokens)) return rc;
  if (!bytes) return bad("bytes is NULL");
  *bytes = workspace_bound(*cfg, n_seqs, n_tokens);
  return FLAME_GR_OK;
}

int flame_kv_append(const flame_kv_config *cfg, const flame_kv_cache *cache, const flame_kv_rows *k, const flame_kv_rows *v, const flame_kv_rows *q, const flame_kv_rows *q_out,
                    const flame_kv_rotation *rotation, const int32_t *offsets, const int32_t *kv_lens, int32_t n_seqs, int64_t n_tokens, int32_t *faults, void *stream) {
  g_kv_error = "";
  if (int rc = check_config(cfg)) return rc;
  if (int rc = check_batch(cfg, n_seqs, n_tokens)) return rc;
  if (!q != !q_out) return bad("q and q_out go together");
  KvRotation rot;
  if (int rc = take_rotation(cfg, rotation, &rot)) return rc;
  if (n_seqs == 0 || n_tokens == 0) return FLAME_GR_OK;
  KvRows kr, vr, qr, qo;
  if (int rc = take_rows(cfg, k, &kr)) return rc;
  if (int rc = take_rows(cfg, v, &vr)) return rc;
  if (q) {
    if (int rc = take_rows(cfg, q, &qr)) return rc;
    if (int rc = take_rows(cfg, q_out, &qo)) return rc;
  }
  KvPages pages;
  if (int rc = take_pages(cfg, cache, &pages)) return rc;
  if (!offsets || !kv_lens) return bad("offsets or kv_lens is NULL");
  return done(launch_kv_append(KvBatch{offsets, kv_lens, n_seqs, n_tokens, faults}, pages, kr, vr, q ? &qr : nullptr, &qo, rot, cfg->n_q_heads, cfg->n_kv_heads, cfg->head_dim, cfg->dtype,
                               (hipStream_t)stream));
}

int flame_kv_prompt(const flame_kv_config *cfg, const flame_kv_rows *q, const flame_kv_rows *k, const flame_kv_rows *v, const int32_t *q_offsets, const int32_t *k_offsets,
                    int32_t n_seqs, int64_t n_tokens, int64_t n_keys, const flame_kv_rows *out, int32_t *faults, void *stream) {
  g_kv_error = "";
  if (int rc = check_config(cfg)) return rc;
  if (int rc = check_batch(cfg, n_seqs, n_tokens)) return rc;
  if (n_keys < 0 || n_keys > kMaxKeys) return bad("n_keys out of range");
  if (n_seqs == 0 || n_tokens == 0) return FLAME_GR_OK;
  KvAttention a{};
  if (int rc = take_rows(cfg, q, &a.q)) return rc;
  if (int rc = take_rows(cfg, out, &a.out)) return rc;
  if (n_keys > 0) {
    if (int rc = take_rows(cfg, k, &a.k)) return rc;
    if (int rc = take_rows(cfg, v, &a.v)) return rc;
  }
  if (!q_offsets) return bad("q_offsets is NULL");
  a.batch = KvBatch{q_offsets, nullptr, n_seqs, n_tokens, faults};
  a.k_offsets = k_offsets;
  a.n_keys = n_keys;
  take_heads(cfg, &a);
  a.splits = 1;
  return done(launch_kv_attention(a, kv_route(*cfg, n_seqs, n_tokens, false, false, kMaxKeys).wavefronts, (hipStream_t)stream));
}

int flame_kv_extend(const flame_kv_config *cfg, const flame_kv_cache *cache, const flame_kv_rows *q, const int32_t *q_offsets, const int32_t *kv_lens, int32_t n_seqs, int64_t n_tokens,
                    const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults, void *stream) {
  g_kv_error = "";
  if (int rc = check_config(cfg)) return rc;
  if (int rc = check_batch(cfg, n_seqs, n_tokens)) return rc;
  if (n_seqs == 0 || n_tokens == 0) return FLAME_GR_OK;
  if (!q_offsets) return bad("q_offsets is NULL");
  return attend_cache(cfg, cache, q, q_offsets, kv_lens, n_seqs, n_tokens, out, workspace, workspace_bytes, faults, stream);
}

int flame_kv_decode(const flame_kv_config *cfg, const flame_kv_cache *cache, const flame_kv_rows *q, const int32_t *kv_lens, int32_t n_seqs, const flame_kv_rows *out, void *workspace,
                    int64_t workspace_bytes, int32_t *faults, void *stream) {
  g_kv_error = "";
  if (int rc = check_config(cfg)) return rc;
  if (int rc = check_batch(cfg, n_seqs, n_seqs)) return rc;
  if (n_seqs == 0) return FLAME_GR_OK;
  return attend_cache(cfg, cache, q, nullptr, kv_lens, n_seqs, n_seqs, out, workspace, workspace_bytes, faults, stream);
}

int flame_kv_shared_workspace_bytes(const flame_kv_config *cfg, int32_t n_groups, int32_t n_seqs, int64_t n_tokens, int64_t *bytes) {
  g_kv_error = "";
  if (int rc = check_config(cfg)) return rc;
  if (int rc = check_groups(cfg, n_groups, n_seqs, n_tokens)) return rc;
  if (!bytes) return bad("bytes is NULL");
  *bytes = shared_workspace_bound(*cfg, n_seqs, n_tokens);
  return FLAME_GR_OK;
}

int flame_kv_shared(const flame_kv_config *cfg, const flame_kv_cache *cache, const flame_kv_rows *q, const int32_t *q_offsets, const int32_t *kv_lens, const flame_kv_groups *groups,
                    int32_t n_seqs, int64_t n_tokens, const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults, void *stream) {
  return attend_shared(cfg, cache, nullptr, true, q, q_offsets, kv_lens, groups, n_seqs, n_tokens, out, workspace, workspace_bytes, faults, stream);
}

int flame_kvq_shared(const flame_kv_config *cfg, const flame_kvq_cache *cache, const flame_kv_rows *q, const int32_t *q_offsets, const int32_t *kv_lens, const flame_kv_groups *groups,
                     int32_t n_seqs, int64_t n_tokens, const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults, void *stream) {
  return attend_shared(cfg, nullptr, cache, false, q, q_offsets, kv_lens, groups, n_seqs, n_tokens, out, workspace, workspace_bytes, faults, stream);
}

int flame_kvq_append(const flame_kv_config *cfg, const flame_kvq_cache *cache, const flame_kv_rows *k, const flame_kv_rows *v, const flame_kv_rows *q, const flame_kv_rows *q_out,
                     const flame_kv_rotation *rotation, const int32_t *offsets, const int32_t *kv_lens, int32_t n_seqs, int64_t n_tokens, int32_t *faults, void *stream) {
  g_kv_error = "";
  if (int rc = check_config(cfg)) return rc;
  if (int rc = check_batch(cfg, n_seqs, n_tokens)) return rc;
  if (!q != !q_out) return bad("q and q_out go together");
  KvRotation rot;
  if (int rc = take_rotation(cfg, rotation, &rot)) return rc;
  if (n_seqs == 0 || n_tokens == 0) return FLAME_GR_OK;
  KvRows kr, vr, qr, qo;
  if (int rc = take_rows(cfg, k, &kr)) return rc;
  if (int rc = take_rows(cfg, v, &vr)) return rc;
  if (q) {
    if (int rc = take_rows(cfg, q, &qr)) return rc;
    if (int rc = take_rows(cfg, q_out, &qo)) return rc;
  }
  KvPages pages;
  KvScales scales;
  if (int rc = take_pages(cfg, cache, &pages, &scales)) return rc;
  if (!offsets || !kv_lens) return bad("offsets or kv_lens is NULL");
  return done(launch_kvq_append(KvBatch{offsets, kv_lens, n_seqs, n_tokens, faults}, pages, scales, kr, vr, q ? &qr : nullptr, &qo, rot, cfg->n_q_heads, cfg->n_kv_heads, cfg->head_dim,
                                cfg->dtype, (hipStream_t)stream));
}

int flame_kvq_read(const flame_kv_config *cfg, const flame_kvq_cache *cache, const int32_t *offsets, const int32_t *kv_lens, int32_t n_seqs, int64_t n_tokens, const flame_kv_rows *k,
                   const flame_kv_rows *v, int32_t *faults, void *stream) {
  g_kv_error = "";
  if (int rc = check_config(cfg)) return rc;
  if (int rc = check_batch(cfg, n_seqs, n_tokens)) return rc;
  if (n_seqs == 0 || n_tokens == 0) return FLAME_GR_OK;
  KvRows kr, vr;
  if (int rc = take_rows(cfg, k, &kr)) return rc;
  if (int rc = take_rows(cfg, v, &vr)) return rc;
  KvPages pages;
  KvScales scales;
  if (int rc = take_pages(cfg, cache, &pages, &scales)) return rc;
  if (!offsets || !kv_lens) return bad("offsets or kv_lens is NULL");
  return done(launch_kvq_read(KvBatch{offsets, kv_lens, n_seqs, n_tokens, faults}, pages, scales, kr, vr, cfg->n_kv_heads, cfg->head_dim, cfg->dtype, (hipStream_t)stream));
}

int flame_kvq_extend(const flame_kv_config *cfg, const flame_kvq_cache *cache, const flame_kv_rows *q, const int32_t *q_offsets, const int32_t *kv_lens, int32_t n_seqs, int64_t n_tokens,
                     const flame_kv_rows *out, void *workspace, int64_t workspace_bytes, int32_t *faults, void *stream) {
  g_kv_error = "";
  if (int rc = check_config(cfg)) return rc;
  if (int rc = check_batch(cfg, n_seqs, n_tokens)) return rc;
  if (n_seqs == 0 || n_tokens == 0) return FLAME_GR_OK;
  if (!q_offsets) return bad("q_offsets is NULL");
  return attend_quantised(cfg, cache, q, q_offsets, kv_lens, n_seqs, n_tokens, out, workspace, workspace_bytes, faults, stream);
}

int flame_kvq_decode(const flame_kv_config *cfg, const flame_kvq_cache *cache, const flame_kv_rows *q, const int32_t *kv_lens, int32_t n_seqs, const flame_kv_rows *out, void *workspace,
                     int64_t workspace_bytes, int32_t *faults, void *stream) {
  g_kv_error = "";
  if (int rc = check_config(cfg)) return rc;
  if (int rc = check_batch(cfg, n_seqs, n_seqs)) return rc;
  if (n_seqs == 0) return FLAME_GR_OK;
  return attend_quantised(cfg, cache, q, nullptr, kv_lens, n_seqs, n_seqs, out, workspace, workspace_bytes, faults, stream);
}

}  // extern "C"
