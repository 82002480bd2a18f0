// Where a token of a sequence lies in a paged cache.  Plain integer arithmetic, for the kernels and for the host.
#pragma once
#include <stdint.h>

#ifdef __HIP__
#define FLAME_HD __host__ __device__ __forceinline__
#else
#define FLAME_HD inline
#endif

namespace flame {

// n / page_size for 0 <= n < 2^31 is (n * magic) >> (31 + shift): magic = ceil(2^(31 + shift) / page_size), 2^shift >= page_size, so that
// the excess of the product, n * (magic * page_size - 2^(31 + shift)) < 2^31 * page_size, never reaches the next multiple.
struct KvPages {
  char *k, *v;
  int64_t page, slot, head;  // strides in bytes
  int32_t n_pages, page_size;
  uint32_t magic;
  int32_t shift;
  const int32_t *table;
  int64_t table_stride;
  int32_t capacity;          // tokens that a row of the table has room for
};

inline void kv_set_page_size(KvPages *p, int32_t page_size) {
  p->page_size = page_size;
  p->shift = 0;
  while ((int64_t)1 << p->shift < page_size) ++p->shift;
  p->magic = (uint32_t)((((uint64_t)1 << (31 + p->shift)) + page_size - 1) / page_size);
}

FLAME_HD uint32_t kv_page_index(const KvPages &p, uint32_t n) { return (uint32_t)(((uint64_t)n * p.magic) >> (31 + p.shift)); }

// Byte offset of token t (0 <= t < capacity) of the sequence whose table row is `table` from the pool's start, or -1 where the table names
// no page of the pool.
FLAME_HD int64_t kv_token_offset(const KvPages &p, const int32_t *table, uint32_t t) {
  const uint32_t i = kv_page_index(p, t);
  const int32_t page = table[i];
  if ((uint32_t)page >= (uint32_t)p.n_pages) return -1;
  return page * p.page + (int64_t)(t - i * (uint32_t)p.page_size) * p.slot;
}

// Tokens of a sequence, within what its row of the table has room for.
FLAME_HD int32_t kv_clip(int32_t len, int32_t capacity) { return len < 0 ? 0 : len < capacity ? len : capacity; }

}  // namespace flame
