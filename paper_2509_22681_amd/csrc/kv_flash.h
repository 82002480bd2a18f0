// Causal softmax attention of packed query rows with grouped heads, over packed keys or a paged cache.
//
// Bound by the matrix pipe and the vector work of the softmax beside it, and in the end by power: one prompt of 32768, 16/2 heads of 128, bf16, runs at 1.0 PFLOP/s (4.4 ms) and a clock of
// 2.0 GHz, with the matrix pipe busy 48 % of the cycles (a plain matrix product of 8192 reaches 1.22 PFLOP/s on this chip).  Forms with fewer cycles ran at a lower clock in the same time.
//
// A workgroup takes 128 query rows of one sequence and key head, row = token * G + head of the
// group (the G query heads that share a key head are rows of one tile: short sequences fill it, and the mask cuts through fewer key tiles), four wavefronts of 32 rows each.  It
// walks the keys in tiles of 32 or 64 (key_block), two stages in LDS, brought there by LDS-DMA loads one tile ahead.  In small launches two or four wavefronts share 32 rows and take 32
// or 64 keys each of tiles that are two or four times as long, with a maximum, sum and accumulator of their own that are joined at the end (kv_route in kv_api.cpp).  Products are transposed as in attn_mfma.hip,
//     S^T[key][row] = K Q^T        A operand = K rows, B operand = Q rows
//     O^T[feature][row] += V^T P^T A operand = V^T rows, B operand = P^T
// so that the first product's accumulator, where a lane has one row and 16 of 32 keys, is the second product's B operand as it stands: elements 8 s + i of a lane in half h are keys
// 16 s + 8 (i / 4) + 4 h + i % 4.  V lies in the cache key by key, and the A operand wants eight keys of a feature per lane: the transposing LDS read (ds_read_b64_tr_b16) gives
// each of 16 lanes one column of four 16-bit rows, so two of them make a fragment.
//
// LDS rows are unpadded, as the DMA fills 1 KB of consecutive bytes, and swizzled by XOR: K in 16-byte chunks with the low bits of the key, V in 32-byte chunks so that the four
// rows and two neighbouring chunks that 32 lanes of a transposing read touch lie in the eight different 32-byte slots of 256 bytes.
//
// Where a key lies: a wavefront looks up 64 keys of a tile, two tiles ahead, and leaves their byte offsets in LDS for the requests of all; packed keys take the same way.  Any page
// size and any strides cost the same.
//
// Masked keys: their logits are -infinity, and their values meet weights of zero.  That is harmless while they are finite.  If a workgroup's
// results are not all finite at the end, it runs its keys once more with the values of masked tiles taken apart (see `careful`), so that infinities and NaN reach exactly the rows that see them.
//
// Over a cache of 8 or 4 bits a thread loads the codes of 16 features at a time into registers, a tile ahead, and when the products of this tile are done it makes the next one's LDS rows of
// them: what follows is the same.  With shared histories (SHARED) a group of sequences is one sequence, whose rows are those of all of them and whose keys are the history; each row
// sees as far as its own sequence and position let it, and all results are parts, which kv_shared.h joins with those of the sequences' own keys.
#pragma once
#include "kernels.h"
#include "kv_codec.h"

namespace flame {

namespace {

// KP wavefronts share 32 query rows and take KT keys of each tile of KP KT apiece.
constexpr int kFlashRows = 128;     // query rows of a workgroup are this / KP
template <typename T, int DH, int KP> constexpr int key_block() { return DH * sizeof(T) >= (KP == 1 ? 512 : KP == 2 ? 256 : 128) ? 32 : 64; }
// Two stages of K and V, and in the end their place has room for the parts of rows: 4 x 32 rows of DH + 4 floats, a maximum and a sum.
template <typename T, int DH, int KP> constexpr int flash_lds_bytes() {
  constexpr int stages = 4 * KP * key_block<T, DH, KP>() * DH * (int)sizeof(T), parts = KP == 1 ? 0 : 4 * 32 * (DH + 6) * 4;
  return stages > parts ? stages : parts;
}
// Workgroups of 4 wavefronts on a compute unit, as LDS and registers allow (three in place of two of heads of 64: 64 prompts of 512..1024, 8 heads, 142 -> 114 us, one of 16384 395 -> 352;
// four in place of three of 32 features 185 -> 165, fp32 three in place of two 622 -> 561).  Over values heads of 32 spill up to 4 registers at these bounds, none of it between the products.
// Over codes, which wait for their conversion in registers, 16-bit heads of 32 spill 9 to 44 with one or two wavefronts to 32 rows, and heads of 64 7 to 11 with one (kv_shared.h: 13 to 29, and 6 to 10).  It pays all the
// same where workgroups are many, and costs something where rounds are few.  us at these bounds | with one workgroup less, f8 (f4), bf16: 32 prompts of 512..1024, 16/16 heads of 32, 81 | 93 (85 | 92), fp32 287 | 313 (286 |
// 312); 64 prompts, 8/2 heads of 64, 107 | 137 (106 | 136); 64 x 64 new over 300..4000, 16/16 of 32, 122 | 116 (123 | 109); 6 x 400 over 4000..16384 186 | 186 (186 | 172, fp16 172 | 172); histories that are shared: 400
// sequences behind 4 of 4000..10000, 16/16 of 32, 57 | 60 (55 | 59), fp32 127 | 139 (127 | 138), 200 of them 40 | 40; 256 behind 2 of 8000..16000, 8/8 of 64, 37 | 41 (37 | 41).
template <typename T, int DH, int KP> constexpr int flash_workgroups() {
  constexpr int lds = flash_lds_bytes<T, DH, KP>();
  return lds > 72 * 1024 ? 1 : DH == 32 && sizeof(T) == 2 && lds <= 32 * 1024 ? 4 : DH * sizeof(T) <= 128 && lds <= 40 * 1024 ? 3 : 2;
}

template <typename T> struct Matrix32;              // (fp32 products are 32x32x2: the third dimension is the lane's half)
template <> struct Matrix32<bf16_t> {
  typedef bf16x8 frag;
  static __device__ __forceinline__ f32x16 mul(frag x, frag y, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0); }
};
template <> struct Matrix32<half_t> {
  typedef f16x8 frag;
  static __device__ __forceinline__ f32x16 mul(frag x, frag y, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, c, 0, 0, 0); }
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// Values of 16 keys, transposed: the fragments of all feature blocks, two reads each.  The builtin for this instruction makes the compiler wait for the LDS-DMA
// loads in flight, which are the next tile's; hence assembly, that waits for its own reads before it ends.
template <int DB, int RB, int AT> __device__ __forceinline__ void read_values(uint32_t stage, uint32_t at, s16x4 (&v)[DB][2]) {
#define READ(o, a, n) "ds_read_b64_tr_b16 " o ", " a " offset:" n "\n\t"
  if constexpr (DB == 4) {
    asm volatile(READ("%0", "%8", "%12") READ("%1", "%8", "%13") READ("%2", "%9", "%12") READ("%3", "%9", "%13")
                 READ("%4", "%10", "%12") READ("%5", "%10", "%13") READ("%6", "%11", "%12") READ("%7", "%11", "%13") "s_waitcnt lgkmcnt(0)"
                 : "=&v"(v[0][0]), "=&v"(v[0][1]), "=&v"(v[1][0]), "=&v"(v[1][1]), "=&v"(v[2][0]), "=&v"(v[2][1]), "=&v"(v[3][0]), "=&v"(v[3][1])
                 : "v"(stage + at), "v"(stage + (at ^ 64)), "v"(stage + (at ^ 128)), "v"(stage + (at ^ 192)), "n"(AT), "n"(AT + 8 * RB)
                 : "memory");
  } else if constexpr (DB == 2) {
    asm volatile(READ("%0", "%4", "%6") READ("%1", "%4", "%7") READ("%2", "%5", "%6") READ("%3", "%5", "%7") "s_waitcnt lgkmcnt(0)"
                 : "=&v"(v[0][0]), "=&v"(v[0][1]), "=&v"(v[1][0]), "=&v"(v[1][1])
                 : "v"(stage + at), "v"(stage + (at ^ 64)), "n"(AT), "n"(AT + 8 * RB)
                 : "memory");
  } else {
    asm volatile(READ("%0", "%2", "%3") READ("%1", "%2", "%4") "s_waitcnt lgkmcnt(0)"
                 : "=&v"(v[0][0]), "=&v"(v[0][1])
                 : "v"(stage + at), "n"(AT), "n"(AT + 8 * RB)
                 : "memory");
  }
#undef READ
}

// A row tile's keys in parts: of at least kPartTiles tiles, up to `splits` of them.
constexpr int kPartTiles = 4;
struct FlashParts { int parts, tiles; };
template <int KW> __device__ __forceinline__ FlashParts flash_parts(int n_seen, int splits) {
  const int tiles = (n_seen + KW - 1) / KW;
  FlashParts p{1, tiles};
  if (splits > 1 && tiles > kPartTiles) {
    const int most = min(splits, tiles / kPartTiles);
    p.tiles = (tiles + most - 1) / most;
    p.parts = (tiles + p.tiles - 1) / p.tiles;
  }
  return p;
}

// Which sequences of the batch have rows: all, or of up to 64 those before the first offsets that are none.
__device__ __forceinline__ int flash_sequences(const KvAttention &a, int lane) {
  if (!a.batch.offsets || a.batch.n_seqs > 64) return a.batch.n_seqs;
  const uint64_t wrong = __builtin_amdgcn_ballot_w64(lane < a.batch.n_seqs && kv_wrong_offsets(a.batch.offsets[min(lane, a.batch.n_seqs - 1)], a.batch.offsets[min(lane, a.batch.n_seqs - 1) + 1]));
  return wrong ? __builtin_ctzll(wrong) : a.batch.n_seqs;
}

// A group of sequences that share a history: its sequences and rows.
struct FlashGroup {
  int b0, b1;
  int64_t first, end;
  bool wrong;
};
__device__ __forceinline__ FlashGroup flash_group(const KvAttention &a, int g, int n_seqs) {
  const int g0 = a.group_offsets[g], g1 = a.group_offsets[g + 1];
  FlashGroup s{0, 0, 0, 0, kv_wrong_offsets(g0, g1)};
  if (s.wrong) return s;
  s.b0 = min(g0, n_seqs);
  s.b1 = min(g1, n_seqs);
  s.first = a.batch.offsets ? a.batch.offsets[s.b0] : s.b0;
  s.end = a.batch.offsets ? a.batch.offsets[s.b1] : s.b1;
  return s;
}
__device__ __forceinline__ int flash_history(const KvAttention &a, const FlashGroup &s) { return s.b0 < s.b1 ? kv_clip(a.prefix_lens[s.b0], a.pages.capacity) : 0; }
// Keys of the history that a row sees.
__device__ __forceinline__ int flash_shared_seen(const KvAttention &a, const FlashGroup &s, int64_t row, int history) {
  int b = (int)min(row, (int64_t)s.b1 - 1);
  int64_t end = row + 1;
  if (a.batch.offsets) {
    int lo = s.b0, hi = s.b1 - 1;                                 // the first sequence that ends behind the row
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (a.batch.offsets[mid + 1] > row) hi = mid;
      else lo = mid + 1;
    }
    b = lo;
    end = a.batch.offsets[b + 1];
    if (row < a.batch.offsets[b] || row >= end) return 0;
  }
  const int64_t sees = kv_clip(a.batch.kv_lens[b], a.pages.capacity) - (end - row) + 1;
  return (int)max((int64_t)0, min(sees, (int64_t)min(history, kv_clip(a.prefix_lens[b], a.pages.capacity))));
}

// How the keys of shared histories are cut where there is room for `budget` workgroups a key head: lane g holds group g (of up to 64), whose `tiles` row tiles have `keys` key tiles each.  All parts have the same
// number of key tiles, the least (of at least kSharedTiles) with which they are no more than the budget; the last one of a row tile may be shorter.  Half the budget does where parts would be of less than
// `long_part` key tiles: one workgroup on a compute unit reads as fast as two, and leaves half as many parts.  us with 512 | 256 workgroups, bf16, 32/8 heads of 128, single tokens: 16 sequences over 16384
// shared tokens 43 | 33, 32 over 8000 41 | 29, 128 over 32000 124 | 162; 400, 16/16 heads of 32, in 4 groups over 4000-10000 51 | 66
constexpr int kSharedTiles = 2, kLongPart = 8;
struct FlashCut {
  int parts, before;     // of a row tile of the lane's group; slots of the groups ahead of it
  int chunk;
};
template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ int flash_dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int flash_scan(int v) {               // inclusive sums over the wavefront
  v += flash_dpp<0x111>(v);                                      // row_shr:1, 2, 4, 8
  v += flash_dpp<0x112>(v);
  v += flash_dpp<0x114>(v);
  v += flash_dpp<0x118>(v);
  v += flash_dpp<0x142, 0xa>(v);                                 // the last lane of a row to the next row
  v += flash_dpp<0x143, 0xc>(v);                                 // lane 31 to the upper half
  return v;
}
__device__ __forceinline__ int flash_wave_sum(int v) { return __builtin_amdgcn_readlane(flash_scan(v), 63); }
__device__ __forceinline__ FlashCut flash_cut(int tiles, int keys, int budget, int long_part) {
  if (keys == 0) tiles = 0;
  const int work = flash_wave_sum((int)min((int64_t)tiles * keys, (int64_t)1 << 24)), rows = flash_wave_sum(tiles);
  budget = max((budget + 1) / 2, min(budget, work / long_part));
  FlashCut c{0, 0, max(kSharedTiles, (work + budget - 1) / max(budget, 1))};
  // (each step adds a sixteenth: from the least that could do to a part for each row tile there are fewer than 200)
  for (;;) {
    c.parts = tiles ? (keys + c.chunk - 1) / c.chunk : 0;
    const int all = flash_wave_sum(tiles * c.parts);
    if (all <= budget || all == rows) break;
    c.chunk += max(1, c.chunk / 16);
  }
  c.before = flash_scan(tiles * c.parts) - tiles * c.parts;
  return c;
}

// (kv_shared.h runs this beside split attention in one launch: `block` of `blocks` is its own.)
template <typename T, int DH, bool PAGED, int KP, int FORM, bool SHARED>
__device__ __forceinline__ void flash_rows(const KvAttention &a, unsigned my_block, unsigned blocks) {
  static_assert(PAGED || (FORM == kPlain && !SHARED), "codes and histories lie in pages");
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int QT = kFlashRows / KP;                             // query rows of a workgroup
  constexpr int KT = key_block<T, DH, KP>(), NJ = KT / 32;        // a wavefront's keys of a tile, 32-key blocks of them
  constexpr int KW = KP * KT;                                     // keys of a tile
  constexpr int RB = DH * (int)sizeof(T), CH = RB / 16;           // bytes of a row, and 16-byte chunks
  constexpr int KS = RB / 32, DB = DH / 32;                       // steps of 32 bytes along a row (16 per lane), feature blocks
  constexpr int TILE = KW * RB;                                   // bytes of a K or V tile
  constexpr int STAGE = 2 * TILE;
  constexpr int RPI = 64 / CH, NI = TILE / 1024 / 4;              // rows of a 1 KB request, requests of a wavefront per tile of K or V
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  __shared__ int64_t at_s[3][PAGED ? 1 : 2][KW];                  // byte offsets of a tile's keys (packed: and values)
  __shared__ uint32_t there_s[3][KW / 32];                        // which of them count
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, lh = lane >> 5;
  const int group = a.n_q_heads / a.n_kv_heads;

  // Which tile.  Tiles with most keys go first: the sequences by their number of keys, and each from its end.
  if (!SHARED && my_block == 0 && a.batch.faults)
    for (int b = threadIdx.x; b < a.batch.n_seqs; b += 256) {
      const int64_t first = a.batch.offsets[b], end = a.batch.offsets[b + 1];
      kv_report_offsets(first, end, a.batch.n_rows, a.batch.faults);
      if (PAGED) {
        kv_clip_length(a.batch.kv_lens[b], a.pages.capacity, a.batch.faults, true);
      } else if (a.k_offsets) {
        kv_report_offsets(a.k_offsets[b], a.k_offsets[b + 1], a.n_keys, a.batch.faults);
      } else {
        kv_report_offsets(first, end, a.n_keys, a.batch.faults);
      }
    }
  // Of a compute unit's workgroups, one is of the first 256 and one of the next: those go the other way round, so that a long one has a short one beside it
  // (4 prompts of 2048, 8/2 heads of 64: 50 -> 40 us, fp32 4 of 1024, 16 heads of 32: 69 -> 60; launches of many more are as before).
  unsigned block = my_block;
  if (!SHARED && flash_workgroups<T, DH, KP>() >= 2) {
    const unsigned placed = min(blocks, 512u);
    if (block >= 256 && block < placed) block = 256 + placed - 1 - block;
  }
  const int kvh = block % a.n_kv_heads;
  const bool balanced = SHARED && a.splits == 0;                  // (see flash_cut)
  const int splits = SHARED ? max(a.splits, 1) : a.splits;
  const int64_t slot = block / a.n_kv_heads / splits;
  int split = block / a.n_kv_heads % splits;
  FlashCut even{1, 0, 0};
  int seq;
  int64_t tile, first, end;                                       // tile: counted from the sequence's end (a group's: from its first row)
  int kv_len = 0;
  const int n_spans = SHARED ? a.n_groups : a.batch.n_seqs, n_seqs = SHARED ? flash_sequences(a, lane) : 0;
  if (n_spans <= 64) {
    // One lane per sequence: the tiles of those that come before it.
    int64_t tiles = 0;
    int b = 0, e = 0, keys = -1;
    bool none = false;
    if (lane < n_spans) {
      if constexpr (SHARED) {
        const FlashGroup s = flash_group(a, lane, n_seqs);
        b = (int)s.first;
        e = (int)s.end;
        none = s.wrong;
        keys = none ? 0 : flash_history(a, s);
      } else {
        b = a.batch.offsets[lane];
        e = a.batch.offsets[lane + 1];
        keys = PAGED ? a.batch.kv_lens[lane] : (int)((int64_t)e - b);
      }
      tiles = (max((int64_t)0, min((int64_t)e, a.batch.n_rows) - b) * group + QT - 1) / QT;
    }
    const uint64_t wrong = __builtin_amdgcn_ballot_w64(none || kv_wrong_offsets(b, e));
    if (wrong && lane >= __builtin_ctzll(wrong)) tiles = 0;
    int before = 0;
    if (balanced) {
      even = flash_cut((int)tiles, (max(keys, 0) + KW - 1) / KW, a.budget, kLongPart * KP);
      if (my_block == 0 && threadIdx.x < 64) a.cuts[lane] = int2{even.before, even.parts};
      before = even.before;
      tiles *= even.parts;
    } else {
      for (int j = 0; j < n_spans; ++j) {
        const int other = __builtin_amdgcn_readlane(keys, j);
        before += other > keys || (other == keys && j < lane) ? __builtin_amdgcn_readlane((int)tiles, j) : 0;
      }
    }
    const uint64_t mine = __builtin_amdgcn_ballot_w64(slot >= before && slot < before + tiles);
    if (!mine) return;
    seq = __builtin_ctzll(mine);
    tile = slot - __builtin_amdgcn_readlane(before, seq);
    if (balanced) {
      even.parts = __builtin_amdgcn_readlane(even.parts, seq);
      split = (int)tile % even.parts;
      tile = (int)tile / even.parts;
    }
    first = __builtin_amdgcn_readlane(b, seq);
    end = __builtin_amdgcn_readlane(e, seq);
    if (PAGED) kv_len = __builtin_amdgcn_readlane(keys, seq);
  } else {
    // Those of sequence b begin at slot offsets[b] * G / QT + b, where there is room for them whatever the lengths; the last sequence goes first.
    const int64_t back_slot = blocks / a.n_kv_heads / splits - 1 - slot;
    int lo = 0, n = n_spans;                                      // the last sequence whose slots begin at or before this one
    while (n > 1) {
      const int step = (n + 63) / 64;
      const int b = lo + min((lane + 1) * step, n - 1);
      int64_t at;
      if constexpr (SHARED) {
        const FlashGroup s = flash_group(a, b, n_seqs);
        at = max(s.first, (int64_t)0);
      } else {
        at = a.batch.offsets[b];
      }
      const bool after = (lane + 1) * step >= n || at * group / QT + b > back_slot;
      const int c = __builtin_ctzll(__builtin_amdgcn_ballot_w64(after) | 1ull << 63);
      lo += c * step;
      n = max(1, min(step, n - c * step));
    }
    seq = min(lo, n_spans - 1);
    if constexpr (SHARED) {
      const FlashGroup s = flash_group(a, seq, n_seqs);
      if (s.wrong) return;
      first = s.first;
      end = s.end;
      kv_len = flash_history(a, s);
    } else {
      first = a.batch.offsets[seq];
      end = a.batch.offsets[seq + 1];
      if (PAGED) kv_len = a.batch.kv_lens[seq];
    }
    const int64_t tiles = (max((int64_t)0, min(end, a.batch.n_rows) - first) * group + QT - 1) / QT;
    tile = tiles - 1 - (back_slot - (first * group / QT + seq));
  }
  if (first < 0 || end < first) return;
  const int rows = (int)max((int64_t)0, min(end, a.batch.n_rows) - first) * group;
  const int row_tiles = (rows + QT - 1) / QT;
  if (tile < 0 || tile >= row_tiles) return;
  const int row0 = SHARED ? (int)tile * QT : (row_tiles - 1 - (int)tile) * QT;

  int n;
  const char *kp, *vp;
  const int32_t *table = nullptr;
  if (PAGED) {
    n = kv_clip(kv_len, a.pages.capacity);
    kp = a.pages.k + kvh * a.pages.head;
    vp = a.pages.v + kvh * a.pages.head;
    if constexpr (!SHARED) table = a.pages.table + seq * a.pages.table_stride;
  } else {
    int64_t k_first = first, k_end = end;
    if (a.k_offsets) {
      k_first = a.k_offsets[seq];
      k_end = a.k_offsets[seq + 1];
    }
    n = k_first < 0 ? 0 : (int)max((int64_t)0, min(k_end, a.n_keys) - k_first);
    kp = a.k.p + k_first * a.k.row + kvh * a.k.head;
    vp = a.v.p + k_first * a.v.row + kvh * a.v.head;
  }
  // keys seen: by the row before the first one of the sequence, by the last row of the workgroup, by the first and last of my wavefront, by my row
  const int64_t back = n - (end - first);
  auto seen_by = [&](int row) { return (int)max((int64_t)0, back + row / group + 1); };
  const int n_seen = SHARED ? n : seen_by(min(row0 + QT, rows) - 1);
  // the workgroup's tiles: all, or a part of them
  const FlashParts cut = balanced ? FlashParts{even.parts, even.chunk} : flash_parts<KW>(n_seen, splits);
  if (split >= cut.parts || (SHARED && n == 0)) return;
  const int t_begin = split * cut.tiles, n_tiles = min(cut.tiles, (n_seen + KW - 1) / KW - t_begin), key0 = t_begin * KW;
  const int part = KP == 1 ? 0 : wave % KP, wave_row = row0 + wave / KP * 32;
  const bool active = wave_row < rows;
  auto my_row = [&]() { return active ? min(wave_row + l32, rows - 1) : row0; };
  int sees, wave_least, wave_most;
  if constexpr (SHARED) {
    const FlashGroup s = flash_group(a, seq, n_seqs);
    table = a.pages.table + s.b0 * a.pages.table_stride;
    sees = flash_shared_seen(a, s, first + my_row() / group, n);
    // over the 32 rows, which both halves of the wavefront have: rotations within 16 lanes, and the two rows of lanes
    int least = sees, most = sees;
    least = min(least, flash_dpp<0x121>(least));
    most = max(most, flash_dpp<0x121>(most));
    least = min(least, flash_dpp<0x122>(least));
    most = max(most, flash_dpp<0x122>(most));
    least = min(least, flash_dpp<0x124>(least));
    most = max(most, flash_dpp<0x124>(most));
    least = min(least, flash_dpp<0x128>(least));
    most = max(most, flash_dpp<0x128>(most));
    wave_least = active ? min(__builtin_amdgcn_readlane(least, 0), __builtin_amdgcn_readlane(least, 16)) : 0;
    wave_most = active ? max(__builtin_amdgcn_readlane(most, 0), __builtin_amdgcn_readlane(most, 16)) : 0;
  } else {
    sees = seen_by(my_row());
    wave_least = active ? seen_by(wave_row) : 0;
    wave_most = active ? seen_by(min(wave_row + 31, rows - 1)) : 0;
  }

  typedef __attribute__((address_space(1))) const void gvoid;
  typedef __attribute__((address_space(3))) void lvoid;
  // Each wavefront looks after 64 keys of a tile, as far as they go.
  const int ring = wave * 64 + lane;
  const bool looks = wave * 64 < KW;
  auto look_up = [&](int t, int64_t (&to)[2]) {                   // of key `ring` of tile t; -1: none
    const int near = min(key0 + t * KW + ring, n - 1);
    if (PAGED) {
      to[0] = kv_token_offset(a.pages, table, (uint32_t)near);
    } else {
      to[0] = near * a.k.row;
      to[1] = near * a.v.row;
    }
  };
  auto publish = [&](int t, const int64_t (&from)[2]) {
    const int64_t k_at = from[0];
    const bool mine = ring < KW;
    if (PAGED && mine && k_at < 0) kv_fault(a.batch.faults, FLAME_KV_FAULT_PAGE);
    if (mine) {
      at_s[t % 3][0][ring] = max(k_at, (int64_t)0);
      if (!PAGED) at_s[t % 3][PAGED ? 0 : 1][ring] = from[1];
    }
    const uint64_t there = __builtin_amdgcn_ballot_w64((!PAGED || k_at >= 0) && key0 + t * KW + ring < n);
    if (mine && (lane & 31) == 0) there_s[t % 3][ring / 32] = (uint32_t)(there >> lane);
  };
  // swizzle: what the chunk index of a row is XORed with (fp32 values are read a row at a time, side by side: no need)
  auto k_key_of = [](int r) { return RB >= 256 ? r & 15 : RB == 128 ? r >> 1 & 7 : r >> 2 & 3; };
  auto v_key_of = [](int r) { return F32 || RB == 64 ? 0 : RB == 256 ? 4 * (r & 3) : 4 * (r >> 1 & 1); };
  // Request j of a tile is rows j RPI..; lane p brings the chunk that belongs at byte 16 p of it.
  const int in_row = lane / CH, chunk = lane % CH;
  auto request = [&](int t) {
    char *stage = lds + (t & 1) * STAGE;
    const int64_t *ka = at_s[t % 3][0], *va = at_s[t % 3][PAGED ? 0 : 1];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int j = wave + 4 * i, r = j * RPI + in_row;
      const int kc = chunk ^ k_key_of(r), vc = chunk ^ v_key_of(r);
      __builtin_amdgcn_global_load_lds((gvoid *)(kp + ka[r] + kc * 16), (lvoid *)(stage + j * 1024), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((gvoid *)(vp + va[r] + vc * 16), (lvoid *)(stage + TILE + j * 1024), 16, 0, 0);
    }
  };

  typedef uint32_t word4 __attribute__((ext_vector_type(4)));
  // Codes of a tile: units of 16 features, those of K and then those of V, one thread after another; CB bytes of codes each, which make CU chunks of a row.
  constexpr int CB = kv_row_bytes<T, FORM>(16), UNITS = KW * DH / 16, NU = 2 * UNITS / 256, CU = 16 * (int)sizeof(T) / 16;
  struct Codes {
    uint32_t w[CB / 4], scale;
  } codes[FORM == kPlain ? 1 : NU];
  auto fetch = [&](int t) {
    if constexpr (FORM != kPlain) {
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const int u = threadIdx.x + 256 * i, in = u & (UNITS - 1), r = in / (DH / 16), c = in % (DH / 16);
        const bool value = UNITS >= 256 ? i >= NU / 2 : u >= UNITS;
        const int64_t from = kvh * a.pages.head + at_s[t % 3][0][r] + c * CB;
        struct alignas(CB) Words { uint32_t w[CB / 4]; };
        const Words y = *(const Words *)((value ? a.pages.v : a.pages.k) + from);
#pragma unroll
        for (int j = 0; j < CB / 4; ++j) codes[i].w[j] = y.w[j];
        codes[i].scale = *(const uint8_t *)((value ? a.v_scales : a.k_scales) + (from >> kv_scale_shift<FORM>()));
      }
    }
  };
  auto land = [&](int t) {
    if constexpr (FORM != kPlain) {
      char *stage = lds + (t & 1) * STAGE;
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const int u = threadIdx.x + 256 * i, in = u & (UNITS - 1), r = in / (DH / 16), c = in % (DH / 16);
        const bool value = UNITS >= 256 ? i >= NU / 2 : u >= UNITS;
        const int key = value ? v_key_of(r) : k_key_of(r);
        char *row = stage + (value ? TILE : 0) + r * RB;
        typedef typename KvPair<T>::vec pair;
        struct alignas(16) Chunks { pair p[8]; } x;
        pair y[4];
        kv_eight<T, FORM>(codes[i].w, kv_scale(codes[i].scale), y);
#pragma unroll
        for (int j = 0; j < 4; ++j) x.p[j] = y[j];
        kv_eight<T, FORM>(codes[i].w + CB / 8, kv_scale(codes[i].scale), y);
#pragma unroll
        for (int j = 0; j < 4; ++j) x.p[4 + j] = y[j];
#pragma unroll
        for (int j = 0; j < CU; ++j) *(word4 *)(row + (((c * CU + j) ^ key) << 4)) = ((const word4 *)&x)[j];
      }
    }
  };
  word4 fq[KS];
  {
    const int row = my_row(), token = row / group, head = kvh * group + row - token * group;
    const char *q = a.q.p + (first + token) * a.q.row + head * a.q.head;
#pragma unroll
    for (int s = 0; s < KS; ++s) fq[s] = *(const word4 *)(q + s * 32 + lh * 16);
  }
  const float scale = a.scale * kLog2e;
  // K: row l32 (+ 32) of the tile, chunk 2 s + lh
  const int ka0 = l32 * RB + ((k_key_of(l32) ^ lh) << 4);         // ^ (s << 5)
  // V: lane l of a transposing read addresses key 4 lh + (l % 16) / 4, features 16 (l / 16 % 2) + 4 (l % 4), and gets feature l % 32 of four keys
  // (rows 8 and 16 further have the same swizzle).  fp32: lane l reads features DB (l % 32).. of key 4 lh
  const int v_row = 4 * lh + (F32 ? 0 : lane >> 2 & 3);
  const int va0 = v_row * RB + (F32 ? l32 * DB * 4 : ((((lane >> 4 & 1) * 2 + (lane >> 1 & 1)) ^ v_key_of(v_row)) << 4) + (lane & 1) * 8);   // ^ (b << 6), + 8 rows each

  f32x16 o[DB];
  float m, l;
  auto tile_step = [&](int t, auto careful_c) __attribute__((always_inline)) {
    constexpr bool careful = decltype(careful_c)::value;
    const char *sk = lds + (t & 1) * STAGE + part * (KT * RB), *sv = sk + TILE;
    const int k0 = key0 + t * KW + part * KT;
    if (k0 >= wave_most) return;
    const uint32_t there_lo = __builtin_amdgcn_readfirstlane((int)there_s[t % 3][part * NJ]), there_hi = NJ == 2 ? __builtin_amdgcn_readfirstlane((int)there_s[t % 3][part * NJ + NJ - 1]) : ~0u;
    const bool masked = k0 + KT > wave_least || (there_lo & there_hi) != 0xffffffffu;
    f32x16 z[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) z[j][e] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const word4 fk = *(const word4 *)(sk + j * (32 * RB) + (ka0 ^ (s << 5)));
        if constexpr (F32) {
#pragma unroll
          for (int i = 0; i < 4; ++i) z[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(fk[i]), __uint_as_float(fq[s][i]), z[j], 0, 0, 0);
        } else {
          typedef typename Matrix32<T>::frag frag;
          z[j] = Matrix32<T>::mul(__builtin_bit_cast(frag, fk), __builtin_bit_cast(frag, fq[s]), z[j]);
        }
      }
    // element e of block j: key 32 j + 8 (e / 4) + 4 lh + e % 4
    uint32_t seen[2] = {~0u, ~0u};                                // of the keys of a block, by their place in it
    if (masked) {
      const int left = sees - k0;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int here = min(32, max(0, left - 32 * j));
        seen[j] = (j ? there_hi : there_lo) & (here == 32 ? ~0u : (1u << here) - 1);
        const uint32_t mine = seen[j] >> (4 * lh);
#pragma unroll
        for (int e = 0; e < 16; ++e) z[j][e] = mine >> (8 * (e >> 2) + (e & 3)) & 1 ? z[j][e] : -INFINITY;
      }
    }
    auto max3 = [](float x, float y, float w) { return fmaxf(fmaxf(x, y), w); };
    float tops[NJ];                                               // as a tree of three-input maxima
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      float x[5];
#pragma unroll
      for (int k = 0; k < 5; ++k) x[k] = max3(z[j][3 * k], z[j][3 * k + 1], z[j][3 * k + 2]);
      tops[j] = max3(max3(x[0], x[1], x[2]), max3(x[3], x[4], z[j][15]), j ? tops[0] : -INFINITY);
    }
    const float top = pair_max(tops[NJ - 1]) * scale;
    // The exponent's reference of a row moves only when its largest logit has left it 2^8 behind: weights stay below 2^8 (fp16, whose reference is lower: 2^15), and rescaling is rare.
    // Each row goes by its own logits, and one that does not move is multiplied by exactly 1: no row's bits depend on the others.
    constexpr float lowered = kv_lowered<T>(8);
    const bool moves = top > (m == -INFINITY ? m : m + (8.f + lowered));
    if (__builtin_amdgcn_ballot_w64(moves)) {
      const float reference = top - lowered, keep = moves ? __builtin_amdgcn_exp2f(m - reference) : 1.f;
      l *= keep;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[b][e] *= keep;
      m = moves ? reference : m;
    }
    const float nm = m == -INFINITY ? 0.f : -m;                   // (nothing seen yet: all weights are 2^-inf)
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          z[j][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j][e], scale, nm));
          sum[e & 3] += z[j][e];
        }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int bit = 8 * (e >> 2) + (e & 3);
          struct alignas(4 * DB) Values { float f[DB]; } v = *(const Values *)(sv + (32 * j + bit) * RB + va0);
          if constexpr (careful) {
            // Values of keys that do not count are zeros; infinite and NaN ones are taken out and added to the rows that see them.
            const bool counts = (j ? there_hi : there_lo) >> (4 * lh + bit) & 1;
            const float one = (float)(seen[j] >> (4 * lh + bit) & 1);
#pragma unroll
            for (int b = 0; b < DB; ++b) {
              const float f = counts ? v.f[b] : 0.f;
              const bool finite = fabsf(f) <= 3.4028235e38f;
              v.f[b] = finite ? f : 0.f;
              if (__builtin_amdgcn_ballot_w64(!finite)) {
                f32x16 none;
#pragma unroll
                for (int i = 0; i < 16; ++i) none[i] = 0.f;
                const f32x16 us = __builtin_amdgcn_mfma_f32_32x32x2f32(!finite && !(f < 0.f) ? 1.f : 0.f, one, none, 0, 0, 0);
                const f32x16 ds = __builtin_amdgcn_mfma_f32_32x32x2f32(!finite && !(f > 0.f) ? 1.f : 0.f, one, none, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] += (us[i] > 0.f ? INFINITY : 0.f) + (ds[i] > 0.f ? -INFINITY : 0.f);
              }
            }
          }
#pragma unroll
          for (int b = 0; b < DB; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(v.f[b], z[j][e], o[b], 0, 0, 0);
        }
    } else {
    typedef typename Matrix32<T>::frag frag;
    frag p[2 * NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j][e], scale, nm));
        sum[e & 3] += w;
        p[2 * j + (e >> 3)][e & 7] = (T)w;
      }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    if constexpr (!careful) {
      typedef __attribute__((address_space(3))) const char *lchar;
      const uint32_t at = (uint32_t)(uintptr_t)(lchar)sv;
      auto products = [&](auto step) __attribute__((always_inline)) {
        constexpr int S = decltype(step)::value;
        s16x4 v[DB][2];
        read_values<DB, RB, S * 16 * RB>(at, va0, v);
#pragma unroll
        for (int b = 0; b < DB; ++b) {
          const s16x8 x = __builtin_shufflevector(v[b][0], v[b][1], 0, 1, 2, 3, 4, 5, 6, 7);
          o[b] = Matrix32<T>::mul(__builtin_bit_cast(frag, x), p[S], o[b]);
        }
      };
      products(std::integral_constant<int, 0>{});
      products(std::integral_constant<int, 1>{});
      if constexpr (NJ == 2) {
        products(std::integral_constant<int, 2>{});
        products(std::integral_constant<int, 3>{});
      }
    } else {
#pragma unroll
    for (int s = 0; s < 2 * NJ; ++s)
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        typedef __attribute__((address_space(3))) s16x4 *ltr;
        const char *va = sv + s * (16 * RB) + (va0 ^ (b << 6));
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ltr)va), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ltr)(va + 8 * RB));
        s16x8 v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        {
          // Values of keys that do not count are zeros; infinite and NaN ones are taken out and added to the rows that see them.
          const uint32_t keys = (s >> 1 ? there_hi : there_lo) >> (16 * (s & 1) + 4 * lh), mine = seen[s >> 1] >> (16 * (s & 1) + 4 * lh);
          bool odd = false;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int bit = 8 * (i >> 2) + (i & 3);
            v[i] = keys >> bit & 1 ? v[i] : (short)0;
            odd |= ((uint32_t)(uint16_t)v[i] & kv_exponent<T>()) == kv_exponent<T>();
          }
          if (__builtin_amdgcn_ballot_w64(odd)) {
            frag up, down, ones;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const short bits = v[i];
              const float f = (float)__builtin_bit_cast(T, bits);
              const bool finite = ((uint32_t)(uint16_t)v[i] & kv_exponent<T>()) != kv_exponent<T>();
              up[i] = (T)(!finite && !(f < 0.f) ? 1.f : 0.f);
              down[i] = (T)(!finite && !(f > 0.f) ? 1.f : 0.f);
              ones[i] = (T)(float)(mine >> (8 * (i >> 2) + (i & 3)) & 1);
              v[i] = finite ? v[i] : (short)0;
            }
            f32x16 none;
#pragma unroll
            for (int e = 0; e < 16; ++e) none[e] = 0.f;
            const f32x16 us = Matrix32<T>::mul(up, ones, none), ds = Matrix32<T>::mul(down, ones, none);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[b][e] += (us[e] > 0.f ? INFINITY : 0.f) + (ds[e] > 0.f ? -INFINITY : 0.f);
          }
        }
        o[b] = Matrix32<T>::mul(__builtin_bit_cast(frag, v), p[s], o[b]);
      }
    }
    }
  };

  auto run = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[b][e] = 0.f;
    m = -INFINITY;
    l = 0.f;
    int64_t next[2] = {0, 0};
    if (looks) {
      look_up(0, next);
      publish(0, next);
      look_up(1, next);
      publish(1, next);
      look_up(2, next);
    }
    __syncthreads();
    if constexpr (FORM == kPlain) {
      request(0);
    } else {
      fetch(0);
      land(0);
    }
    for (int t = 0; t < n_tiles; ++t) {
      if constexpr (FORM == kPlain) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();                                            // tile t has landed, and everybody has left tile t - 1
      if (t + 1 < n_tiles) {
        if constexpr (FORM == kPlain) request(t + 1);
        else fetch(t + 1);
      }
      if (looks) {
        publish(t + 2, next);
        look_up(t + 3, next);
      }
      if constexpr (FORM != kPlain) __builtin_amdgcn_sched_barrier(0);
      tile_step(t, careful);
      if constexpr (FORM != kPlain) {
        __builtin_amdgcn_sched_barrier(0);
        if (t + 1 < n_tiles) land(t + 1);
      }
    }
  };
  if (n_tiles > 0) {
    run(std::false_type{});
    bool odd = false;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) odd |= !(fabsf(o[b][e]) <= 3.4e38f);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (__syncthreads_or(odd)) {
      run(std::true_type{});
      __syncthreads();
    }
  } else {
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[b][e] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
  l = pair_sum(l);
  if constexpr (KP > 1) {
    // The parts of a row are joined through LDS, in the order of the wavefronts.
    constexpr int PR = DH + 4;
    float *po = (float *)lds, *pm = po + 4 * 32 * PR, *pl = pm + 4 * 32;
    static_assert((4 * 32 * PR + 8 * 32) * 4 <= flash_lds_bytes<T, DH, KP>(), "the parts fit in the stages' place");
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int at = 8 * (e >> 2) + 4 * lh + (e & 3);
        po[(wave * 32 + l32) * PR + (F32 ? DB * at + b : 32 * b + at)] = o[b][e];
      }
    if (lh == 0) {
      pm[wave * 32 + l32] = m;
      pl[wave * 32 + l32] = l;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < QT * DH / 1024; ++i) {
      const int at = threadIdx.x + 256 * i, r = at / (DH / 4), f = at % (DH / 4) * 4, first_part = (r / 32 * KP) * 32 + r % 32;
      const int row = row0 + r;
      if (row >= rows) continue;
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < KP; ++w) top = fmaxf(top, pm[first_part + 32 * w]);
      const float ref = top == -INFINITY ? 0.f : top;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KP; ++w) {
        const float mw = pm[first_part + 32 * w], take = mw == top ? 1.f : __builtin_amdgcn_exp2f(mw - ref);
        const f32x4 ow = *(const f32x4 *)(po + (first_part + 32 * w) * PR + f);
        sum += pl[first_part + 32 * w] * take;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += ow[e] * take;
      }
      const int tk = row / group, h = kvh * group + row - tk * group;
      if (SHARED || cut.parts > 1) {
        const int64_t to = balanced ? (slot * a.n_kv_heads + kvh) * QT + r : kv_part_row(a, split, (first + tk) * a.n_q_heads + h);
        *(f32x4 *)(a.parts + to * DH + f) = x;
        if (f == 0) (SHARED ? kv_shared_state(a) : kv_part_state(a, a.splits))[to] = float2{top, sum};
        continue;
      }
      const bool nothing = top == -INFINITY && sum == 0.f;        // (as below)
      const float inv = 1.f / sum;
      typedef T out4 __attribute__((ext_vector_type(4)));
      out4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = kv_round<T>(nothing ? 0.f : x[e] * inv);
      *(out4 *)(a.out.p + (first + tk) * a.out.row + h * a.out.head + f * sizeof(T)) = y;
    }
    return;
  }
  if (SHARED || cut.parts > 1) {
    if (wave_row + l32 >= rows) return;
    const int row = wave_row + l32, tk = row / group;
    const int64_t to = balanced ? (slot * a.n_kv_heads + kvh) * QT + row - row0 : kv_part_row(a, split, (first + tk) * a.n_q_heads + kvh * group + row - tk * group);
    float *po = a.parts + to * DH;
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        struct alignas(4 * DB) Values { float f[DB]; } x;
#pragma unroll
        for (int b = 0; b < DB; ++b) x.f[b] = o[b][e];
        *(Values *)(po + DB * (8 * (e >> 2) + 4 * lh + (e & 3))) = x;
      }
    } else {
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) *(f32x4 *)(po + 32 * b + 8 * i + 4 * lh) = f32x4{o[b][4 * i], o[b][4 * i + 1], o[b][4 * i + 2], o[b][4 * i + 3]};
    }
    if (lh == 0) (SHARED ? kv_shared_state(a) : kv_part_state(a, a.splits))[to] = float2{m, l};
    return;
  }
  // A row whose logits are all -infinity has zeros, though its weights of zero may have met infinite values or NaN.  (NaN logits leave l NaN.)  That is for the whole row to say: parts keep what they have
  // met, as a row with a logit above -infinity in another part is NaN where it sees one.
  const bool nothing = m == -INFINITY && l == 0.f;
  const float inv = 1.f / l;
  // Rows to memory: each wavefront turns its 32 x DH patch in LDS, 16-byte chunks XORed with the row.
  char *patch = lds + wave * (32 * RB);
  static_assert(KP > 1 || 4 * 32 * RB <= 2 * STAGE, "the patches fit in the stages");
  if constexpr (F32) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      // features DB m..DB m + DB - 1 of row l32, m = 8 (e / 4) + 4 lh + e % 4
      const int at = (8 * (e >> 2) + 4 * lh + (e & 3)) * DB * 4;
      struct alignas(4 * DB) Values { float f[DB]; } x;
#pragma unroll
      for (int b = 0; b < DB; ++b) x.f[b] = nothing ? 0.f : o[b][e] * inv;
      *(Values *)(patch + l32 * RB + (((at >> 4) ^ (l32 & (CH - 1))) << 4) + (at & 15)) = x;
    }
  } else {
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // features 32 b + 8 i + 4 lh + 0..3 of row l32
        s16x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __builtin_bit_cast(short, kv_round<T>(nothing ? 0.f : o[b][4 * i + e] * inv));
        *(s16x4 *)(patch + l32 * RB + (((4 * b + i) ^ (l32 & (CH - 1))) << 4) + lh * 8) = x;
      }
  }
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < 32 / RPI; ++i) {
    const int r = i * RPI + in_row, row = wave_row + r;
    if (row < rows) {
      const int tk = row / group, h = kvh * group + row - tk * group;
      *(word4 *)(a.out.p + (first + tk) * a.out.row + h * a.out.head + chunk * 16) = *(const word4 *)(patch + r * RB + ((chunk ^ (r & (CH - 1))) << 4));
    }
  }
}

template <typename T, int DH, bool PAGED, int KP, int FORM>
__global__ __launch_bounds__(256, (flash_workgroups<T, DH, KP>())) void kv_flash_kernel(KvAttention a) {
  flash_rows<T, DH, PAGED, KP, FORM, false>(a, blockIdx.x, gridDim.x);
}

// Adds up the parts of rows whose keys were cut, in the order of the keys.  DH / 4 lanes a head, and a workgroup 256 / (DH / 4) heads of a token, so that all loads of a lane are in
// flight at once (128 new tokens, 32 heads of 128, 16 parts: 9.6 us; with a workgroup per token, and the parts one after another, 25).
template <typename T, int DH, int KP>
__global__ __launch_bounds__(256) void kv_flash_join_kernel(KvAttention a) {
  constexpr int KW = KP * key_block<T, DH, KP>(), QT = kFlashRows / KP;
  constexpr int H = 256 / (DH / 4);                               // heads of a workgroup
  const int blocks = (a.n_q_heads + H - 1) / H;
  const int64_t q_row = blockIdx.x / blocks;
  const int head = blockIdx.x % blocks * H + threadIdx.x / (DH / 4), f = threadIdx.x % (DH / 4) * 4;
  const int seq = kv_find_sequence(a.batch.offsets, a.batch.n_seqs, q_row, threadIdx.x & 63);
  if (seq >= a.batch.n_seqs || head >= a.n_q_heads) return;
  const int64_t first = a.batch.offsets[seq], end = a.batch.offsets[seq + 1];
  if (first < 0 || q_row < first || q_row >= end) return;
  const int group = a.n_q_heads / a.n_kv_heads, n = kv_clip(a.batch.kv_lens[seq], a.pages.capacity);
  const int rows = (int)(min(end, a.batch.n_rows) - first) * group;
  const int64_t back = n - (end - first);
  const int row = (int)(q_row - first) * group + head % group;
  const int last = min(row / QT * QT + QT, rows) - 1;             // of the row's tile
  const int parts = flash_parts<KW>((int)max((int64_t)0, back + last / group + 1), a.splits).parts;
  if (parts == 1) return;
  const int64_t step = a.batch.n_rows * a.n_q_heads, from = q_row * a.n_q_heads + head;
  const float2 *state = kv_part_state(a, a.splits) + from;
  const float *sums = a.parts + from * DH + f;
  float m = -INFINITY, l = 0.f;
#pragma unroll 8
  for (int p = 0; p < parts; ++p) m = fmaxf(m, state[p * step].x);
  const float ref = m == -INFINITY ? 0.f : m;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int p = 0; p < parts; ++p) {
    const float2 ml = state[p * step];
    const f32x4 x = *(const f32x4 *)(sums + p * step * DH);
    const float take = ml.x == m ? 1.f : __builtin_amdgcn_exp2f(ml.x - ref);
    l += ml.y * take;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += x[e] * take;
  }
  const bool nothing = m == -INFINITY && l == 0.f;                // (see flash_rows)
  const float inv = 1.f / l;
  typedef T out4 __attribute__((ext_vector_type(4)));
  out4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = kv_round<T>(nothing ? 0.f : o[e] * inv);
  *(out4 *)(a.out.p + q_row * a.out.row + head * a.out.head + f * sizeof(T)) = y;
}

template <typename T, int DH, bool PAGED, int KP, int FORM> hipError_t launch_flash(const KvAttention &a, hipStream_t stream) {
  static std::atomic<uint64_t> raised{0};
  constexpr int kBytes = flash_lds_bytes<T, DH, KP>();
  const hipError_t e = raise_lds_limit(reinterpret_cast<const void *>(&kv_flash_kernel<T, DH, PAGED, KP, FORM>), kBytes, raised);
  if (e != hipSuccess) return e;
  const int64_t slots = a.batch.n_rows * (a.n_q_heads / a.n_kv_heads) / (kFlashRows / KP) + a.batch.n_seqs;
  kv_flash_kernel<T, DH, PAGED, KP, FORM><<<(unsigned)(slots * a.n_kv_heads * a.splits), 256, kBytes, stream>>>(a);
  if (a.splits > 1) kv_flash_join_kernel<T, DH, KP><<<(unsigned)(a.batch.n_rows * ((a.n_q_heads * (DH / 4) + 255) / 256)), 256, 0, stream>>>(a);
  return hipGetLastError();
}

// F is called with the call's element type, width and wavefronts per 32 rows.
template <typename F> void flash_with_shape(const KvAttention &a, int wavefronts, F f) {
  kv_with_type(a.dtype, [&](auto t) {
    using T = decltype(t);
    kv_with_width(a.head_dim, [&](auto width) {
      if (wavefronts == 1) f(t, width, std::integral_constant<int, 1>{});
      if (wavefronts == 2) f(t, width, std::integral_constant<int, 2>{});
      if constexpr (decltype(width)::value * sizeof(T) < 512)     // (LDS has no room for four wavefronts' tiles of wider rows)
        if (wavefronts == 4) f(t, width, std::integral_constant<int, 4>{});
    });
  });
}

}  // namespace

}  // namespace flame
