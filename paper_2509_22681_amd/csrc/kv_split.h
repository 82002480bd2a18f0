// Softmax attention of few query rows over long paged caches: the work is split over the keys and joined.
//
// Bound by memory: a sequence's keys and values are read once, 2 n Hkv D values, and each takes part in 4 G operations per query token
// (G query heads share a key head), far below what the matrix pipe does in that time.  So everything serves the loads:
//   - A unit is a block of 16 query rows of one sequence and key head (row = token * G + head of the group; a decoding step
//     with G <= 16 has one unit per key head, whose keys and values are then read once), and a tile 32 of its keys (16 in fp32).  The tiles of all units form one
//     line, which a fixed number of wavefronts cuts into equal parts: every wavefront streams the same number of bytes whatever the lengths of the sequences, one long sequence fills the chip,
//     and nothing depends on the host knowing the lengths.  A wavefront works alone: no barriers, no LDS traffic but for the
//     row offsets.
//   - Keys and values go from memory straight into the registers of the matrix operands, one tile ahead of the arithmetic (16 KB
//     in flight per wavefront at D = 128).  Products are transposed, S^T[key][row] = K Q^T and O^T[feature][row] += V^T P^T.  With the keys of two 16-row blocks dealt out as
//     8 (m / 4) + m % 4 and 4 more, the weights that a lane gets from the first product are those of keys 8 g..8 g + 7 (g = lane / 16), which is
//     what the second product wants from it; and a lane that reads D/16 features of these eight keys holds the A operand of the second product up to a
//     transposition within its own registers (byte permutes of word pairs), feature D/16 * m + j in product j.
// 64 ragged sequences of 100..8192 tokens (32/8 heads of 128, bf16) read 1.13 GB in 220 us, 5.1 TB/s, and their join takes 5; three of 60000..131072 (32/4 heads) 731 MB in 148 and 7.
// A unit that ends within its wavefront is written; the others leave maximum, sum and unnormalised rows in the workspace, for a second kernel that
// adds up a unit's parts in the order of their keys.  Every part and every join has a fixed order: the same call gives the same bits.
//
// Over a cache of 8 or 4 bits the loads are codes, half or a quarter of the bytes, with a scale byte for each lane's piece of a row; they become operands in the registers, two features an instruction,
// ahead of the products (features are dealt out to a lane so that its codes of a key lie side by side: any order will do for the first product if queries have the same).  With shared histories
// (SHARED) a unit's keys are the sequence's own alone, those from prefix_lens[b] on, and all units leave parts, whole ones in a plane of the row tiles' parts (kv_flash.h).
#pragma once
#include <algorithm>

#include "kv_codec.h"

namespace flame {

namespace {

// Wavefronts per SIMD, as their registers allow, and in all.  Two tiles of values in flight fill the registers: 128 features spill 10 of 256 (44 bytes a lane; fp32 13, 56), and scalars go to lanes of
// others (some 350 of 128 features in 16 bits, fewer in the rest).  Decoding of many keys runs at
// memory speed all the same.  Codes take less: none of their kernels spills vectors (128 features, 16 bits: f8 199 registers, f4 169).
constexpr int split_occupancy(int dh) { return dh == 128 ? 2 : dh == 64 ? 3 : 4; }
constexpr int split_workers(int dh) { return 1024 * split_occupancy(dh); }
constexpr int kRows = 16;           // query rows of a unit

template <typename T, int DH, int FORM> struct SplitShape {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int KT = F32 ? 16 : 32;          // keys of a tile
  static constexpr int VF = DH / 16;                // features of a lane in the second product
  // of stored codes: features of a piece that a lane loads of a key's row, pieces, and bytes of one
  static constexpr int PF = FORM == kF4 && DH == 128 ? 32 : DH == 32 ? 8 : 16, NP = DH / 4 / PF, PB = FORM == kF4 ? PF / 2 : PF;
};
template <int BYTES> struct SplitWords {            // a lane's load
  static constexpr int N = (BYTES + 3) / 4;
  uint32_t w[N];
  __device__ __forceinline__ void load(const char *p) {
    if constexpr (BYTES >= 4) {
      struct alignas(BYTES) Words { uint32_t w[N]; };
      const Words y = *(const Words *)p;
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = y.w[i];
    } else if constexpr (BYTES == 2) {
      w[0] = *(const uint16_t *)p;
    } else {
      w[0] = *(const uint8_t *)p;
    }
  }
};

// What a wavefront knows of a sequence.
struct SplitSeq {
  int first;          // its first query row
  int rows, blocks;   // query rows times G, and units per key head
  int n, back;        // keys; keys that the row before the first one would see
  int tiles;          // of one unit
  bool wrong;         // offsets that are none
  int skip;           // shared keys ahead of its own
};

template <int KT, bool SHARED> __device__ __forceinline__ SplitSeq split_sequence(const KvAttention &a, int b, bool report) {
  SplitSeq s;
  s.n = kv_clip_length(a.batch.kv_lens[b], a.pages.capacity, a.batch.faults, report);
  s.skip = SHARED ? kv_clip_length(a.prefix_lens[b], a.pages.capacity, a.batch.faults, report) : 0;
  int64_t m = 1, full = 1;
  s.first = b;
  s.wrong = false;
  if (a.batch.offsets) {
    const int64_t first = a.batch.offsets[b], end = a.batch.offsets[b + 1];
    s.first = (int)first;
    full = end - first;
    s.wrong = kv_wrong_offsets(first, end);
    if (report) kv_report_offsets(first, end, a.batch.n_rows, a.batch.faults);
    m = s.wrong ? 0 : max((int64_t)0, min(full, a.batch.n_rows - first));
  }
  const int group = a.n_q_heads / a.n_kv_heads;
  s.back = (int)max(s.n - full - s.skip, -((int64_t)1 << 30));
  if constexpr (SHARED) s.n = max(0, s.n - s.skip);
  s.rows = (int)(m * group);                        // (rows times heads is below 2^25)
  s.blocks = (s.rows + kRows - 1) / kRows;
  s.tiles = s.rows ? max(1, (s.n + KT - 1) / KT) : 0;   // (a unit without keys writes zeros)
  return s;
}

// Of up to 64 sequences each lane keeps one; of more they are read again.
template <bool SHARED> __device__ __forceinline__ SplitSeq split_from_lane(const SplitSeq &s, int lane) {
  return SplitSeq{__builtin_amdgcn_readlane(s.first, lane), __builtin_amdgcn_readlane(s.rows, lane), __builtin_amdgcn_readlane(s.blocks, lane),
                  __builtin_amdgcn_readlane(s.n, lane), __builtin_amdgcn_readlane(s.back, lane), __builtin_amdgcn_readlane(s.tiles, lane), false,
                  SHARED ? __builtin_amdgcn_readlane(s.skip, lane) : 0};
}

__device__ __forceinline__ int64_t split_scan(int64_t v) {        // inclusive sums over the wavefront
  const auto step = [&](auto moved) { v += moved; };
  const auto dpp = [&](auto ctrl, auto mask) {
    const int lo = __builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(mask)::value, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), decltype(ctrl)::value, decltype(mask)::value, 0xf, false);
    return (int64_t)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo);
  };
  step(dpp(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{}));   // row_shr:1
  step(dpp(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{}));
  step(dpp(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{}));
  step(dpp(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{}));
  step(dpp(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{}));   // the last lane of a row to the next row
  step(dpp(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{}));   // lane 31 to the upper half
  return v;
}

__device__ __forceinline__ int64_t split_lane(int64_t v, int lane) {
  return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)v, lane));
}

// Tiles of all units, and of those the sequence that holds tile `at` (at < 0: not asked) with its first tile.  at >= total: sequence n_seqs.
struct SplitPlace {
  int64_t total, first_tile;
  int seq;
  SplitSeq mine;      // the lane's sequence, of up to 64
};

template <int KT, bool SHARED, typename F> __device__ __forceinline__ SplitPlace split_find(const KvAttention &a, int lane, int heads, bool reports, F target) {
  SplitPlace p{0, 0, a.batch.n_seqs, SplitSeq{}};
  int lo = 0, n = a.batch.n_seqs;
  int64_t base = 0, at = 0;
  for (bool top = true;; top = false) {
    // lane i: the tiles of `chunk` sequences from lo + i chunk on, of one sequence in the end
    const bool report = top && reports && threadIdx.x < 64;
    int64_t mine = 0;
    int chunk = 1;
    if (n <= 64) {
      if (lane < n) {
        const SplitSeq s = split_sequence<KT, SHARED>(a, lo + lane, report);
        mine = (int64_t)s.blocks * s.tiles;
        if (top) p.mine = s;
      }
      if (top && a.batch.offsets) {
        const uint64_t wrong = __builtin_amdgcn_ballot_w64(p.mine.wrong);
        if (wrong && lane >= __builtin_ctzll(wrong)) mine = p.mine.rows = p.mine.blocks = p.mine.tiles = 0;
      }
    } else {
      // the wavefront reads 64 neighbours at a time
      chunk = (n + 4095) / 4096 * 64;
      for (int i = 0; i * chunk < n; ++i) {
        int64_t sum = 0;
        for (int k = lane; k < chunk; k += 64) {
          if (i * chunk + k >= n) break;
          const SplitSeq s = split_sequence<KT, SHARED>(a, lo + i * chunk + k, report);
          sum += (int64_t)s.blocks * s.tiles;
        }
        const int64_t all = split_lane(split_scan(sum), 63);
        if (lane == i) mine = all;
      }
    }
    mine *= heads;
    const int64_t sums = split_scan(mine);
    if (top) {
      p.total = split_lane(sums, 63);
      at = target(p.total);
      if (at >= p.total) return p;
    }
    const uint64_t beyond = __builtin_amdgcn_ballot_w64(base + sums > at);
    if (!beyond) return p;                            // (only if the lengths changed under the call)
    const int l = __builtin_ctzll(beyond);
    base += split_lane(sums, l) - split_lane(mine, l);
    lo += l * chunk;
    n = min(chunk, n - l * chunk);
    if (chunk == 1) {
      p.seq = lo;
      p.first_tile = base;
      return p;
    }
  }
}

// Parts of a worker: the one it begins with, and one that goes on behind its end.
constexpr int split_part_floats(int dh) { return kRows * dh + 2 * kRows; }
// The workspace: the parts [workers][2], and behind them for every output row which workers have its parts (the first one twice, plus 1 if its part there is the second; the last one).
constexpr int64_t split_parts_floats(int dh) { return (int64_t)split_workers(dh) * 2 * split_part_floats(dh); }

__device__ __forceinline__ float split_max(float v) {             // over the four lanes that share a query row
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float split_sum(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// VF features of a lane from their codes, as words of the element type.
template <typename T, int FORM, int VF, int J = 0> __device__ __forceinline__ void split_values(const uint32_t *codes, float scale, uint32_t *v) {
  const auto y = KvPair<T>::template get<FORM, FORM == kF8 ? J & 1 : J>(codes[FORM == kF8 ? J >> 1 : 0], scale);
  if constexpr (sizeof(T) == 4) {
    v[2 * J] = __float_as_uint(y[0]);
    v[2 * J + 1] = __float_as_uint(y[1]);
  } else {
    v[J] = __builtin_bit_cast(uint32_t, y);
  }
  if constexpr (2 * J + 2 < VF) split_values<T, FORM, VF, J + 1>(codes, scale, v);
}

template <typename T> struct Matrix16;
template <> struct Matrix16<bf16_t> {
  typedef bf16x8 frag;
  static __device__ __forceinline__ f32x4 mul(frag x, frag y, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0); }
};
template <> struct Matrix16<half_t> {
  typedef f16x8 frag;
  static __device__ __forceinline__ f32x4 mul(frag x, frag y, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0); }
};

// (kv_shared.h runs this beside row tiles in one launch: block `my_block` of its own, `workers` wavefronts in all.)
template <typename T, int DH, int FORM, bool SHARED>
__device__ __forceinline__ void split_units(const KvAttention &a, float *__restrict__ parts, unsigned my_block, int workers) {
  typedef SplitShape<T, DH, FORM> S;
  constexpr int KT = S::KT, VF = S::VF;
  constexpr bool F32 = S::F32;
  constexpr int KB = KT / 16;                                     // 16-key blocks of a tile
  constexpr int KS = DH * (int)sizeof(T) / 64;                    // 64-byte steps of a key row: 16 bytes per lane each
  constexpr int VK = KT / 4;                                      // keys of a lane in the second product
  constexpr int VB = VF * (int)sizeof(T);                         // bytes of a lane per value row: 4..32
  constexpr int VW = VB / 4;
  typedef uint32_t word4 __attribute__((ext_vector_type(4)));
  __shared__ int64_t offset_s[4][2][KT];
  __shared__ __attribute__((aligned(16))) uint32_t scale_s[4][FORM == kPlain ? 1 : 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  // Codes of a token's heads lie side by side where its page is laid out token by token, several heads to a line of the caches, and so do scales.  So of codes, up to four wavefronts of a workgroup take the
  // same tiles of neighbouring heads: `together` of them share a stretch of the line, which is shorter by as much.  Storage for parts goes by head first, so that a head's parts are neighbours.
  const int together = FORM == kPlain ? 1 : a.n_kv_heads % 4 == 0 ? 4 : a.n_kv_heads % 2 == 0 ? 2 : 1;
  const int stretches = workers / together, stretch = FORM == kPlain ? my_block * 4 + wave : my_block * (4 / together) + wave / together;
  const int my_head = FORM == kPlain ? 0 : wave % together, worker = FORM == kPlain ? stretch : my_head * stretches + stretch;
  const int heads = FORM == kPlain ? a.n_kv_heads : a.n_kv_heads / together;
  int64_t per = 0;
  SplitPlace place = split_find<KT, SHARED>(a, lane, heads, my_block == 0, [&](int64_t total) {
    per = (total + stretches - 1) / stretches;
    return (int64_t)stretch * per;
  });
  int64_t tile = (int64_t)stretch * per;                          // on the line of all tiles
  const int64_t tile_end = min(tile + per, place.total);
  const float scale = a.scale * kLog2e;
  const int group = a.n_q_heads / a.n_kv_heads;
  int seq = place.seq;
  int64_t seq_tile = place.first_tile;
  bool begins = true;                                             // the unit is the worker's first
  while (tile < tile_end && seq < a.batch.n_seqs) {
    const SplitSeq s = a.batch.n_seqs <= 64 ? split_from_lane<SHARED>(place.mine, seq) : split_sequence<KT, SHARED>(a, seq, false);
    int64_t in_seq = tile - seq_tile;
    const int64_t seq_tiles = (int64_t)heads * s.blocks * s.tiles;
    if (in_seq >= seq_tiles) {                                    // (sequences without rows have none)
      seq_tile += seq_tiles;
      ++seq;
      continue;
    }
    const int unit = (int)(in_seq / s.tiles), t0 = (int)(in_seq - (int64_t)unit * s.tiles);
    const int t1 = (int)min((int64_t)s.tiles, t0 + (tile_end - tile));
    const int head_group = unit / s.blocks, block = unit - head_group * s.blocks, kvh = FORM == kPlain ? head_group : head_group * together + my_head;
    const int32_t *table = a.pages.table + seq * a.pages.table_stride;
    const char *kp = a.pages.k + kvh * a.pages.head, *vp = a.pages.v + kvh * a.pages.head;
    // my query row (the column of the accumulators), and the keys it sees
    const int row = block * kRows + l16;
    const bool row_there = row < s.rows;
    const int token = (row_there ? row : block * kRows) / group, head = kvh * group + (row_there ? row : block * kRows) - token * group;
    const int sees = s.back + token + 1;
    const int sees_least = s.back + block * kRows / group + 1;    // of the block's first row
    word4 fq[KS];
    {
      const char *q = a.q.p + (s.first + token) * a.q.row + head * a.q.head;
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        constexpr int SF = 16 / sizeof(T);                        // features of a step, of which a piece has PF / SF
        const int at = FORM == kPlain ? i * 64 + g * 16 : ((i / (S::PF / SF) * 4 + g) * S::PF + i % (S::PF / SF) * SF) * (int)sizeof(T);
        fq[i] = *(const word4 *)(q + at);
      }
    }
    f32x4 o[VF];
#pragma unroll
    for (int j = 0; j < VF; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    const char *scales_of_lane = (lane < 32 ? a.v_scales : a.k_scales) + (FORM == kPlain ? 0 : kvh * a.pages.head >> kv_scale_shift<FORM>());

    // Row offsets of a tile: key k by lane k; keys behind the last one repeat it, keys in pages that the table does not name get the pool's first row, and neither counts.
    auto look_up = [&](int t) -> int64_t {
      const int key = min(t * KT + (lane & (KT - 1)), s.n - 1);
      return key < 0 ? -1 : kv_token_offset(a.pages, table, (uint32_t)key + (SHARED ? s.skip : 0));
    };
    // The same in two steps: which page, and, once that is there, where.
    struct Page { int32_t page; uint32_t slot; };
    auto page_of = [&](int t) -> Page {
      const int key = min(t * KT + (lane & (KT - 1)), s.n - 1);
      const uint32_t token = (uint32_t)max(key, 0) + (SHARED ? s.skip : 0), i = kv_page_index(a.pages, token);
      return Page{table[i], token - i * (uint32_t)a.pages.page_size};
    };
    auto place_of = [&](const Page &p) -> int64_t { return (uint32_t)p.page < (uint32_t)a.pages.n_pages ? p.page * a.pages.page + (int64_t)p.slot * a.pages.slot : -1; };
    struct Values {
      word4 k[KB][KS];
      uint32_t v[VK][VW];
    };
    struct Codes {
      SplitWords<S::PB> kc[KB][S::NP];
      SplitWords<kv_row_bytes<T, FORM>(VF)> vc[VK];
      uint32_t scales;                                            // of key lane % KT: of its value in the lower half of the wavefront, else of the key itself
    };
    struct Tile : std::conditional_t<FORM == kPlain, Values, Codes> {
      uint64_t there;                                             // lanes' keys that count
    };
    auto request = [&](Tile &x, int t, int64_t offset) {
      if (offset < 0 && s.n > 0 && lane < KT) kv_fault(a.batch.faults, FLAME_KV_FAULT_PAGE);
      x.there = __builtin_amdgcn_ballot_w64(offset >= 0 && t * KT + (lane & (KT - 1)) < s.n);
      int64_t *at = offset_s[wave][t & 1];
      if (lane < KT) at[lane] = max(offset, (int64_t)0);
      __builtin_amdgcn_wave_barrier();
      if constexpr (FORM != kPlain) {
        const char *k_at = kp + g * S::PB, *v_at = vp + l16 * kv_row_bytes<T, FORM>(VF);
#pragma unroll
        for (int b = 0; b < KB; ++b) {
          const char *row_at = k_at + at[F32 ? l16 : 8 * (l16 >> 2) + 4 * b + (l16 & 3)];
#pragma unroll
          for (int p = 0; p < S::NP; ++p) x.kc[b][p].load(row_at + p * 4 * S::PB);
        }
#pragma unroll
        for (int i = 0; i < VK; ++i) x.vc[i].load(v_at + at[VK * g + i]);
        SplitWords<DH / 32> w;
        w.load(scales_of_lane + (max(offset, (int64_t)0) >> kv_scale_shift<FORM>()));
        x.scales = w.w[0];
      } else {
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        const char *row_at = kp + at[F32 ? l16 : 8 * (l16 >> 2) + 4 * b + (l16 & 3)];
#pragma unroll
        for (int i = 0; i < KS; ++i) x.k[b][i] = *(const word4 *)(row_at + i * 64 + g * 16);
      }
#pragma unroll
      for (int i = 0; i < VK; ++i) {
        const char *row_at = vp + at[VK * g + i];
        if constexpr (VB == 32) {
          // fp32, 128 features: lanes side by side take 16 bytes each of either half
          const word4 x0 = *(const word4 *)(row_at + l16 * 16), x1 = *(const word4 *)(row_at + 256 + l16 * 16);
#pragma unroll
          for (int w = 0; w < 4; ++w) { x.v[i][w] = x0[w]; x.v[i][4 + w] = x1[w]; }
        } else {
          struct alignas(VB) Words { uint32_t w[VW]; };
          const Words y = *(const Words *)(row_at + l16 * VB);
#pragma unroll
          for (int w = 0; w < VW; ++w) x.v[i][w] = y.w[w];
        }
      }
      }
    };
    auto add = [&](Tile &loaded, int t) {
      Values made;
      if constexpr (FORM != kPlain) {
        typedef typename KvPair<T>::vec pair;
        constexpr int W8 = FORM == kF8 ? 2 : 1, KE = F32 ? 2 : 1;       // words of eight features' codes, steps that they make
        scale_s[wave][lane] = loaded.scales;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int e = 0; e < DH / 32; ++e) {
            const int p = e / (S::PF / 8), sub = e % (S::PF / 8);
            pair y[4];
            const uint32_t scales = scale_s[wave][32 + (F32 ? l16 : 8 * (l16 >> 2) + 4 * b + (l16 & 3))];
            kv_eight<T, FORM>(loaded.kc[b][p].w + sub * W8, kv_scale_of(scales, (p * 4 + g) * S::PF / 32), y);
            if constexpr (F32) {
              made.k[b][KE * e] = word4{__float_as_uint(y[0][0]), __float_as_uint(y[0][1]), __float_as_uint(y[1][0]), __float_as_uint(y[1][1])};
              made.k[b][KE * e + 1] = word4{__float_as_uint(y[2][0]), __float_as_uint(y[2][1]), __float_as_uint(y[3][0]), __float_as_uint(y[3][1])};
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) made.k[b][e][i] = __builtin_bit_cast(uint32_t, y[i]);
            }
          }
      }
      Values &x = [&]() -> Values & { if constexpr (FORM == kPlain) return loaded; else return made; }();
      const uint64_t there = loaded.there;
      f32x4 z[KB];
#pragma unroll
      for (int b = 0; b < KB; ++b) z[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KS; ++i)
#pragma unroll
        for (int b = 0; b < KB; ++b) {
          if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) z[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.k[b][i][j]), __uint_as_float(fq[i][j]), z[b], 0, 0, 0);
          } else {
            typedef typename Matrix16<T>::frag frag;
            z[b] = Matrix16<T>::mul(__builtin_bit_cast(frag, x.k[b][i]), __builtin_bit_cast(frag, fq[i]), z[b]);
          }
        }
      // element e of block b: key VK g + 4 b + e of the tile
      const int k0 = t * KT + VK * g;
      const uint32_t here = (uint32_t)(there >> (VK * g)) & ((1u << VK) - 1);                       // of my VK keys those that count,
      const uint32_t seen = here & ((1u << max(0, min(VK, sees - k0))) - 1);                         // and those of them that my row sees
      const bool masked = there != ~0ull || t * KT + KT > sees_least;
      float w[VK];
#pragma unroll
      for (int i = 0; i < VK; ++i) w[i] = z[i >> 2][i & 3] * scale;
      if (masked) {
#pragma unroll
        for (int i = 0; i < VK; ++i) w[i] = seen >> i & 1 ? w[i] : -INFINITY;
      }
      float top = w[0];
#pragma unroll
      for (int i = 1; i < VK; ++i) top = fmaxf(top, w[i]);
      const float m_new = fmaxf(m, split_max(top) - kv_lowered<T>(0));   // the reference of the exponents
      const float m_at = m_new == -INFINITY ? 0.f : m_new;       // (nothing seen yet: all weights are 2^-inf)
      // (codes: without the branch, around which the compiler copies all sums: 32 products in place of 50 moves a tile of 128 features)
      if (FORM != kPlain || __builtin_amdgcn_ballot_w64(m_new != m)) {
        const float keep = m == m_new ? 1.f : __builtin_amdgcn_exp2f(m - m_at);
        l *= keep;
#pragma unroll
        for (int j = 0; j < VF; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[j][e] *= keep;
        m = m_new;
      }
#pragma unroll
      for (int i = 0; i < VK; ++i) {
        w[i] = __builtin_amdgcn_exp2f(w[i] - m_at);
        l += w[i];
      }
      if constexpr (FORM != kPlain) {
        float vs[VK];
#pragma unroll
        for (int i = 0; i < VK; ++i) vs[i] = kv_scale_of(scale_s[wave][VK * g + i], l16 * VF / 32);
        if (masked) {
          // Codes of keys that do not count are zeros, and a block that is NaN, which a row that does not see it must not meet in a product, is taken out and added to the rows that do see it.  (A lane's
          // features are of one block.)
          constexpr float kNone = INFINITY;                             // (the bits of scale byte 255)
          const auto take_out = [&](int i) {
            vs[i] = 0.f;
#pragma unroll
            for (int n = 0; n < loaded.vc[i].N; ++n) loaded.vc[i].w[n] = 0;
          };
          bool odd = false;
#pragma unroll
          for (int i = 0; i < VK; ++i) {
            if (!(here >> i & 1)) take_out(i);
            odd |= vs[i] == kNone;
          }
          if (__builtin_amdgcn_ballot_w64(odd)) {
            f32x4 nans = {0.f, 0.f, 0.f, 0.f};
            if constexpr (F32) {
#pragma unroll
              for (int i = 0; i < VK; ++i) nans = __builtin_amdgcn_mfma_f32_16x16x4f32(vs[i] == kNone ? 1.f : 0.f, (float)(seen >> i & 1), nans, 0, 0, 0);
            } else {
              typename Matrix16<T>::frag of, ones;
#pragma unroll
              for (int i = 0; i < VK; ++i) {
                of[i] = (T)(vs[i] == kNone ? 1.f : 0.f);
                ones[i] = (T)(float)(seen >> i & 1);
              }
              nans = Matrix16<T>::mul(of, ones, nans);
            }
#pragma unroll
            for (int j = 0; j < VF; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[j][e] += nans[e] > 0.f ? NAN : 0.f;
#pragma unroll
            for (int i = 0; i < VK; ++i)
              if (vs[i] == kNone) take_out(i);
          }
        }
#pragma unroll
        for (int i = 0; i < VK; ++i) split_values<T, FORM, VF>(loaded.vc[i].w, vs[i], x.v[i]);
      } else if (masked) {
        // Values of keys that do not count are zeros, and infinite or NaN ones, which a row that does not see them must not meet in a product, are taken out and
        // added to the rows that do see them.
        bool odd = false;
#pragma unroll
        for (int i = 0; i < VK; ++i)
#pragma unroll
          for (int n = 0; n < VW; ++n) {
            x.v[i][n] = here >> i & 1 ? x.v[i][n] : 0u;
            odd |= not_finite<T>(x.v[i][n]);
          }
        if (__builtin_amdgcn_ballot_w64(odd)) {
          const f32x4 none = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < VF; ++j) {
            f32x4 up = none, down = none;
            if constexpr (F32) {
#pragma unroll
              for (int i = 0; i < VK; ++i) {
                const float v = __uint_as_float(x.v[i][j]), one = (float)(seen >> i & 1);
                up = __builtin_amdgcn_mfma_f32_16x16x4f32(v != v || v == INFINITY ? 1.f : 0.f, one, up, 0, 0, 0);
                down = __builtin_amdgcn_mfma_f32_16x16x4f32(v != v || v == -INFINITY ? 1.f : 0.f, one, down, 0, 0, 0);
              }
            } else {
              typename Matrix16<T>::frag u, d, ones;
#pragma unroll
              for (int i = 0; i < VK; ++i) {
                const float v = (float)__builtin_bit_cast(T, (uint16_t)(x.v[i][j >> 1] >> (16 * (j & 1))));
                u[i] = (T)(v != v || v == INFINITY ? 1.f : 0.f);
                d[i] = (T)(v != v || v == -INFINITY ? 1.f : 0.f);
                ones[i] = (T)(float)(seen >> i & 1);
              }
              up = Matrix16<T>::mul(u, ones, none);
              down = Matrix16<T>::mul(d, ones, none);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) o[j][e] += (up[e] > 0.f ? INFINITY : 0.f) + (down[e] > 0.f ? -INFINITY : 0.f);
          }
#pragma unroll
          for (int i = 0; i < VK; ++i)
#pragma unroll
            for (int n = 0; n < VW; ++n) x.v[i][n] = only_finite<T>(x.v[i][n]);
        }
      }
      if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < VK; ++i)
#pragma unroll
          for (int j = 0; j < VF; ++j) o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.v[i][j]), w[i], o[j], 0, 0, 0);
      } else {
        typedef typename Matrix16<T>::frag frag;
        frag p;
#pragma unroll
        for (int i = 0; i < VK; ++i) p[i] = (T)w[i];
#pragma unroll
        for (int j = 0; j < VF; ++j) {
          // feature VF l16 + j of keys VK g..VK g + 7: the lower or upper halves of word j / 2 of the eight rows
          word4 f;
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_perm(x.v[2 * i + 1][j >> 1], x.v[2 * i][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
          o[j] = Matrix16<T>::mul(__builtin_bit_cast(frag, f), p, o[j]);
        }
      }
    };
    if (s.n > 0) {
      Tile x, y;
      if constexpr (FORM != kPlain || SHARED) {
        // Loads return in order: a page that is asked for ahead of a tile's loads is known while those are still on their way, and the next tile's can follow them (f4, three long sequences 58.8 -> 52.0 us;
        // 64 ragged ones 87 -> 80, f8 123 -> 119; a third tile in registers: 53.7, 81.7, 121).
        Page next = page_of(t0);
        Page after = page_of(min(t0 + 1, t1 - 1));
        request(x, t0, place_of(next));
        next = after;
#pragma unroll 1
        for (int t = t0; t < t1; t += 2) {
          after = page_of(min(t + 2, t1 - 1));
          __builtin_amdgcn_sched_barrier(0);
          request(y, min(t + 1, t1 - 1), place_of(next));
          __builtin_amdgcn_sched_barrier(0);
          add(x, t);
          __builtin_amdgcn_sched_barrier(0);
          if (t + 1 >= t1) break;
          next = page_of(min(t + 3, t1 - 1));
          __builtin_amdgcn_sched_barrier(0);
          request(x, min(t + 2, t1 - 1), place_of(after));
          __builtin_amdgcn_sched_barrier(0);
          add(y, t + 1);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
      request(x, t0, look_up(t0));
      int64_t next = look_up(min(t0 + 1, t1 - 1));
#pragma unroll 1
      for (int t = t0; t < t1; t += 2) {
        request(y, min(t + 1, t1 - 1), next);
        next = look_up(min(t + 2, t1 - 1));
        __builtin_amdgcn_sched_barrier(0);
        add(x, t);
        __builtin_amdgcn_sched_barrier(0);
        if (t + 1 >= t1) break;
        request(x, min(t + 2, t1 - 1), next);
        next = look_up(min(t + 3, t1 - 1));
        __builtin_amdgcn_sched_barrier(0);
        add(y, t + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      }
    }
    l = split_sum(l);
    if (t0 == 0 && row_there && g == 0) {
      const int last = t1 == s.tiles ? worker : (int)((tile + s.tiles - 1) / per) + (worker - stretch);
      ((int2 *)(parts + split_parts_floats(DH)))[(int64_t)(s.first + token) * a.n_q_heads + head] = int2{2 * worker + !begins, last};
    }
    // accumulator element e of product j: feature VF (4 g + e) + j of my row (plain fp32 with 128 features: 4 (4 g + e) + j % 4 of half j / 4)
    auto feature = [&](int e, int j) { return VB == 32 && FORM == kPlain ? 64 * (j >> 2) + 4 * (4 * g + e) + (j & 3) : VF * (4 * g + e) + j; };
    if (SHARED && t0 == 0 && t1 == s.tiles) {
      if (row_there) {
        const int64_t to = (int64_t)(s.first + token) * a.n_q_heads + head;
        if (g == 0) kv_own_state(a)[to] = float2{m, l};
        float *sums = a.own + to * DH;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < VF; ++j) sums[feature(e, j)] = o[j][e];
      }
    } else if (t0 == 0 && t1 == s.tiles) {
      if (row_there) {
        T *out = (T *)(a.out.p + (s.first + token) * a.out.row + head * a.out.head);
        const bool nothing = m == -INFINITY && l == 0.f;              // (NaN logits leave l NaN)
        const float inv = 1.f / l;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < VF; ++j) out[feature(e, j)] = kv_round<T>(nothing ? 0.f : o[j][e] * inv);
      }
    } else if (row_there) {
      float *part = parts + ((int64_t)worker * 2 + (begins ? 0 : 1)) * split_part_floats(DH);
      if (g == 0) {
        part[l16] = m;
        part[kRows + l16] = l;
      }
      float *to = part + 2 * kRows + l16 * DH;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < VF; ++j) to[feature(e, j)] = o[j][e];
    }
    tile += t1 - t0;
    begins = false;
  }
}

template <typename T, int DH, int FORM>
__global__ __launch_bounds__(256, split_occupancy(DH)) void kv_split_kernel(KvAttention a, float *__restrict__ parts) {
  split_units<T, DH, FORM, false>(a, parts, blockIdx.x, split_workers(DH));
}

// Adds up the parts of the query rows and heads whose units were cut; a workgroup looks at `rows` of them.  Bound by latency (4 to 8 us): DH / 4 lanes share a part, so that
// 8 to 32 parts are read at once.  (With the units looked for again by every workgroup, 4096 sequences took 350 us more.)
template <typename T, int DH>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttention a, const float *__restrict__ parts, int rows) {
  constexpr int L = DH / 4, P = 256 / L;                          // lanes of a part, parts at once
  __shared__ float m_s[P], l_s[P], o_s[P][DH + 4];
  const int lane = threadIdx.x & 63;
  const int group = a.n_q_heads / a.n_kv_heads;
  const int64_t first_row = (int64_t)blockIdx.x * rows;           // rows here are rows times heads
  int2 of = {0, 0};
  const int64_t mine = first_row + lane;
  bool cut = lane < rows && mine < a.batch.n_rows * a.n_q_heads;
  if (cut) of = ((const int2 *)(parts + split_parts_floats(DH)))[mine];
  int start = cut ? (int)(mine / a.n_q_heads) : 0;                // the first row of the row's sequence
  if (a.batch.offsets) {
    // Rows that no sequence has were left as they were, and so was what is here about them.
    for (int i = 0; i < rows; ++i) {
      const int64_t row = (first_row + i) / a.n_q_heads;
      const int seq = kv_find_sequence(a.batch.offsets, a.batch.n_seqs, row, lane);
      const int64_t first = seq < a.batch.n_seqs ? a.batch.offsets[seq] : -1;
      if (lane == i) {
        cut &= first >= 0 && row >= first;
        start = (int)first;
      }
    }
  }
  cut &= of.x >> 1 < of.y && of.x >= 0 && of.y < split_workers(DH);
  for (uint64_t left = __builtin_amdgcn_ballot_w64(cut); left; left &= left - 1) {
    const int which = __builtin_ctzll(left);
    const int code = __builtin_amdgcn_readlane(of.x, which), w0 = code >> 1, w1 = __builtin_amdgcn_readlane(of.y, which);
    const int64_t q_row = (first_row + which) / a.n_q_heads;
    const int head = (int)(first_row + which - q_row * a.n_q_heads);
    const int r = (((int)q_row - __builtin_amdgcn_readlane(start, which)) * group + head % group) % kRows, p = threadIdx.x / L, f = threadIdx.x % L * 4;
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int w = w0 + p; w <= w1; w += P) {
      const float *part = parts + ((int64_t)w * 2 + (w == w0 ? code & 1 : 0)) * split_part_floats(DH);
      const float mw = part[r], lw = part[kRows + r];
      const f32x4 ow = *(const f32x4 *)(part + 2 * kRows + r * DH + f);
      const float m_new = fmaxf(m, mw), m_at = m_new == -INFINITY ? 0.f : m_new;
      const float keep = m == m_new ? 1.f : __builtin_amdgcn_exp2f(m - m_at), take = mw == m_new ? 1.f : __builtin_amdgcn_exp2f(mw - m_at);
      l = l * keep + lw * take;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = o[i] * keep + ow[i] * take;
      m = m_new;
    }
    *(f32x4 *)&o_s[p][f] = o;
    if (f == 0) { m_s[p] = m; l_s[p] = l; }
    __syncthreads();
    if (threadIdx.x < DH) {
      float top = -INFINITY, sum = 0.f, out = 0.f;
#pragma unroll
      for (int i = 0; i < P; ++i) top = fmaxf(top, m_s[i]);
      const float at = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float take = m_s[i] == top ? 1.f : __builtin_amdgcn_exp2f(m_s[i] - at);
        sum += l_s[i] * take;
        out += o_s[i][threadIdx.x] * take;
      }
      ((T *)(a.out.p + (int64_t)q_row * a.out.row + head * a.out.head))[threadIdx.x] = kv_round<T>(top == -INFINITY && sum == 0.f ? 0.f : out / sum);
    }
    __syncthreads();
  }
}

template <int FORM> hipError_t launch_split(const KvAttention &a, void *workspace, hipStream_t stream) {
  // A workgroup of the join per row and head up to 16384 (most of more are not cut: there are no more cut units than wavefronts), and no more of them than lanes.
  const int64_t joins = a.batch.n_rows * a.n_q_heads;
  const int rows = (int)std::min((joins + 16383) / 16384, (int64_t)64);
  kv_with_type(a.dtype, [&](auto t) {
    using T = decltype(t);
    kv_with_width(a.head_dim, [&](auto width) {
      constexpr int DH = decltype(width)::value;
      kv_split_kernel<T, DH, FORM><<<split_workers(DH) / 4, 256, 0, stream>>>(a, (float *)workspace);
      kv_join_kernel<T, DH><<<(unsigned)((joins + rows - 1) / rows), 256, 0, stream>>>(a, (const float *)workspace, rows);
    });
  });
  return hipGetLastError();
}

}  // namespace

}  // namespace flame
