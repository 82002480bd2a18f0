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
#include <algorithm>

#include "kv_device.h"

namespace flame {

namespace {

// Wavefronts per SIMD, as their registers allow, and in all.  Two tiles in flight fill the registers: 128 features spill 11 to 13 of 256 (48 to 56 bytes a lane), and scalars go to lanes of
// others (some 350 of 128 features in 16 bits, fewer in the rest).  Decoding of many keys runs at
// memory speed all the same.
constexpr int split_occupancy(int dh) { return dh == 128 ? 2 : dh == 64 ? 3 : 4; }
constexpr int split_workers(int dh) { return 1024 * split_occupancy(dh); }
constexpr int kRows = 16;           // query rows of a unit

template <typename T, int DH> struct SplitShape {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int KT = F32 ? 16 : 32;          // keys of a tile
  static constexpr int VF = DH / 16;                // features of a lane in the second product
};

// What a wavefront knows of a sequence.
struct SplitSeq {
  int first;          // its first query row
  int rows, blocks;   // query rows times G, and units per key head
  int n, back;        // keys; keys that the row before the first one would see
  int tiles;          // of one unit
  bool wrong;         // offsets that are none
};

template <int KT> __device__ __forceinline__ SplitSeq split_sequence(const KvAttention &a, int b, bool report) {
  SplitSeq s;
  s.n = kv_clip_length(a.batch.kv_lens[b], a.pages.capacity, a.batch.faults, report);
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
  s.back = (int)max(s.n - full, -((int64_t)1 << 30));
  s.rows = (int)(m * group);                        // (rows times heads is below 2^25)
  s.blocks = (s.rows + kRows - 1) / kRows;
  s.tiles = s.rows ? max(1, (s.n + KT - 1) / KT) : 0;   // (a unit without keys writes zeros)
  return s;
}

// Of up to 64 sequences each lane keeps one; of more they are read again.
__device__ __forceinline__ SplitSeq split_from_lane(const SplitSeq &s, int lane) {
  return SplitSeq{__builtin_amdgcn_readlane(s.first, lane), __builtin_amdgcn_readlane(s.rows, lane), __builtin_amdgcn_readlane(s.blocks, lane),
                  __builtin_amdgcn_readlane(s.n, lane), __builtin_amdgcn_readlane(s.back, lane), __builtin_amdgcn_readlane(s.tiles, lane), false};
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

template <int KT, typename F> __device__ __forceinline__ SplitPlace split_find(const KvAttention &a, int lane, F target) {
  SplitPlace p{0, 0, a.batch.n_seqs, SplitSeq{}};
  int lo = 0, n = a.batch.n_seqs;
  int64_t base = 0, at = 0;
  for (bool top = true;; top = false) {
    // lane i: the tiles of `chunk` sequences from lo + i chunk on, of one sequence in the end
    const bool report = top && blockIdx.x == 0 && threadIdx.x < 64;
    int64_t mine = 0;
    int chunk = 1;
    if (n <= 64) {
      if (lane < n) {
        const SplitSeq s = split_sequence<KT>(a, lo + lane, report);
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
          const SplitSeq s = split_sequence<KT>(a, lo + i * chunk + k, report);
          sum += (int64_t)s.blocks * s.tiles;
        }
        const int64_t all = split_lane(split_scan(sum), 63);
        if (lane == i) mine = all;
      }
    }
    mine *= a.n_kv_heads;
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

template <typename T> struct Matrix16;
template <> struct Matrix16<bf16_t> {
  typedef bf16x8 frag;
  static __device__ __forceinline__ f32x4 mul(frag x, frag y, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0); }
};
template <> struct Matrix16<half_t> {
  typedef f16x8 frag;
  static __device__ __forceinline__ f32x4 mul(frag x, frag y, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0); }
};

template <typename T, int DH>
__global__ __launch_bounds__(256, split_occupancy(DH)) void kv_split_kernel(KvAttention a, float *__restrict__ parts) {
  typedef SplitShape<T, DH> S;
  constexpr int KT = S::KT, VF = S::VF;
  constexpr bool F32 = S::F32;
  constexpr int KB = KT / 16;                                     // 16-key blocks of a tile
  constexpr int KS = DH * (int)sizeof(T) / 64;                    // 64-byte steps of a key row: 16 bytes per lane each
  constexpr int VK = KT / 4;                                      // keys of a lane in the second product
  constexpr int VB = VF * (int)sizeof(T);                         // bytes of a lane per value row: 4..32
  constexpr int VW = VB / 4;
  typedef uint32_t word4 __attribute__((ext_vector_type(4)));
  __shared__ int64_t offset_s[4][2][KT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int worker = blockIdx.x * 4 + wave;
  int64_t per = 0;
  SplitPlace place = split_find<KT>(a, lane, [&](int64_t total) {
    per = (total + split_workers(DH) - 1) / split_workers(DH);
    return (int64_t)worker * per;
  });
  int64_t tile = (int64_t)worker * per;                           // on the line of all tiles
  const int64_t tile_end = min(tile + per, place.total);
  const float scale = a.scale * kLog2e;
  const int group = a.n_q_heads / a.n_kv_heads;
  int seq = place.seq;
  int64_t seq_tile = place.first_tile;
  bool begins = true;                                             // the unit is the worker's first
  while (tile < tile_end && seq < a.batch.n_seqs) {
    const SplitSeq s = a.batch.n_seqs <= 64 ? split_from_lane(place.mine, seq) : split_sequence<KT>(a, seq, false);
    int64_t in_seq = tile - seq_tile;
    const int64_t seq_tiles = (int64_t)a.n_kv_heads * s.blocks * s.tiles;
    if (in_seq >= seq_tiles) {                                    // (sequences without rows have none)
      seq_tile += seq_tiles;
      ++seq;
      continue;
    }
    const int unit = (int)(in_seq / s.tiles), t0 = (int)(in_seq - (int64_t)unit * s.tiles);
    const int t1 = (int)min((int64_t)s.tiles, t0 + (tile_end - tile));
    const int kvh = unit / s.blocks, block = unit - kvh * s.blocks;
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
      for (int i = 0; i < KS; ++i) fq[i] = *(const word4 *)(q + i * 64 + g * 16);
    }
    f32x4 o[VF];
#pragma unroll
    for (int j = 0; j < VF; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    // Row offsets of a tile: key k by lane k; keys behind the last one repeat it, keys in pages that the table does not name get the pool's first row, and neither counts.
    auto look_up = [&](int t) -> int64_t {
      const int key = min(t * KT + (lane & (KT - 1)), s.n - 1);
      return key < 0 ? -1 : kv_token_offset(a.pages, table, (uint32_t)key);
    };
    struct Tile {
      word4 k[KB][KS];
      uint32_t v[VK][VW];
      uint64_t there;                                             // lanes' keys that count
    };
    auto request = [&](Tile &x, int t, int64_t offset) {
      if (offset < 0 && s.n > 0 && lane < KT) kv_fault(a.batch.faults, FLAME_KV_FAULT_PAGE);
      x.there = __builtin_amdgcn_ballot_w64(offset >= 0 && t * KT + (lane & (KT - 1)) < s.n);
      int64_t *at = offset_s[wave][t & 1];
      if (lane < KT) at[lane] = max(offset, (int64_t)0);
      __builtin_amdgcn_wave_barrier();
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
    };
    auto add = [&](Tile &x, int t) {
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
      const uint32_t here = (uint32_t)(x.there >> (VK * g)) & ((1u << VK) - 1);                       // of my VK keys those that count,
      const uint32_t seen = here & ((1u << max(0, min(VK, sees - k0))) - 1);                         // and those of them that my row sees
      const bool masked = x.there != ~0ull || t * KT + KT > sees_least;
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
      if (__builtin_amdgcn_ballot_w64(m_new != m)) {
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
      if (masked) {
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
    l = split_sum(l);
    if (t0 == 0 && row_there && g == 0) {
      const int last = t1 == s.tiles ? worker : (int)((tile + s.tiles - 1) / per);
      ((int2 *)(parts + split_parts_floats(DH)))[(int64_t)(s.first + token) * a.n_q_heads + head] = int2{2 * worker + !begins, last};
    }
    // accumulator element e of product j: feature VF (4 g + e) + j of my row (fp32 with 128 features: 4 (4 g + e) + j % 4 of half j / 4)
    auto feature = [&](int e, int j) { return VB == 32 ? 64 * (j >> 2) + 4 * (4 * g + e) + (j & 3) : VF * (4 * g + e) + j; };
    if (t0 == 0 && t1 == s.tiles) {
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

}  // namespace

int64_t kv_split_workspace_bytes(int32_t head_dim, int64_t rows) {
  return split_parts_floats(head_dim) * 4 + (rows + 1) / 2 * 16;
}

hipError_t launch_kv_split(const KvAttention &a, void *workspace, hipStream_t stream) {
  // A workgroup of the join per row and head up to 16384 (most of more are not cut: there are no more cut units than wavefronts), and no more of them than lanes.
  const int64_t joins = a.batch.n_rows * a.n_q_heads;
  const int rows = (int)std::min((joins + 16383) / 16384, (int64_t)64);
  kv_with_type(a.dtype, [&](auto t) {
    using T = decltype(t);
    kv_with_width(a.head_dim, [&](auto width) {
      constexpr int DH = decltype(width)::value;
      kv_split_kernel<T, DH><<<split_workers(DH) / 4, 256, 0, stream>>>(a, (float *)workspace);
      kv_join_kernel<T, DH><<<(unsigned)((joins + rows - 1) / rows), 256, 0, stream>>>(a, (const float *)workspace, rows);
    });
  });
  return hipGetLastError();
}

}  // namespace flame
