// Keys and values of new tokens into a cache of 8 or 4 bits, keys and queries rotated by their positions on the way; and rows back out of one.
//
// Bound by memory: each row is read once and written once, in half or a quarter of its bytes.  A wavefront takes a few tokens side by side: lane i finds the sequence, position and page of the i-th,
// and their rows are dealt out to the lanes, whatever the number of heads.  Appending, a lane takes eight features of a row, so that four lanes side by side have the 32 of a block, whose largest size goes
// between them in two DPP steps, and the conversions of the chip divide by the scale and round, two features an instruction.  The partner of a feature that turns is half the rotated features
// away or next to it: pairs (j, j + r/2) read the eight partners too, which are other lanes' features and come from the caches (r is a multiple of 16, so eight features lie on one side of
// r/2).  Reading, a lane makes 16 bytes of a row.
#include "kv_codec.h"
#include "kv_rotate.h"

namespace flame {

namespace {

constexpr int kWaves = 4;           // of a workgroup
constexpr int kAppendTokens = 4;    // of a wavefront, at most: their angles are in LDS

template <typename T> __device__ __forceinline__ void load_eight(const char *p, float (&x)[8]) {
  struct alignas(16) Values { T v[8]; };
  const Values y = *(const Values *)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)y.v[i];
}
template <bool STREAM> __device__ __forceinline__ void store16(char *p, f32x4 x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, (f32x4 *)p);
  else *(f32x4 *)p = x;
}
template <typename T, bool STREAM> __device__ __forceinline__ void store_eight(char *p, const float (&x)[8]) {
  struct alignas(16) Values { T v[8]; } y;
#pragma unroll
  for (int i = 0; i < 8; ++i) y.v[i] = kv_round<T>(x[i]);
#pragma unroll
  for (int i = 0; i < (int)sizeof(y) / 16; ++i) store16<STREAM>(p + 16 * i, ((const f32x4 *)&y)[i]);
}

// Feature block `at` (of eight) of a row, turned.
template <typename T> __device__ __forceinline__ void load_turned(const char *row, int at, const KvRotation &rot, const float2 *turn, float (&x)[8]) {
  constexpr int B = 8 * sizeof(T);
  load_eight<T>(row + at * B, x);
  if (at >= rot.pairs / 4) return;                                // (pairs / 4 blocks turn)
  if (rot.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float2 cs = turn[at * 4 + i / 2];
      const float a = x[i], b = x[i + 1];
      x[i] = a * cs.x - b * cs.y;
      x[i + 1] = a * cs.y + b * cs.x;
    }
  } else {
    const int half = rot.pairs / 8;
    const bool low = at < half;
    float y[8];
    load_eight<T>(row + (low ? at + half : at - half) * B, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 cs = turn[(low ? at : at - half) * 8 + i];
      x[i] = low ? x[i] * cs.x - y[i] * cs.y : y[i] * cs.y + x[i] * cs.x;
    }
  }
}

template <int CTRL> __device__ __forceinline__ uint32_t lane_max(uint32_t v) { return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false)); }

// Eight features of a block into the cache; `to`: where their codes go, from the pool's start.
template <typename T, int FORM> __device__ __forceinline__ void store_codes(char *pool, char *scales, int64_t to, float (&x)[8]) {
  uint32_t most = 0;                                              // as bits: infinities and NaN are larger than all else
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
  most = lane_max<0x4e>(lane_max<0xb1>(most));                    // quad_perm: neighbours, then pairs
  constexpr float largest = kv_largest<T, FORM>();
  constexpr int kTop = FORM == kF8 ? 8 : 2;                       // exponent of the largest code
  constexpr uint32_t kOver = FORM == kF8 ? 0x680001u : 0x600000u; // fraction of a size that would round beyond it: past 464 / 256, from 7 / 4
  const uint32_t size = min(most, __float_as_uint(largest));
  const int e = max((int)(size >> 23) - 127 - kTop + ((size & 0x7fffffu) >= kOver), kv_least_exponent<T, FORM>());
  const float scale = kv_scale((uint32_t)(e + 127));
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = fminf(fmaxf(x[i], -largest), largest);
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  if constexpr (FORM == kF8) {
    s16x2 w[2] = {};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[i], x[4 * i], x[4 * i + 1], scale, false);
      w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[i], x[4 * i + 2], x[4 * i + 3], scale, true);
    }
    *(uint2 *)(pool + to) = uint2{__builtin_bit_cast(uint32_t, w[0]), __builtin_bit_cast(uint32_t, w[1])};
  } else {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    *(uint32_t *)(pool + to) = w;
  }
  if ((threadIdx.x & 3) == 0) *(uint8_t *)(scales + (to >> kv_scale_shift<FORM>())) = most >= 0x7f800000u ? 255 : (uint8_t)(e + 127);
}

// A lane's token, of the wavefront's `count` from row0 on.
struct Token {
  int64_t position, at;        // in its sequence, in the pools in bytes; at < 0: nowhere
  bool there;
};
__device__ __forceinline__ Token find_tokens(const KvBatch &batch, const KvPages &pages, int64_t row0, int count, int lane) {
  if (batch.faults)
    for (int64_t b = (int64_t)blockIdx.x * (64 * kWaves) + threadIdx.x; b < batch.n_seqs; b += (int64_t)gridDim.x * (64 * kWaves))
      kv_report_offsets(batch.offsets[b], batch.offsets[b + 1], batch.n_rows, batch.faults);
  Token t{0, -1, false};
  if (row0 >= batch.n_rows) return t;
  const int64_t row = row0 + lane;
  // (behind the last sequence there is nothing to look for; of up to 64, which are looked at once, offsets that are none may lie behind those that have rows)
  bool open = lane < count && row < batch.n_rows && (batch.n_seqs <= 64 || row < batch.offsets[batch.n_seqs]);
  int seq = 0;
  int64_t first = 0, end = 0;
  // From the first token's sequence on (of up to 64 from the first one), a lane holds one sequence of 64: lane i looks among them for the first one that ends behind its token, ahead of offsets that are none.
  for (int s0 = batch.n_seqs <= 64 ? 0 : kv_find_sequence(batch.offsets, batch.n_seqs, row0, lane); s0 < batch.n_seqs; s0 += 64) {
    int b = 0, e = 0;
    if (s0 + lane < batch.n_seqs) {
      b = batch.offsets[s0 + lane];
      e = batch.offsets[s0 + lane + 1];
    }
    const uint64_t wrong = __builtin_amdgcn_ballot_w64(kv_wrong_offsets(b, e));
    const int limit = wrong ? __builtin_ctzll(wrong) : min(64, batch.n_seqs - s0);
    int at = 0;                                                   // sequences that end at or ahead of the token
#pragma unroll
    for (int step = 32; step; step >>= 1) {
      const int probe = __shfl(e, at + step - 1);
      if (at + step <= limit && probe <= row) at += step;
    }
    if (at == 63 && limit == 64 && __builtin_amdgcn_readlane(e, 63) <= row) at = 64;
    const int mine_b = __shfl(b, min(at, 63)), mine_e = __shfl(e, min(at, 63));
    if (open && at < limit) {
      open = false;
      seq = s0 + at;
      first = mine_b;
      end = mine_e;
      t.there = row >= first;                                     // (else ahead of the first sequence)
    }
    if (wrong || limit < 64 || !__builtin_amdgcn_ballot_w64(open)) break;
  }
  if (!t.there) return t;
  t.position = (int64_t)batch.kv_lens[seq] - end + row;
  const bool placed = t.position >= 0 && t.position < pages.capacity;
  if (placed) t.at = kv_token_offset(pages, pages.table + seq * pages.table_stride, (uint32_t)t.position);
  if (t.at < 0) kv_fault(batch.faults, placed ? FLAME_KV_FAULT_PAGE : FLAME_KV_FAULT_LENGTH);
  return t;
}

__device__ __forceinline__ int64_t of_lane(int64_t v, int lane) {
  return (int64_t)(((uint64_t)(uint32_t)__shfl((int)(v >> 32), lane) << 32) | (uint32_t)__shfl((int)v, lane));
}

template <typename T, int FORM, bool STREAM>
__global__ __launch_bounds__(64 * kWaves) void kvq_append_kernel(KvBatch batch, KvPages pages, KvScales scales, KvRows k, KvRows v, KvRows q, KvRows q_out, KvRotation rot, int n_q, int n_kv, int head_dim,
                                                                int count) {
  __shared__ float2 turn_s[kWaves][kAppendTokens][kMaxRotationPairs];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row0 = ((int64_t)blockIdx.x * kWaves + wave) * count;
  const Token t = find_tokens(batch, pages, row0, count, lane);
  if (!__builtin_amdgcn_ballot_w64(t.there)) return;
  for (int i = 0; i < count; ++i) {
    const int64_t position = of_lane(t.position, i);
    if (lane < rot.pairs) turn_s[wave][i][lane] = cos_sin_of_turn(rot.turns[lane] * (uint64_t)position);
  }
  // (a wavefront reads only what it wrote itself)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int per_row = head_dim / 8, shift = per_row == 4 ? 2 : per_row == 8 ? 3 : 4;      // lanes of a row
  const int at = lane & (per_row - 1), rows = 64 / per_row;
  const int written = t.there && t.position >= 0;                 // the token's query
  // rows (token, head) of keys and values, then of queries; the grid's second dimension shares them
  for (int r = rows * blockIdx.y; r < count * n_kv; r += rows * gridDim.y) {
    const int mine = r + (lane >> shift), i = mine / n_kv, h = mine - i * n_kv;
    const int64_t page_at = of_lane(t.at, i & 63);
    if (i >= count || page_at < 0) continue;
    const int64_t row = row0 + i, to = page_at + h * pages.head + kv_row_bytes<T, FORM>(8) * at;
    float x[8], y[8];
    load_turned<T>(k.p + row * k.row + h * k.head, at, rot, turn_s[wave][i], x);
    load_eight<T>(v.p + row * v.row + h * v.head + at * 8 * sizeof(T), y);
    store_codes<T, FORM>(pages.k, scales.k, to, x);
    store_codes<T, FORM>(pages.v, scales.v, to, y);
  }
  if (!q.p) return;
  // (a row's lanes are of one wavefront, which loads all of them before it stores any: q_out may be q)
  for (int r = rows * blockIdx.y; r < count * n_q; r += rows * gridDim.y) {
    const int mine = r + (lane >> shift), i = mine / n_q, h = mine - i * n_q;
    const int go = __shfl(written, i & 63);                       // (by all lanes: one that is switched off has nothing to be read from it)
    if (!go || i >= count) continue;
    const int64_t row = row0 + i;
    float x[8];
    load_turned<T>(q.p + row * q.row + h * q.head, at, rot, turn_s[wave][i], x);
    store_eight<T, STREAM>(q_out.p + row * q_out.row + h * q_out.head + at * 8 * sizeof(T), x);
  }
}

template <int BYTES> __device__ __forceinline__ void load_codes(const char *p, uint32_t (&w)[2]) {
  w[1] = 0;
  if constexpr (BYTES == 8) {
    const uint2 y = *(const uint2 *)p;
    w[0] = y.x;
    w[1] = y.y;
  } else if constexpr (BYTES == 4) {
    w[0] = *(const uint32_t *)p;
  } else {
    w[0] = *(const uint16_t *)p;
  }
}

template <typename T, int FORM, bool STREAM>
__global__ __launch_bounds__(64 * kWaves) void kvq_read_kernel(KvBatch batch, KvPages pages, KvScales scales, KvRows k, KvRows v, int n_kv, int head_dim, int count) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row0 = ((int64_t)blockIdx.x * kWaves + wave) * count;
  const Token t = find_tokens(batch, pages, row0, count, lane);
  if (!__builtin_amdgcn_ballot_w64(t.at >= 0)) return;
  constexpr int E = 16 / sizeof(T);                                       // features of a lane: 16 bytes, so that a store fills lines
  const int per_row = head_dim / E, shift = __builtin_ctz(per_row);
  const int at = lane & (per_row - 1), rows = 64 / per_row;
  constexpr int B = kv_row_bytes<T, FORM>(E);
  typedef typename KvPair<T>::vec pair;
  struct alignas(16) Out { pair p[E / 2]; };
  constexpr int U = 4;                                                    // rows of a lane at once: their loads are all in flight
  for (int r = 0; r < count * n_kv; r += U * rows) {
    uint32_t kc[U][2], vc[U][2], ks[U], vs[U];
    int64_t row[U];
    int h[U];
    bool go[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int mine = r + u * rows + (lane >> shift), i = mine / n_kv;
      h[u] = mine - i * n_kv;
      const int64_t page_at = of_lane(t.at, i & 63);
      go[u] = i < count && page_at >= 0;
      row[u] = row0 + i;
      const int64_t from = page_at + h[u] * pages.head + B * at;
      if (!go[u]) continue;
      load_codes<B>(pages.k + from, kc[u]);
      load_codes<B>(pages.v + from, vc[u]);
      ks[u] = *(const uint8_t *)(scales.k + (from >> kv_scale_shift<FORM>()));
      vs[u] = *(const uint8_t *)(scales.v + (from >> kv_scale_shift<FORM>()));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!go[u]) continue;
      pair x[4], y[4];
      kv_eight<T, FORM>(kc[u], kv_scale(ks[u]), x);
      kv_eight<T, FORM>(vc[u], kv_scale(vs[u]), y);
      Out kx, vx;
#pragma unroll
      for (int n = 0; n < E / 2; ++n) {
        kx.p[n] = x[n];
        vx.p[n] = y[n];
      }
      store16<STREAM>(k.p + row[u] * k.row + h[u] * k.head + at * 16, __builtin_bit_cast(f32x4, kx));
      store16<STREAM>(v.p + row[u] * v.row + h[u] * v.head + at * 16, __builtin_bit_cast(f32x4, vx));
    }
  }
}

// Rows of more than kStream bytes go past the caches: they are not there any more when the next kernel wants them, and what would be is lost.  us in the caches | past them (of the two halves of a read, or of the
// queries): read of 2 x 79 MB (bf16, 8 heads of 128) f8 56 | 37, f4 48 | 32, 2 x 40 MB 31 | 21, 26 | 18, 2 x 200 MB 127 | 112, 112 | 104, 2 x 34 MB (2 heads of 64) 28 | 19, 18 | 17, fp32 of 2 x 130 MB 73 | 49, 69 | 45;
// append of 4800 tokens with 39 MB of queries (32/8 heads of 128) 29 | 21, of 12000 66 | 62, 63 | 59.  Up to 2 x 24 MB both take the same within a microsecond or two (2 x 16 MB 10.4 | 10.3, f4 10.1 | 8.6), and a next kernel
// finds small rows in the caches.
constexpr int64_t kStream = 16 << 20;
template <typename F> void with_stored(int32_t dtype, int32_t form, int64_t bytes, F f) {
  kv_with_type(dtype, [&](auto t) {
    const auto go = [&](auto stream) {
      if (form == kF8) f(t, std::integral_constant<int, kF8>{}, stream);
      else f(t, std::integral_constant<int, kF4>{}, stream);
    };
    if (bytes > kStream) go(std::true_type{});
    else go(std::false_type{});
  });
}

// Tokens of a wavefront: as many as give its lanes `rounds` rows' pieces each, but not so many that few wavefronts are left (one token each of 48 sequences, 8/2 heads of 64: 8.8 us by wavefronts of four).
int tokens_of(int64_t n_rows, int lanes_of_token, int rounds, int most) {
  int count = 1;
  while (count < most && count * lanes_of_token < 64 * rounds && n_rows / (2 * count) >= (count * lanes_of_token < 64 ? 1024 : 4096)) count *= 2;
  return count;
}
unsigned blocks_of(const KvBatch &batch, int count) { return (unsigned)((batch.n_rows + count * kWaves - 1) / (count * kWaves)); }

}  // namespace

hipError_t launch_kvq_append(const KvBatch &batch, const KvPages &pages, const KvScales &scales, const KvRows &k, const KvRows &v, const KvRows *q, const KvRows *q_out,
                             const KvRotation &rotation, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype, hipStream_t stream) {
  const int count = tokens_of(batch.n_rows, n_kv_heads * head_dim / 8, 1, kAppendTokens);
  // Few tokens: several wavefronts share the heads of theirs, up to one for each 64 lanes' worth of queries (one token each of 256 sequences, 32/8 heads of 128: 13.2 us with one).
  int share = 1;
  while (share * 2 * (64 / (head_dim / 8)) <= count * n_q_heads && batch.n_rows / count * share < 4096) share *= 2;
  const int64_t bytes = batch.n_rows * n_q_heads * head_dim * (dtype == FLAME_KV_F32 ? 4 : 2);
  with_stored(dtype, scales.form, bytes, [&](auto t, auto form, auto past) {
    kvq_append_kernel<decltype(t), decltype(form)::value, decltype(past)::value><<<dim3(blocks_of(batch, count), share), 64 * kWaves, 0, stream>>>(batch, pages, scales, k, v, q ? *q : KvRows{}, q ? *q_out : KvRows{}, rotation,
                                                                                                           n_q_heads, n_kv_heads, head_dim, count);
  });
  return hipGetLastError();
}

hipError_t launch_kvq_read(const KvBatch &batch, const KvPages &pages, const KvScales &scales, const KvRows &k, const KvRows &v, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                           hipStream_t stream) {
  const int token_bytes = n_kv_heads * head_dim * (dtype == FLAME_KV_F32 ? 4 : 2), count = tokens_of(batch.n_rows, token_bytes / 16, 4, 64);
  with_stored(dtype, scales.form, batch.n_rows * token_bytes, [&](auto t, auto form, auto past) {
    kvq_read_kernel<decltype(t), decltype(form)::value, decltype(past)::value><<<blocks_of(batch, count), 64 * kWaves, 0, stream>>>(batch, pages, scales, k, v, n_kv_heads, head_dim, count);
  });
  return hipGetLastError();
}

}  // namespace flame
