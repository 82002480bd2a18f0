// Keys and values of new tokens into a cache of 8 or 4 bits, keys and queries rotated by their positions on the way; and rows back out of one.
//
// Bound by memory: each row is read once and written once, in half or a quarter of its bytes.  One wavefront takes one token with all its heads, as in kv_append.hip: the heads share the token's page,
// position and angles.  A lane takes eight features of a row, so that four lanes side by side have the 32 of a block, whose largest size goes between them in two DPP steps, and the
// conversions of the chip divide by the scale and round, two features an instruction.  The partner of a feature that turns is half the rotated features away or next to it: pairs
// (j, j + r/2) read the eight partners too, which are other lanes' features and come from the caches (r is a multiple of 16, so eight features lie on one side of r/2).
#include "kv_codec.h"
#include "kv_rotate.h"

namespace flame {

namespace {

constexpr int kTokensPerBlock = 4;

template <typename T> __device__ __forceinline__ void load_eight(const char *p, float (&x)[8]) {
  struct alignas(16) Values { T v[8]; };
  const Values y = *(const Values *)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)y.v[i];
}
template <typename T> __device__ __forceinline__ void store_eight(char *p, const float (&x)[8]) {
  struct alignas(16) Values { T v[8]; } y;
#pragma unroll
  for (int i = 0; i < 8; ++i) y.v[i] = kv_round<T>(x[i]);
  *(Values *)p = y;
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

// The wavefront's token: its sequence and place, for both directions.
struct Token {
  int64_t row, position, at;   // of the arrays, of the sequence, of the pools in bytes; at < 0: nowhere
  bool there;
};
__device__ __forceinline__ Token find_token(const KvBatch &batch, const KvPages &pages, int lane, int wave) {
  if (batch.faults)
    for (int64_t b = (int64_t)blockIdx.x * (64 * kTokensPerBlock) + threadIdx.x; b < batch.n_seqs; b += (int64_t)gridDim.x * (64 * kTokensPerBlock))
      kv_report_offsets(batch.offsets[b], batch.offsets[b + 1], batch.n_rows, batch.faults);
  Token t{(int64_t)blockIdx.x * kTokensPerBlock + wave, 0, -1, false};
  if (t.row >= batch.n_rows) return t;
  const int seq = kv_find_sequence(batch.offsets, batch.n_seqs, t.row, lane);
  if (seq >= batch.n_seqs) return t;                                      // behind the last sequence
  const int64_t first = batch.offsets[seq], end = batch.offsets[seq + 1];
  if (first < 0 || t.row < first || t.row >= end) return t;               // ahead of the first one, or offsets that are none
  t.there = true;
  t.position = (int64_t)batch.kv_lens[seq] - end + t.row;
  const bool placed = t.position >= 0 && t.position < pages.capacity;
  if (placed) t.at = kv_token_offset(pages, pages.table + seq * pages.table_stride, (uint32_t)t.position);
  if (t.at < 0 && lane == 0) kv_fault(batch.faults, placed ? FLAME_KV_FAULT_PAGE : FLAME_KV_FAULT_LENGTH);
  return t;
}

template <typename T, int FORM>
__global__ __launch_bounds__(64 * kTokensPerBlock) void kvq_append_kernel(KvBatch batch, KvPages pages, KvScales scales, KvRows k, KvRows v, KvRows q, KvRows q_out, KvRotation rot, int n_q, int n_kv,
                                                                         int head_dim) {
  __shared__ float2 turn_s[kTokensPerBlock][kMaxRotationPairs];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Token t = find_token(batch, pages, lane, wave);
  if (!t.there) return;
  if (lane < rot.pairs) turn_s[wave][lane] = cos_sin_of_turn(rot.turns[lane] * (uint64_t)t.position);
  // (a wavefront reads only what it wrote itself)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const float2 *turn = turn_s[wave];
  const int per_row = head_dim / 8;                                       // lanes of a row: 4, 8 or 16
  const int at = lane & (per_row - 1), row0 = lane / per_row, rows = 64 / per_row;
  if (t.at >= 0)
    for (int h = row0; h < n_kv; h += rows) {
      const int64_t to = t.at + h * pages.head + kv_row_bytes<T, FORM>(8) * at;
      float x[8], y[8];
      load_turned<T>(k.p + t.row * k.row + h * k.head, at, rot, turn, x);
      load_eight<T>(v.p + t.row * v.row + h * v.head + at * 8 * sizeof(T), y);
      store_codes<T, FORM>(pages.k, scales.k, to, x);
      store_codes<T, FORM>(pages.v, scales.v, to, y);
    }
  if (q.p && t.position >= 0)
    // (a row's lanes are of one wavefront, which loads all of them before it stores any: q_out may be q)
    for (int h = row0; h < n_q; h += rows) {
      float x[8];
      load_turned<T>(q.p + t.row * q.row + h * q.head, at, rot, turn, x);
      store_eight<T>(q_out.p + t.row * q_out.row + h * q_out.head + at * 8 * sizeof(T), x);
    }
}

template <typename T, int FORM>
__global__ __launch_bounds__(64 * kTokensPerBlock) void kvq_read_kernel(KvBatch batch, KvPages pages, KvScales scales, KvRows k, KvRows v, int n_kv, int head_dim) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Token t = find_token(batch, pages, lane, wave);
  if (t.at < 0) return;
  const int per_row = head_dim / 8;
  const int at = lane & (per_row - 1), row0 = lane / per_row, rows = 64 / per_row;
  constexpr int W = FORM == kF8 ? 2 : 1;
  typedef typename KvPair<T>::vec pair;
  struct alignas(16) Out { pair p[4]; };
  for (int h = row0; h < n_kv; h += rows) {
    const int64_t from = t.at + h * pages.head + kv_row_bytes<T, FORM>(8) * at;
    struct alignas(4 * W) Codes { uint32_t w[W]; };
    const Codes kc = *(const Codes *)(pages.k + from), vc = *(const Codes *)(pages.v + from);
    const float ks = kv_scale(*(const uint8_t *)(scales.k + (from >> kv_scale_shift<FORM>()))), vs = kv_scale(*(const uint8_t *)(scales.v + (from >> kv_scale_shift<FORM>())));
    Out x, y;
    kv_eight<T, FORM>(kc.w, ks, x.p);
    kv_eight<T, FORM>(vc.w, vs, y.p);
    *(Out *)(k.p + t.row * k.row + h * k.head + at * 8 * sizeof(T)) = x;
    *(Out *)(v.p + t.row * v.row + h * v.head + at * 8 * sizeof(T)) = y;
  }
}

template <typename F> void with_stored(int32_t dtype, int32_t form, F f) {
  kv_with_type(dtype, [&](auto t) {
    if (form == kF8) f(t, std::integral_constant<int, kF8>{});
    else f(t, std::integral_constant<int, kF4>{});
  });
}

unsigned blocks_of(const KvBatch &batch) { return (unsigned)((batch.n_rows + kTokensPerBlock - 1) / kTokensPerBlock); }

}  // namespace

hipError_t launch_kvq_append(const KvBatch &batch, const KvPages &pages, const KvScales &scales, const KvRows &k, const KvRows &v, const KvRows *q, const KvRows *q_out,
                             const KvRotation &rotation, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype, hipStream_t stream) {
  with_stored(dtype, scales.form, [&](auto t, auto form) {
    kvq_append_kernel<decltype(t), decltype(form)::value><<<blocks_of(batch), 64 * kTokensPerBlock, 0, stream>>>(batch, pages, scales, k, v, q ? *q : KvRows{}, q ? *q_out : KvRows{}, rotation,
                                                                                                             n_q_heads, n_kv_heads, head_dim);
  });
  return hipGetLastError();
}

hipError_t launch_kvq_read(const KvBatch &batch, const KvPages &pages, const KvScales &scales, const KvRows &k, const KvRows &v, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                           hipStream_t stream) {
  with_stored(dtype, scales.form, [&](auto t, auto form) {
    kvq_read_kernel<decltype(t), decltype(form)::value><<<blocks_of(batch), 64 * kTokensPerBlock, 0, stream>>>(batch, pages, scales, k, v, n_kv_heads, head_dim);
  });
  return hipGetLastError();
}

}  // namespace flame
