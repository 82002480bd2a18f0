// Device helpers of the operators on a paged key/value cache: whose row is this, how long is its sequence, where does a token lie.
#pragma once
#include <type_traits>

#include "device_common.h"
#include "kv.h"

namespace flame {

__device__ __forceinline__ void kv_fault(int32_t *faults, int32_t bits) {
  if (faults) atomicOr(faults, bits);
}

// A sequence whose offsets are none: it has no rows, and of up to 64 sequences neither do those behind it, whose offsets may claim the rows of others.
__device__ __forceinline__ bool kv_wrong_offsets(int64_t first, int64_t end) { return first < 0 || end < first; }
__device__ __forceinline__ void kv_report_offsets(int64_t first, int64_t end, int64_t n_rows, int32_t *faults) {
  if (kv_wrong_offsets(first, end) || end > n_rows) kv_fault(faults, FLAME_KV_FAULT_OFFSET);
}

// The sequence whose rows hold row t, for the wavefront: the first b with offsets[b + 1] > t.  64 probes at a time, so one
// load's latency for up to 64 sequences and two up to 4096.  n_seqs where the row is behind the last sequence, or behind offsets that are none.  Whatever the
// offsets hold, the probes stay within offsets[0..n_seqs].  (A row may still be ahead of its sequence, and of more than 64 behind it: callers look.)
__device__ __forceinline__ int kv_find_sequence(const int32_t *offsets, int n_seqs, int64_t t, int lane) {
  int lo = 0, n = n_seqs;
  while (n > 64) {
    const int step = (n + 63) / 64;
    const int at = lo + min((lane + 1) * step, n);
    const uint64_t beyond = __builtin_amdgcn_ballot_w64(offsets[at] > t);
    const int c = beyond ? __builtin_ctzll(beyond) : 64;
    if (c * step >= n) return lo + n;
    lo += c * step;
    n = min(step, n - c * step);
  }
  int first = 0, end = 0;
  if (lane < n) {
    first = offsets[lo + lane];
    end = offsets[lo + lane + 1];
  }
  const uint64_t beyond = __builtin_amdgcn_ballot_w64(lane < n && end > t), wrong = __builtin_amdgcn_ballot_w64(lane < n && kv_wrong_offsets(first, end));
  const int found = beyond ? __builtin_ctzll(beyond) : n;
  return wrong && __builtin_ctzll(wrong) <= found ? n_seqs : lo + found;
}

// Tokens of a sequence, within what its row of the table has room for.
__device__ __forceinline__ int kv_clip_length(int len, int capacity, int32_t *faults, bool report) {
  const int n = kv_clip(len, capacity);
  if (report && n != len) kv_fault(faults, FLAME_KV_FAULT_LENGTH);
  return n;
}

// Element type as a template argument of the launches.
template <typename F> inline void kv_with_type(int32_t dtype, F f) {
  if (dtype == FLAME_KV_F32) f(0.f);
  else if (dtype == FLAME_KV_BF16) f((bf16_t)0.f);
  else f((half_t)0.f);
}

template <typename F> inline void kv_with_width(int32_t head_dim, F f) {
  if (head_dim == 32) f(std::integral_constant<int, 32>{});
  else if (head_dim == 64) f(std::integral_constant<int, 64>{});
  else f(std::integral_constant<int, 128>{});
}

// Infinities and NaN in a word of one fp32 or two 16-bit values.
template <typename T> constexpr uint32_t kv_exponent() { return sizeof(T) == 4 ? 0x7f800000u : std::is_same<T, bf16_t>::value ? 0x7f80u : 0x7c00u; }
template <typename T> __device__ __forceinline__ bool not_finite(uint32_t w) {
  constexpr uint32_t E = kv_exponent<T>();
  return sizeof(T) == 4 ? (w & E) == E : (w & E) == E || (w >> 16 & E) == E;
}
template <typename T> __device__ __forceinline__ uint32_t only_finite(uint32_t w) {
  constexpr uint32_t E = kv_exponent<T>();
  if (sizeof(T) == 4) return (w & E) == E ? 0u : w;
  return ((w & E) == E ? 0u : w & 0xffffu) | ((w >> 16 & E) == E ? 0u : w & 0xffff0000u);
}

// Parts of rows whose keys were cut, in the workspace: of every part and output row the sums [planes][rows][features], and behind them the maxima and weights [planes][rows].
__device__ __forceinline__ int64_t kv_part_row(const KvAttention &a, int plane, int64_t row) { return plane * a.batch.n_rows * a.n_q_heads + row; }
__device__ __forceinline__ float2 *kv_part_state(const KvAttention &a, int planes) { return (float2 *)(a.parts + planes * a.batch.n_rows * a.n_q_heads * a.head_dim); }

// With shared histories: the parts of the histories, whose states stand behind a.part_rows of them, and the results over the sequences' own keys, a row each.
__device__ __forceinline__ float2 *kv_shared_state(const KvAttention &a) { return (float2 *)(a.parts + a.part_rows * a.head_dim); }
__device__ __forceinline__ float2 *kv_own_state(const KvAttention &a) { return (float2 *)(a.own + a.batch.n_rows * a.n_q_heads * a.head_dim); }

// Softmax weights are 2^(logit - reference), and `above` is what log2 of a weight may come to.  fp16 weights would be zeros from 2^-25 on, thousands of which can make up a row's result
// beside one of 1; they are held as high as its range has room (up to 2^15), by a reference that is as much lower, in numerator and denominator alike.  Others need no such place.
template <typename T> constexpr float kv_lowered(int above) { return std::is_same<T, half_t>::value ? (float)(15 - above) : 0.f; }

// One rounding of an fp32 result, to nearest; an fp16 one past the largest finite value becomes infinite, as in IEEE arithmetic.
template <typename T> __device__ __forceinline__ T kv_round(float v) { return (T)v; }

}  // namespace flame
