// Causal softmax attention of packed query rows with grouped heads, over packed keys or a paged cache.
//
// One wavefront per query row and head runs through the row's keys once, one key at a time, with the running maximum and sum of the softmax:
// the lanes share the features.
#include "kv_device.h"

namespace flame {

namespace {

template <typename T, int DH>
__global__ __launch_bounds__(256) void kv_attention_kernel(KvAttention a) {
  constexpr int N = DH >= 64 ? DH / 64 : 1;           // features per lane
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = item / a.n_q_heads;
  const int h = (int)(item % a.n_q_heads), kvh = h / (a.n_q_heads / a.n_kv_heads);
  if (row >= a.batch.n_rows) return;
  int seq = (int)row;
  int64_t first = row, end = row + 1;
  if (a.batch.offsets) {
    seq = kv_find_sequence(a.batch.offsets, a.batch.n_seqs, row, lane);
    if (seq >= a.batch.n_seqs) return;
    first = a.batch.offsets[seq];
    end = a.batch.offsets[seq + 1];
    if (row < first || first < 0 || end > a.batch.n_rows) {
      if (lane == 0) kv_fault(a.batch.faults, FLAME_KV_FAULT_OFFSET);
      if (row < first || first < 0) return;
    }
  }
  int64_t n, k_first = 0;
  if (a.pages.table) {
    n = kv_clip_length(a.batch.kv_lens[seq], a.pages.capacity, a.batch.faults, lane == 0);
  } else {
    const int32_t *ko = a.k_offsets ? a.k_offsets : a.batch.offsets;
    k_first = ko[seq];
    n = ko[seq + 1] - k_first;
    if (k_first < 0 || n < 0 || k_first + n > a.n_keys) {
      if (lane == 0) kv_fault(a.batch.faults, FLAME_KV_FAULT_OFFSET);
      n = k_first < 0 ? 0 : max((int64_t)0, min(n, a.n_keys - k_first));
    }
  }
  const int64_t seen = n - end + row + 1;             // keys that the row sees
  const int f = lane * N;
  const bool has = f < DH;
  float q[N], o[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    q[i] = has ? (float)((const T *)(a.q.p + row * a.q.row + h * a.q.head))[f + i] : 0.f;
    o[i] = 0.f;
  }
  const float scale = a.scale * kLog2e;
  float m = -INFINITY, l = 0.f;
  const int32_t *table = a.pages.table ? a.pages.table + seq * a.pages.table_stride : nullptr;
  for (int64_t c = 0; c < seen; ++c) {
    const char *kp, *vp;
    if (table) {
      const int64_t at = kv_token_offset(a.pages, table, (uint32_t)c);
      if (at < 0) {
        if (lane == 0) kv_fault(a.batch.faults, FLAME_KV_FAULT_PAGE);
        continue;
      }
      kp = a.pages.k + at + kvh * a.pages.head;
      vp = a.pages.v + at + kvh * a.pages.head;
    } else {
      kp = a.k.p + (k_first + c) * a.k.row + kvh * a.k.head;
      vp = a.v.p + (k_first + c) * a.v.row + kvh * a.v.head;
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s += has ? q[i] * (float)((const T *)kp)[f + i] : 0.f;
    s = wave_sum(s) * scale;
    const float m_new = fmaxf(m, s);
    const float keep = m == m_new ? 1.f : __builtin_amdgcn_exp2f(m - m_new), w = s == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s - m_new);
    l = l * keep + w;
    m = m_new;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = o[i] * keep + w * (has ? (float)((const T *)vp)[f + i] : 0.f);
  }
  if (!has) return;
#pragma unroll
  for (int i = 0; i < N; ++i) ((T *)(a.out.p + row * a.out.row + h * a.out.head))[f + i] = kv_round<T>(m == -INFINITY && l == 0.f ? 0.f : o[i] / l);
}

}  // namespace

hipError_t launch_kv_attention(const KvAttention &a, hipStream_t stream) {
  const unsigned blocks = (unsigned)((a.batch.n_rows * a.n_q_heads + 3) / 4);
  kv_with_type(a.dtype, [&](auto t) {
    using T = decltype(t);
    if (a.head_dim == 32) kv_attention_kernel<T, 32><<<blocks, 256, 0, stream>>>(a);
    else if (a.head_dim == 64) kv_attention_kernel<T, 64><<<blocks, 256, 0, stream>>>(a);
    else kv_attention_kernel<T, 128><<<blocks, 256, 0, stream>>>(a);
  });
  return hipGetLastError();
}

}  // namespace flame
