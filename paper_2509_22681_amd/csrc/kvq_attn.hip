// Causal softmax attention over a cache of 8 or 4 bits, and over histories that several sequences share: one wavefront per query row and head, a key per lane.
#include "kv_codec.h"

namespace flame {

namespace {

// Feature d of a stored row.
template <typename T, int FORM> __device__ __forceinline__ float stored(const char *pool, const char *scales, int64_t row, int d) {
  if constexpr (FORM == kPlain) return (float)((const T *)(pool + row))[d];
  else {
    const int64_t at = row + (FORM == kF8 ? d : d >> 1);
    const float scale = kv_scale(*(const uint8_t *)(scales + (at >> kv_scale_shift<FORM>())));
    const uint32_t code = *(const uint8_t *)(pool + at);
    const auto x = KvPair<T>::template get<FORM, 0>(code, scale);
    return (float)(FORM == kF4 && (d & 1) ? x[1] : x[0]);
  }
}

template <typename T, int FORM>
__global__ __launch_bounds__(256) void kvq_simple_kernel(KvAttention a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x == 0 && a.batch.faults) {
    for (int b = threadIdx.x; b < a.batch.n_seqs; b += 256) {
      kv_clip_length(a.batch.kv_lens[b], a.pages.capacity, a.batch.faults, true);
      if (a.batch.offsets) kv_report_offsets(a.batch.offsets[b], a.batch.offsets[b + 1], a.batch.n_rows, a.batch.faults);
      if (a.group_offsets) kv_clip_length(a.prefix_lens[b], a.pages.capacity, a.batch.faults, true);
    }
    if (threadIdx.x == 0 && a.group_offsets && (a.group_offsets[0] != 0 || a.group_offsets[a.n_groups] != a.batch.n_seqs)) kv_fault(a.batch.faults, FLAME_KV_FAULT_OFFSET);
    for (int g = threadIdx.x; g < a.n_groups; g += 256) {
      const int g0 = a.group_offsets[g], g1 = a.group_offsets[g + 1];
      kv_report_offsets(g0, g1, a.batch.n_seqs, a.batch.faults);
      if (g0 >= 0)
        for (int b = g0; b < min(g1, a.batch.n_seqs); ++b)
          if (kv_clip(a.prefix_lens[b], a.pages.capacity) > kv_clip(a.prefix_lens[g0], a.pages.capacity)) kv_fault(a.batch.faults, FLAME_KV_FAULT_LENGTH);
    }
  }
  const int64_t at = (int64_t)blockIdx.x * 4 + wave;
  if (at >= a.batch.n_rows * a.n_q_heads) return;
  const int64_t row = at / a.n_q_heads;
  const int head = (int)(at - row * a.n_q_heads), kvh = head / (a.n_q_heads / a.n_kv_heads);
  int seq = (int)row;
  int64_t first = row, end = row + 1;
  if (a.batch.offsets) {
    seq = kv_find_sequence(a.batch.offsets, a.batch.n_seqs, row, lane);
    if (seq >= a.batch.n_seqs) return;
    first = a.batch.offsets[seq];
    end = a.batch.offsets[seq + 1];
    if (first < 0 || row < first || row >= end) return;
  }
  const int n = kv_clip(a.batch.kv_lens[seq], a.pages.capacity);
  const int sees = (int)max((int64_t)0, n - (end - row) + 1);
  int trunk = 0, from = 0, trunk_seq = seq;                       // keys below `trunk` are the group's, from `from` on the sequence's own
  if (a.group_offsets) {
    from = kv_clip(a.prefix_lens[seq], a.pages.capacity);
    const int g = kv_find_sequence(a.group_offsets, a.n_groups, seq, lane);
    if (g < a.n_groups && a.group_offsets[g] >= 0 && a.group_offsets[g] <= seq) {
      trunk_seq = a.group_offsets[g];
      trunk = min(from, kv_clip(a.prefix_lens[trunk_seq], a.pages.capacity));
    }
  }
  float q[2] = {0.f, 0.f}, o[2] = {0.f, 0.f}, m = -INFINITY, l = 0.f;
  const T *qp = (const T *)(a.q.p + row * a.q.row + head * a.q.head);
  for (int i = 0; i < 2; ++i)
    if (lane + 64 * i < a.head_dim) q[i] = (float)qp[lane + 64 * i];
  const float scale = a.scale * kLog2e;
  for (int k0 = 0; k0 < sees; k0 += 64) {
    const int key = k0 + lane;
    const bool mine = key < sees && (key < trunk || key >= from);
    int64_t at_row = -1;
    if (mine) {
      at_row = kv_token_offset(a.pages, a.pages.table + (key < trunk ? trunk_seq : seq) * a.pages.table_stride, (uint32_t)key);
      if (at_row < 0) kv_fault(a.batch.faults, FLAME_KV_FAULT_PAGE);
    }
    const bool there = at_row >= 0;
    at_row += kvh * a.pages.head;
    float z = 0.f;
    for (int d = 0; d < a.head_dim; ++d) {
      const float x = there ? stored<T, FORM>(a.pages.k, a.k_scales, at_row, d) : 0.f;
      z += x * __shfl(d < 64 ? q[0] : q[1], d & 63);
    }
    z = there ? z * scale : -INFINITY;
    float top = z;
    for (int s = 32; s; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
    const float m_new = fmaxf(m, top), m_at = m_new == -INFINITY ? 0.f : m_new, keep = m == m_new ? 1.f : __builtin_amdgcn_exp2f(m - m_at);
    const float w = __builtin_amdgcn_exp2f(z - m_at);
    float sum = w;
    for (int s = 32; s; s >>= 1) sum += __shfl_xor(sum, s);
    l = l * keep + sum;
    o[0] *= keep;
    o[1] *= keep;
    m = m_new;
    for (uint64_t left = __builtin_amdgcn_ballot_w64(there); left; left &= left - 1) {
      const int j = __builtin_ctzll(left);
      const float wj = __shfl(w, j);
      const int64_t rj = __shfl((long long)at_row, j);
      for (int i = 0; i < 2; ++i)
        if (lane + 64 * i < a.head_dim) o[i] += wj * stored<T, FORM>(a.pages.v, a.v_scales, rj, lane + 64 * i);
    }
  }
  T *out = (T *)(a.out.p + row * a.out.row + head * a.out.head);
  const bool nothing = m == -INFINITY && l == 0.f;
  for (int i = 0; i < 2; ++i)
    if (lane + 64 * i < a.head_dim) out[lane + 64 * i] = kv_round<T>(nothing ? 0.f : o[i] / l);
}

}  // namespace

hipError_t launch_kvq_attention(const KvAttention &a, hipStream_t stream) {
  kv_with_type(a.dtype, [&](auto t) {
    kv_with_form(a.form, [&](auto form) {
      kvq_simple_kernel<decltype(t), decltype(form)::value><<<(unsigned)((a.batch.n_rows * a.n_q_heads + 3) / 4), 256, 0, stream>>>(a);
    });
  });
  return hipGetLastError();
}

}  // namespace flame
