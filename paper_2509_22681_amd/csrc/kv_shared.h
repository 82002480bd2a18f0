// Attention of groups of sequences over histories that they share, and over their own tokens behind them (flame_kv_shared, flame_kvq_shared).
//
// A row's softmax is cut at the end of what its sequence shares.  Row tiles (kv_flash.h) take the rows of a whole group over the history, cut into parts along the keys where tiles are few, so that a history
// is read once for 128 rows (tokens times heads of a key head) and not once for each sequence; split attention (kv_split.h) takes each sequence's rows over its own tokens; both leave maxima,
// sums and unnormalised rows, which the kernel here joins, planes in their order: the same call gives the same bits.
#pragma once
#include "kv_flash.h"
#include "kv_split.h"

namespace flame {

namespace {

// Row tiles over the histories in the first workgroups, split attention over the sequences' own keys in those behind them.  Own keys fill the places that the tiles leave, and where those take nearly all of the
// chip's, as parts of equal length do, begin when tiles end (96 sequences with 20-800 tokens of their own behind 8 histories of 2000-12000, 32/8 heads of 128, bf16: tiles alone 54 us, own keys alone 45, both 100).
// The registers are those of the two together at the row tiles' bounds: over values 128 features spill 19 (fp32 22) of 256 and 16-bit heads of 64 with one
// wavefront to 32 rows 7 of 168, over codes heads of 32 spill 13 to 29 and heads of 64 up to 10 (see flash_workgroups).
template <typename T, int DH, int KP, int FORM>
__global__ __launch_bounds__(256, (flash_workgroups<T, DH, KP>())) void kv_shared_kernel(KvAttention a, float *__restrict__ split_parts) {
  const unsigned tiles = gridDim.x - a.split_blocks;
  if (blockIdx.x < tiles) flash_rows<T, DH, true, KP, FORM, true>(a, blockIdx.x, tiles);
  else split_units<T, DH, FORM, true>(a, split_parts, blockIdx.x - tiles, a.split_blocks * 4);
}

// Bound by latency and by the planes, which it reads once (8 us in that call).  DH / 4 lanes a head, and a workgroup 256 / (DH / 4) heads of a row.
template <typename T, int DH, int KP>
__global__ __launch_bounds__(256) void kv_shared_join_kernel(KvAttention a, const float *__restrict__ split_parts) {
  constexpr int KW = KP * key_block<T, DH, KP>(), QT = kFlashRows / KP;
  constexpr int H = 256 / (DH / 4);
  const int lane = threadIdx.x & 63;
  if (blockIdx.x == 0 && a.batch.faults) {
    if (threadIdx.x == 0 && (a.group_offsets[0] != 0 || a.group_offsets[a.n_groups] != a.batch.n_seqs)) kv_fault(a.batch.faults, FLAME_KV_FAULT_OFFSET);
    for (int g = threadIdx.x; g < a.n_groups; g += 256) kv_report_offsets(a.group_offsets[g], a.group_offsets[g + 1], a.batch.n_seqs, a.batch.faults);
    for (int b = threadIdx.x; b < a.batch.n_seqs; b += 256) {
      int lo = 0, hi = a.n_groups;                                // the first group that ends behind the sequence
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.group_offsets[mid + 1] > b) hi = mid;
        else lo = mid + 1;
      }
      const int b0 = lo < a.n_groups ? a.group_offsets[lo] : b;
      if (b0 >= 0 && b0 < b && kv_clip(a.prefix_lens[b], a.pages.capacity) > kv_clip(a.prefix_lens[b0], a.pages.capacity)) kv_fault(a.batch.faults, FLAME_KV_FAULT_LENGTH);
    }
  }
  const int blocks = (a.n_q_heads + H - 1) / H;
  const int64_t q_row = blockIdx.x / blocks;
  const int head = blockIdx.x % blocks * H + threadIdx.x / (DH / 4), f = threadIdx.x % (DH / 4) * 4;
  int seq = (int)q_row;
  int64_t first = q_row;
  if (a.batch.offsets) {
    seq = kv_find_sequence(a.batch.offsets, a.batch.n_seqs, q_row, lane);
    if (seq >= a.batch.n_seqs) return;
    first = a.batch.offsets[seq];
    if (first < 0 || q_row < first || q_row >= a.batch.offsets[seq + 1]) return;
  }
  // parts of the history
  int parts = 0;
  int64_t part_at = 0, step = a.batch.n_rows * a.n_q_heads;       // the first one's row, and from one to the next
  const int64_t from = q_row * a.n_q_heads + head;
  const int group = a.n_q_heads / a.n_kv_heads, kvh = head / group;
  int2 of = {0, 0};
  if (head < a.n_q_heads) of = ((const int2 *)(split_parts + split_parts_floats(DH)))[from];
  const int g = kv_find_sequence(a.group_offsets, a.n_groups, seq, lane);
  if (g < a.n_groups) {
    const int b0 = a.group_offsets[g];
    if (b0 >= 0 && b0 <= seq) {
      const int history = kv_clip(a.prefix_lens[b0], a.pages.capacity);
      if (history > 0 && a.splits == 0) {
        const int64_t group_first = a.batch.offsets ? a.batch.offsets[b0] : b0;
        const int2 cut = a.cuts[g];
        const int64_t row = (q_row - group_first) * group + head % group;
        parts = cut.y;
        part_at = ((cut.x + row / QT * parts) * a.n_kv_heads + kvh) * QT + row % QT;
        step = (int64_t)a.n_kv_heads * QT;
        // (offsets of more than 64 sequences that are none may claim other rows than were counted)
        if (row < 0 || parts < 0 || part_at + (parts - 1) * step >= a.part_rows) parts = 0;
      } else if (history > 0) {
        parts = flash_parts<KW>(history, a.splits).parts;
        part_at = from;
      }
    }
  }
  if (head >= a.n_q_heads) return;
  const float2 *state = kv_shared_state(a) + part_at;
  const float *sums = a.parts + part_at * DH + f;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  const auto add = [&](float mw, float lw, f32x4 ow) {
    const float m_new = fmaxf(m, mw), m_at = m_new == -INFINITY ? 0.f : m_new;
    const float keep = m == m_new ? 1.f : __builtin_amdgcn_exp2f(m - m_at), take = mw == m_new ? 1.f : __builtin_amdgcn_exp2f(mw - m_at);
    l = l * keep + lw * take;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = o[i] * keep + ow[i] * take;
    m = m_new;
  };
#pragma unroll 8
  for (int p = 0; p < parts; ++p) {
    const float2 ml = state[p * step];
    add(ml.x, ml.y, *(const f32x4 *)(sums + p * step * DH));
  }
  // the sequence's own keys: one plane, or parts of wavefronts
  if (of.x >= 0 && of.x >> 1 < of.y && of.y < split_workers(DH)) {
    const int r = (int)(((q_row - first) * group + head % group) % kRows);
    for (int w = of.x >> 1; w <= of.y; ++w) {
      const float *part = split_parts + ((int64_t)w * 2 + (w == of.x >> 1 ? of.x & 1 : 0)) * split_part_floats(DH);
      add(part[r], part[kRows + r], *(const f32x4 *)(part + 2 * kRows + r * DH + f));
    }
  } else {
    const float2 ml = kv_own_state(a)[from];
    add(ml.x, ml.y, *(const f32x4 *)(a.own + from * DH + f));
  }
  // A row whose logits are all -infinity has zeros, though its weights of zero may have met infinite values or NaN.  (NaN logits leave l NaN.)
  const bool nothing = m == -INFINITY && l == 0.f;
  const float inv = 1.f / l;
  typedef T out4 __attribute__((ext_vector_type(4)));
  out4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = kv_round<T>(nothing ? 0.f : o[i] * inv);
  *(out4 *)(a.out.p + q_row * a.out.row + head * a.out.head + f * sizeof(T)) = y;
}

template <int FORM> hipError_t launch_shared(const KvAttention &call, const KvSharedRoute &route, void *split_workspace, hipStream_t stream) {
  hipError_t e = hipErrorInvalidValue;
  flash_with_shape(call, route.wavefronts, [&](auto t, auto width, auto kp) {
    using T = decltype(t);
    constexpr int DH = decltype(width)::value, KP = decltype(kp)::value, kBytes = flash_lds_bytes<T, DH, KP>();
    if constexpr (DH < 128 || KP < 4) {                           // (kv_shared_route)
    static std::atomic<uint64_t> raised{0};
    e = raise_lds_limit(reinterpret_cast<const void *>(&kv_shared_kernel<T, DH, KP, FORM>), kBytes, raised);
    if (e != hipSuccess) return;
    KvAttention a = call;
    a.split_blocks = split_workers(DH) / 4;
    const int64_t tiles = a.n_groups ? route.slots * a.n_kv_heads * std::max(a.splits, 1) : 0;
    kv_shared_kernel<T, DH, KP, FORM><<<(unsigned)(a.split_blocks + tiles), 256, kBytes, stream>>>(a, (float *)split_workspace);
    kv_shared_join_kernel<T, DH, KP><<<(unsigned)(a.batch.n_rows * ((a.n_q_heads * (DH / 4) + 255) / 256)), 256, 0, stream>>>(a, (const float *)split_workspace);
    e = hipGetLastError();
    }
  });
  return e;
}

}  // namespace

}  // namespace flame
