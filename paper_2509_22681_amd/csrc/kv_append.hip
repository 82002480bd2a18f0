// Keys and values of new tokens into a paged cache, keys and queries rotated by their positions on the way.
//
// Bound by memory: every row is read once and written once, and the arithmetic is six operations per pair of features.  16 ragged prompts of
// 64..4096 tokens (32/8 heads of 128, bf16, 626 MB in and out) take 122 us, 5.1 TB/s, which a plain copy of 1 GiB reaches; one token each of 32
// sequences takes 5 us, a launch and a few dependent loads.  One
// wavefront takes one token with all its heads, because the heads share the token's page, position and angles: lane j makes
// the cosine and sine of pair j once (up to 64 pairs: one per lane) and leaves them in LDS, from where the rows' lanes read theirs.  A row of
// D features is D * size / 32 lanes with two 16-byte pieces each: with pairs (j, j + r/2) the pieces hold the two features of every pair, with
// neighbours as pairs each piece has its own.
#include "kv_rotate.h"

namespace flame {

namespace {

constexpr int kTokensPerBlock = 4;

template <typename T> struct Piece { typedef T vec __attribute__((ext_vector_type(16 / sizeof(T)))); };

template <typename T>
__global__ __launch_bounds__(64 * kTokensPerBlock) void kv_append_kernel(KvBatch batch, KvPages pages, KvRows k, KvRows v, KvRows q, KvRows q_out, KvRotation rot,
                                                                       int n_q, int n_kv, int head_dim) {
  typedef typename Piece<T>::vec vec;
  constexpr int E = 16 / sizeof(T);
  __shared__ float2 turn_s[kTokensPerBlock][kMaxRotationPairs];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (batch.faults)
    for (int64_t b = (int64_t)blockIdx.x * (64 * kTokensPerBlock) + threadIdx.x; b < batch.n_seqs; b += (int64_t)gridDim.x * (64 * kTokensPerBlock))
      kv_report_offsets(batch.offsets[b], batch.offsets[b + 1], batch.n_rows, batch.faults);
  const int64_t token = (int64_t)blockIdx.x * kTokensPerBlock + wave;
  if (token >= batch.n_rows) return;
  const int seq = kv_find_sequence(batch.offsets, batch.n_seqs, token, lane);
  if (seq >= batch.n_seqs) return;                                        // behind the last sequence
  const int64_t first = batch.offsets[seq], end = batch.offsets[seq + 1];
  if (first < 0 || token < first || token >= end) return;                 // ahead of the first one, or offsets that are none
  const int64_t position = (int64_t)batch.kv_lens[seq] - end + token;
  const bool placed = position >= 0 && position < pages.capacity;
  int64_t to = -1;
  if (placed) to = kv_token_offset(pages, pages.table + seq * pages.table_stride, (uint32_t)position);
  if (to < 0 && lane == 0) kv_fault(batch.faults, placed ? FLAME_KV_FAULT_PAGE : FLAME_KV_FAULT_LENGTH);
  if (lane < rot.pairs) turn_s[wave][lane] = cos_sin_of_turn(rot.turns[lane] * (uint64_t)position);
  // (a wavefront reads only what it wrote itself)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int per_row = head_dim / (2 * E);                                 // lanes of a row
  const int slot = lane & (per_row - 1), row0 = lane / per_row, rows = 64 / per_row;
  // the lane's two pieces: the two halves of E pairs, or two neighbouring pieces
  const int r = 2 * rot.pairs, half_pieces = r / (2 * E);
  const bool split = !rot.interleaved && slot < half_pieces;
  const int c0 = split ? slot : 2 * slot, c1 = split ? slot + half_pieces : 2 * slot + 1;
  const float2 *turn = turn_s[wave];
  auto rotate = [&](vec &a, vec &b) {
    if (split) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float2 cs = turn[slot * E + i];
        const float x = (float)a[i], y = (float)b[i];
        a[i] = kv_round<T>(x * cs.x - y * cs.y);
        b[i] = kv_round<T>(x * cs.y + y * cs.x);
      }
    } else if (rot.interleaved && slot < half_pieces) {
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        const float2 ca = turn[(c0 * E + i) >> 1], cb = turn[(c1 * E + i) >> 1];
        const float x = (float)a[i], y = (float)a[i + 1], z = (float)b[i], w = (float)b[i + 1];
        a[i] = kv_round<T>(x * ca.x - y * ca.y);
        a[i + 1] = kv_round<T>(x * ca.y + y * ca.x);
        b[i] = kv_round<T>(z * cb.x - w * cb.y);
        b[i + 1] = kv_round<T>(z * cb.y + w * cb.x);
      }
    }
  };
  if (to >= 0) {
    for (int h = row0; h < n_kv; h += rows) {
      const char *ks = k.p + token * k.row + h * k.head, *vs = v.p + token * v.row + h * v.head;
      vec a = *(const vec *)(ks + c0 * 16), b = *(const vec *)(ks + c1 * 16);
      const vec va = *(const vec *)(vs + c0 * 16), vb = *(const vec *)(vs + c1 * 16);
      rotate(a, b);
      char *kd = pages.k + to + h * pages.head, *vd = pages.v + to + h * pages.head;
      *(vec *)(kd + c0 * 16) = a;
      *(vec *)(kd + c1 * 16) = b;
      *(vec *)(vd + c0 * 16) = va;
      *(vec *)(vd + c1 * 16) = vb;
    }
  }
  if (q.p && position >= 0) {
    for (int h = row0; h < n_q; h += rows) {
      const char *qs = q.p + token * q.row + h * q.head;
      vec a = *(const vec *)(qs + c0 * 16), b = *(const vec *)(qs + c1 * 16);
      rotate(a, b);
      char *qd = q_out.p + token * q_out.row + h * q_out.head;
      *(vec *)(qd + c0 * 16) = a;
      *(vec *)(qd + c1 * 16) = b;
    }
  }
}

}  // namespace

hipError_t launch_kv_append(const KvBatch &batch, const KvPages &pages, const KvRows &k, const KvRows &v, const KvRows *q, const KvRows *q_out,
                            const KvRotation &rotation, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype, hipStream_t stream) {
  const unsigned blocks = (unsigned)((batch.n_rows + kTokensPerBlock - 1) / kTokensPerBlock);
  kv_with_type(dtype, [&](auto t) {
    kv_append_kernel<decltype(t)><<<blocks, 64 * kTokensPerBlock, 0, stream>>>(batch, pages, k, v, q ? *q : KvRows{}, q ? *q_out : KvRows{}, rotation, n_q_heads, n_kv_heads, head_dim);
  });
  return hipGetLastError();
}

}  // namespace flame
