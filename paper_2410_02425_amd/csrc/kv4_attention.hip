// Attention over the cache held in 4 bits.
#include <algorithm>

#include "batch.hpp"
#include "kv4.hpp"

namespace lp {

// A wave per (row, query head): its lanes are the keys of a block for the scores,
// the dims for the values.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_attention_kernel(const T *__restrict__ q, T *__restrict__ out,
                                                            PrefixBatch b) {
  typedef Kv4<HD> F;
  constexpr int J = F::J, DPL = HD / 64;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t rh = (int64_t)blockIdx.x * 4 + wave;
  const int t = (int)(rh / b.n_heads), h = (int)(rh - (int64_t)t * b.n_heads);
  if (t >= b.rows) return;
  int seq = -1, i = 0;
  if (!b.seq_start) {
    seq = t;
  } else {
    for (int j = 0; j < b.n_seq; ++j) {
      int start, n;
      seq_rows(b, j, start, n);
      if (t >= start && t < start + n) seq = j, i = t - start;
    }
    if (seq < 0) return;
  }
  const int ctx = i < b.max_new ? row_ctx(b, seq, i) : 0;
  const int slot = b.seq_slot[seq];
  const uint8_t *cache = (const uint8_t *)b.kv.k;
  const float scale = rsqrtf((float)HD);
  const T *qr = q + rh * HD;
  float m = -INFINITY, sum = 0.f, o[DPL];
#pragma unroll
  for (int d = 0; d < DPL; ++d) o[d] = 0.f;
  for (int e = 0; e * KV_BLOCK < ctx; ++e) {
    const int id = e < b.kv.max_blocks ? b.kv.block_table[(int64_t)slot * b.kv.max_blocks + e] : -1;
    if (id < 0 || id >= b.kv.n_blocks) continue;
    const uint8_t *blk = cache + ((int64_t)id * b.kv.n_kv_heads + h / (b.n_heads / b.kv.n_kv_heads)) * F::BYTES;
    const int keys = min(ctx - e * KV_BLOCK, KV_BLOCK);
    float s = 0.f;
    for (int w = 0; w < HD / 8; ++w) {
      const int o8 = w / J, j = w % J;
      const uint32_t c = *(const uint32_t *)(blk + F::k_row(lane) + 4 * w);
      const f32x2_t x[4] = {kv4_pair32<0>(c), kv4_pair32<1>(c), kv4_pair32<2>(c), kv4_pair32<3>(c)};
      float part = 0.f;
      for (int d = 0; d < 8; ++d) part = fmaf(Act<T>::ld(qr[32 * j + 8 * o8 + d]), x[d / 2][d % 2], part);
      s = fmaf(part, (float)*(const _Float16 *)(blk + F::k_scale(lane, j)), s);
    }
    s = lane < keys ? s * scale : -INFINITY;
    const float nm = fmaxf(m, wave_max(s)), m0 = nm == -INFINITY ? 0.f : nm;
    const float corr = m == nm ? 1.f : expf(m - nm), p = expf(s - m0);
    m = nm;
    sum = sum * corr + wave_sum(p);
#pragma unroll
    for (int d = 0; d < DPL; ++d) o[d] *= corr;
    for (int k = 0; k < keys; ++k) {
      const float pk = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(p), k));
#pragma unroll
      for (int d = 0; d < DPL; ++d) {
        const int dim = d * 64 + lane, j = dim / 32, r = dim % 32 / 2, byte = J * r + j;
        const uint32_t c = *(const uint8_t *)(blk + F::v_word(k, byte / 4) + byte % 4);
        const float x = kv4_pair32<0>(c >> (dim % 2 * 4))[0];
        o[d] = fmaf(pk, x * (float)*(const _Float16 *)(blk + F::v_scale(k, j)), o[d]);
      }
    }
  }
#pragma unroll
  for (int d = 0; d < DPL; ++d) out[rh * HD + d * 64 + lane] = round_to<T>(sum == 0.f ? 0.f : o[d] / sum);
}

size_t kv4_attention_ws_bytes(bool, int, int, int, int, int) { return 0; }

template <typename T>
bool launch_kv4_attention(const T *q, T *out, const PrefixBatch &b, float *, hipStream_t s) {
  const int64_t wgs = ((int64_t)b.rows * b.n_heads + 3) / 4;
  if (wgs >= 1 << 23) return false;  // a launch has fewer than 2^32 threads
  if (b.kv.head_dim == 128)
    kv4_attention_kernel<T, 128><<<(unsigned)wgs, 256, 0, s>>>(q, out, b);
  else
    kv4_attention_kernel<T, 64><<<(unsigned)wgs, 256, 0, s>>>(q, out, b);
  return true;
}

#define INST(T) template bool launch_kv4_attention<T>(const T *, T *, const PrefixBatch &, float *, hipStream_t);
INST(float)
INST(bf16_t)
INST(f16_t)
#undef INST

}  // namespace lp
