// Rows into the cache held in 4 bits, quantised as they are written, and back.
#include <algorithm>

#include "batch.hpp"
#include "kv4.hpp"

namespace lp {

// ------------------------------------------------------------------ append

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}

// K and V of a row and head: 16 lanes, lane r with dims 32 j + 2 r and the next of
// every group j, so that a group's largest magnitude is four steps over the lanes
// and a lane's J bytes are V's as they lie; K's words are a transpose of bytes
// among four lanes.  A wave takes four consecutive rows of a head: of a prompt
// they fill whole lines.  q heads: a thread takes W rotary pairs.
template <typename T, int HD, int W>
__global__ __launch_bounds__(256) void kv4_append_kernel(QkvAppend a, T *__restrict__ q, uint8_t *__restrict__ cache,
                                                         int kv_wgs) {
  typedef Kv4<HD> F;
  constexpr int HALF = HD / 2, J = F::J;
  if ((int)blockIdx.x >= kv_wgs) {
    typedef float vec __attribute__((ext_vector_type(W)));
    typedef T out_vec __attribute__((ext_vector_type(W)));
    constexpr int TH = HALF / W;  // threads of a head
    const int per = (a.n_heads * TH + 255) / 256, b = blockIdx.x - kv_wgs;
    const int r = b / per, e = (b - r * per) * 256 + threadIdx.x, h = e / TH, i = e % TH * W;
    if (h >= a.n_heads) return;
    const float *x = a.qkv + r * a.ld + h * HD + i;
    const vec x0 = *(const vec *)x, x1 = *(const vec *)(x + HALF);
    const int pos = a.row_pos[r];
    if (pos < 0 || pos >= a.n_pos) return;
    const vec cs = *(const vec *)(a.rope_cos + (int64_t)pos * HALF + i);
    const vec sn = *(const vec *)(a.rope_sin + (int64_t)pos * HALF + i);
    out_vec y0, y1;
#pragma unroll
    for (int e = 0; e < W; ++e) {
      float r0, r1;
      rope_rotate(x0[e], x1[e], cs[e], sn[e], r0, r1);
      y0[e] = round_to<T>(r0);
      y1[e] = round_to<T>(r1);
    }
    T *dst = q + ((int64_t)r * a.n_heads + h) * HD + i;
    *(out_vec *)dst = y0;
    *(out_vec *)(dst + HALF) = y1;
    return;
  }
  const int heads = 2 * a.n_kv_heads, h = blockIdx.x % heads;
  const int row = blockIdx.x / heads * 16 + threadIdx.x / 16, l = threadIdx.x & 15;
  if (row >= a.rows) return;
  const int pos = a.row_pos[row];
  const int64_t entry = a.row_entry[row];
  const float *src = a.qkv + row * a.ld + (int64_t)(a.n_heads + h) * HD + 2 * l;
  f32x2_t x[J];
#pragma unroll
  for (int j = 0; j < J; ++j) x[j] = *(const f32x2_t *)(src + 32 * j);
  if (pos < 0 || pos >= a.n_pos || entry < 0 || entry >= a.n_blocks * KV_BLOCK) return;
  const bool is_k = h < a.n_kv_heads;
  if (is_k) {
#pragma unroll
    for (int j = 0; j < J / 2; ++j) {
      const f32x2_t cs = *(const f32x2_t *)(a.rope_cos + (int64_t)pos * HALF + 32 * j + 2 * l);
      const f32x2_t sn = *(const f32x2_t *)(a.rope_sin + (int64_t)pos * HALF + 32 * j + 2 * l);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float r0, r1;
        rope_rotate(x[j][e], x[j + J / 2][e], cs[e], sn[e], r0, r1);
        x[j][e] = r0;
        x[j + J / 2][e] = r1;
      }
    }
  }
  uint32_t word = 0;
  uint16_t own_scale = 0;  // lane j < J: group j's
#pragma unroll
  for (int j = 0; j < J; ++j) {
    uint32_t m = max(__float_as_uint(x[j][0]) & 0x7FFFFFFFu, __float_as_uint(x[j][1]) & 0x7FFFFFFFu);
    m = max(m, dpp_u32<0xB1>(m));   // quad_perm 1,0,3,2
    m = max(m, dpp_u32<0x4E>(m));   // quad_perm 2,3,0,1
    m = max(m, dpp_u32<0x141>(m));  // row_half_mirror
    m = max(m, dpp_u32<0x140>(m));  // row_mirror
    const float s = kv4_scale(m);
    if (l == j) own_scale = __builtin_bit_cast(uint16_t, (_Float16)s);
    word |= (kv4_code(x[j][0], s) | kv4_code(x[j][1], s) << 4) << (8 * j);
  }
  const int p = (int)(entry % KV_BLOCK);
  const int head = is_k ? h : h - a.n_kv_heads;
  uint8_t *dst = cache + (entry / KV_BLOCK * a.n_kv_heads + head) * (int64_t)F::BYTES;
  if (is_k) {
    // lane 4 i + b has byte b of word j of octet row i as its byte j
    const int b = l & 3;
    const uint32_t w0 = dpp_u32<0x00>(word), w1 = dpp_u32<0x55>(word), w2 = dpp_u32<0xAA>(word),
                   w3 = dpp_u32<0xFF>(word);
    const int sh = 8 * b;
    const uint32_t k = (w0 >> sh & 255u) | (w1 >> sh & 255u) << 8 | (w2 >> sh & 255u) << 16 | w3 >> sh << 24;
    if (b < J) *(uint32_t *)(dst + F::k_row(p) + l / 4 * 4 * J + 4 * b) = k;
    if (l < J) *(uint16_t *)(dst + F::k_scale(p, l)) = own_scale;
  } else {
    if constexpr (J == 4)
      *(uint32_t *)(dst + F::v_word(p, l)) = word;
    else
      *(uint16_t *)(dst + F::v_word(p, l / 2) + l % 2 * 2) = (uint16_t)word;
    if (l < J) *(uint16_t *)(dst + F::v_scale(p, l)) = own_scale;
  }
}

template <typename T, int HD, int W>
static void launch_append(const QkvAppend &a, T *q, uint8_t *cache, hipStream_t s) {
  const int per = (a.n_heads * (HD / 2 / W) + 255) / 256;
  const int kv_wgs = ceil_div(a.rows, 16) * 2 * a.n_kv_heads;
  kv4_append_kernel<T, HD, W><<<kv_wgs + a.rows * per, 256, 0, s>>>(a, q, cache, kv_wgs);
}

template <typename T>
void launch_kv4_append(const QkvAppend &a, T *q, uint8_t *cache, hipStream_t s) {
  // 16-byte reads of q heads where the rows and tables allow them, else 8-byte ones
  const bool w4 = a.ld % 4 == 0 && (((uintptr_t)a.qkv | (uintptr_t)a.rope_cos | (uintptr_t)a.rope_sin) & 15) == 0;
  if (a.head_dim == 128)
    w4 ? launch_append<T, 128, 4>(a, q, cache, s) : launch_append<T, 128, 2>(a, q, cache, s);
  else
    w4 ? launch_append<T, 64, 4>(a, q, cache, s) : launch_append<T, 64, 2>(a, q, cache, s);
}

// ------------------------------------------------------------------ read

// A thread takes one word (8 codes) of K or V of a row and head.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Read a, T *__restrict__ k, T *__restrict__ v) {
  typedef Kv4<HD> F;
  constexpr int J = F::J, WORDS = HD / 8;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int w = (int)(i % WORDS);
  const int64_t unit = i / WORDS;
  const int h = (int)(unit % (2 * a.n_kv_heads));
  const int64_t row = unit / (2 * a.n_kv_heads);
  if (row >= a.rows) return;
  const int64_t from = a.src_entry[row], to = a.dst_entry[row];
  if (from < 0 || from >= a.n_blocks * KV_BLOCK || to < 0 || to >= a.n_dst_blocks * KV_BLOCK) return;
  const bool is_k = h < a.n_kv_heads;
  const int head = is_k ? h : h - a.n_kv_heads, p = (int)(from % KV_BLOCK), d = (int)(to % KV_BLOCK);
  const uint8_t *src = a.cache + (from / KV_BLOCK * a.n_kv_heads + head) * (int64_t)F::BYTES;
  const int64_t base = (to / KV_BLOCK * a.n_kv_heads + head) * (int64_t)(KV_BLOCK * HD);
  const auto pairs = [](uint32_t c, f32x2_t *x) __attribute__((always_inline)) {
    x[0] = kv4_pair32<0>(c);
    x[1] = kv4_pair32<1>(c);
    x[2] = kv4_pair32<2>(c);
    x[3] = kv4_pair32<3>(c);
  };
  f32x2_t x[4];
  if (is_k) {
    const int o = w / J, j = w % J;
    pairs(*(const uint32_t *)(src + F::k_row(p) + 4 * w), x);
    const float s = (float)*(const _Float16 *)(src + F::k_scale(p, j));
    T *dst = k + base + d * HD + 32 * j + 8 * o;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      dst[2 * b] = round_to<T>(x[b][0] * s);
      dst[2 * b + 1] = round_to<T>(x[b][1] * s);
    }
  } else {
    pairs(*(const uint32_t *)(src + F::v_word(p, w)), x);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int j = b % J, r = (4 * w + b) / J;
      const float s = (float)*(const _Float16 *)(src + F::v_scale(p, j));
      T *dst = v + base + (int64_t)(32 * j + 2 * r) * KV_BLOCK + d;
      dst[0] = round_to<T>(x[b][0] * s);
      dst[KV_BLOCK] = round_to<T>(x[b][1] * s);
    }
  }
}

template <typename T>
void launch_kv4_read(const Kv4Read &a, T *k, T *v, hipStream_t s) {
  const int64_t threads = (int64_t)a.rows * 2 * a.n_kv_heads * (a.head_dim / 8);
  const unsigned wgs = (unsigned)((threads + 255) / 256);
  if (a.head_dim == 128)
    kv4_read_kernel<T, 128><<<wgs, 256, 0, s>>>(a, k, v);
  else
    kv4_read_kernel<T, 64><<<wgs, 256, 0, s>>>(a, k, v);
}

#define INST(T)                                                                        \
  template void launch_kv4_append<T>(const QkvAppend &, T *, uint8_t *, hipStream_t); \
  template void launch_kv4_read<T>(const Kv4Read &, T *, T *, hipStream_t);
INST(float)
INST(bf16_t)
INST(f16_t)
#undef INST

}  // namespace lp
