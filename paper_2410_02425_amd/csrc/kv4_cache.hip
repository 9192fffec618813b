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
// they fill whole lines.  q heads: a thread takes W rotary pairs.  Bound by memory:
// 4,200 rows of 8B heads in bf16, 109 MB read and 39 written, 31 us, 4.8 TB/s, the
// rate of a copy; 64 rows 3.7 us, latency.
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

// Whether rows q .. q + 3 go from four places side by side to four others, both
// on a multiple of four: their V words are then one 16-byte load, and a dim's
// four positions one store.
__device__ __forceinline__ bool kv4_quartet(const Kv4Read &a, int q) {
  if (q < 0 || q > a.rows - 4) return false;
  const int64_t s = a.src_entry[q], d = a.dst_entry[q];
  if (s < 0 || d < 0 || ((s | d) & 3) || s >= a.n_blocks * KV_BLOCK || d >= a.n_dst_blocks * KV_BLOCK) return false;
  bool run = true;
#pragma unroll
  for (int i = 1; i < 4; ++i) run = run && a.src_entry[q + i] == s + i && a.dst_entry[q + i] == d + i;
  return run;
}

// A K row's octets i of every group (J words), scaled: J runs of eight dims.
template <typename T, int J, typename W, typename S>
__device__ __forceinline__ void kv4_k_store(T *dst, const W &c, const S &s) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const f32x2_t y[4] = {kv4_pair32<0>(c[j]), kv4_pair32<1>(c[j]), kv4_pair32<2>(c[j]), kv4_pair32<3>(c[j])};
    vec8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = round_to<T>(y[e / 2][e % 2] * (float)s[j]);
    *(vec8 *)(dst + 32 * j) = o;
  }
}

// V's word w of four positions, scaled: eight dims of `there` positions from dst on.
// With `paired` the lane beside (^ 1) has the four positions beside: of a 16-bit
// type each stores eight positions of every other dim then, 16 bytes.
template <typename T, int J, typename S>
__device__ __forceinline__ void kv4_v_store(T *dst, const u32x4_tt &x, const S *s, int w, int there, bool paired) {
  typedef T vec4 __attribute__((ext_vector_type(4)));
  // pairs of positions: bytes of even dims, of odd ones
  uint32_t lo[2], hi[2];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    lo[y] = (x[2 * y] & 0x0F0F0F0Fu) | ((x[2 * y + 1] << 4) & 0xF0F0F0F0u);
    hi[y] = ((x[2 * y] >> 4) & 0x0F0F0F0Fu) | (x[2 * y + 1] & 0xF0F0F0F0u);
  }
  auto byte = [&](auto b_c) __attribute__((always_inline)) {
    constexpr int b = decltype(b_c)::value, j = b % J;
    const int d = 32 * j + 2 * ((4 * w + b) / J);
    vec4 o[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const f32x2_t y0 = kv4_pair32<b>(z ? hi[0] : lo[0]), y1 = kv4_pair32<b>(z ? hi[1] : lo[1]);
      o[z] = vec4{round_to<T>(y0[0] * (float)s[j][0]), round_to<T>(y0[1] * (float)s[j][1]),
                  round_to<T>(y1[0] * (float)s[j][2]), round_to<T>(y1[1] * (float)s[j][3])};
    }
    if constexpr (sizeof(T) == 2)
      if (paired) {
        typedef uint32_t two_t __attribute__((ext_vector_type(2)));
        const bool odd = threadIdx.x & 1;
        const two_t o0 = __builtin_bit_cast(two_t, o[0]), o1 = __builtin_bit_cast(two_t, o[1]), send = odd ? o0 : o1;
        const two_t got = {dpp_u32<0xB1>(send[0]), dpp_u32<0xB1>(send[1])}, low = odd ? got : o0, high = odd ? o1 : got;
        const u32x4_tt v = {low[0], low[1], high[0], high[1]};
        __builtin_nontemporal_store(v, (u32x4_tt *)(dst + d * KV_BLOCK + (odd ? KV_BLOCK - 4 : 0)));
        return;
      }
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      T *to = dst + (d + z) * KV_BLOCK;
      if (there >= 4) {
        __builtin_nontemporal_store(o[z], (vec4 *)to);
      } else {
        for (int e = 0; e < there; ++e) to[e] = o[z][e];
      }
    }
  };
  byte(std::integral_constant<int, 0>());
  byte(std::integral_constant<int, 1>());
  byte(std::integral_constant<int, 2>());
  byte(std::integral_constant<int, 3>());
}

// A workgroup takes about ROWS rows of a head.  It begins at the first of its ROWS
// places in the list that goes to a multiple of ROWS, if there is one, and ends
// where the next workgroup begins: rows in the order of their positions are then
// taken block by block, and no line of V is written by two workgroups.
//   * Rows that go from the beginning of a block to the beginning of one, place by
//     place: all loads are requested at once, four threads a row of K, a thread
//     a word of V of four positions, so that a wave's stores are whole lines of
//     dims' positions.
//   * Others: quartets (rows that go from four places to four) are listed first
//     and stored alike, rows of no quartet go one by one.
// Bound by memory, which is nearly all writes: 16 contexts of 1,500 of 13B heads in
// bf16, 630 MB, 144 us, 4.4 TB/s (K and V in turn with lists for all rows 231, with
// workgroups at blocks' beginnings 185, the loads at once 153, V past the cache 149,
// 16 bytes of V a store 147, K through the cache 144).
template <typename T, int HD, int ROWS>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Read a, T *__restrict__ k, T *__restrict__ v) {
  typedef Kv4<HD> F;
  constexpr int J = F::J, WORDS = HD / 8;
  typedef uint32_t words_t __attribute__((ext_vector_type(J)));
  typedef _Float16 scales_t __attribute__((ext_vector_type(J)));
  typedef _Float16 half4 __attribute__((ext_vector_type(4)));
  __shared__ int first[ROWS], counts[2];  // quartets' first rows from the front, single rows from the back
  const int t = threadIdx.x, lane = t & 63;
  const int tile = blockIdx.x / a.n_kv_heads, h = blockIdx.x - tile * a.n_kv_heads;
  const int64_t src_end = a.n_blocks * KV_BLOCK, dst_end = a.n_dst_blocks * KV_BLOCK;
  auto src_of = [&](uint64_t from) __attribute__((always_inline)) {
    return a.cache + (from / KV_BLOCK * a.n_kv_heads + h) * F::BYTES;
  };
  auto dst_of = [&](uint64_t to) __attribute__((always_inline)) {
    return (int64_t)((to / KV_BLOCK * a.n_kv_heads + h) * (KV_BLOCK * HD));
  };
  // the entries of this workgroup's places and of the next one's
  const int at = tile * ROWS;
  int64_t s[2], d[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int r = at + x * ROWS + lane;
    const bool there = lane < ROWS && r < a.rows;
    s[x] = there ? a.src_entry[r] : -1;
    d[x] = there ? a.dst_entry[r] : -1;
  }
  const uint64_t b0 = __ballot((d[0] & (ROWS - 1)) == 0), b1 = __ballot((d[1] & (ROWS - 1)) == 0);
  const int skip = tile && b0 ? __builtin_ctzll(b0) : 0;
  int r0 = at + skip;
  const int end = min(at + ROWS + (b1 ? __builtin_ctzll(b1) : 0), a.rows);
  if (ROWS == 64 && r0 < end) {
    const int n = min(ROWS, end - r0);
    const uint64_t s0 = readlane_u64(s[0], skip), d0 = readlane_u64(d[0], skip);
    bool run = true;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int i = x * ROWS + lane - skip;  // of the rows from r0 on
      run = run && (i < 0 || i >= n || (s[x] == (int64_t)s0 + i && d[x] == (int64_t)d0 + i));
    }
    if (__all(run) && ((s0 | d0) & 63) == 0 && s0 < (uint64_t)src_end && d0 < (uint64_t)dst_end) {
      const uint8_t *src = src_of(s0);
      const int row = t / 4, i = t % 4;
      const int q = t % 16, w = t / 16;
      int there = w < WORDS ? n - 4 * q : 0;
      // four positions that go on in the next workgroup's places are stored here, like any quartet
      if (there > 0 && there < 4 && kv4_quartet(a, r0 + 4 * q)) there = 4;
      words_t kc;
      scales_t ks;
      u32x4_tt x;
      half4 vs[J];
      if (row < n) {
        kc = *(const words_t *)(src + F::k_row(row) + 4 * J * i);
        ks = *(const scales_t *)(src + F::k_scale(row, 0));
      }
      if (there > 0) {
        x = *(const u32x4_tt *)(src + F::v_word(4 * q, w));
#pragma unroll
        for (int j = 0; j < J; ++j) vs[j] = *(const half4 *)(src + F::v_scale(4 * q, j));
      }
      if (row < n) kv4_k_store<T, J>(k + dst_of(d0) + row * HD + 8 * i, kc, ks);
      if (there > 0) kv4_v_store<T, J>(v + dst_of(d0) + 4 * q, x, vs, w, there, n >= 4 * (q | 1) + 4);
      r0 += n;
    }
  }
  for (; r0 < end; r0 += ROWS) {
    const int n = min(ROWS, end - r0);
    if (t < 64) {
      const int r = r0 + t;
      const bool lead = t < n && kv4_quartet(a, r);
      bool single = false;
      if (!lead && t < n) {
        const int64_t from = a.src_entry[r], to = a.dst_entry[r];
        single = from >= 0 && from < src_end && to >= 0 && to < dst_end && !kv4_quartet(a, r - (int)(to & 3));
      }
      const uint64_t leads = __ballot(lead), singles = __ballot(single), below = (1ull << t) - 1;
      if (lead) first[__popcll(leads & below)] = r;
      if (single) first[ROWS - 1 - __popcll(singles & below)] = r;
      if (t == 0) counts[0] = __popcll(leads), counts[1] = __popcll(singles);
    }
    if (t / 4 < n) {
      const int i = t % 4;
      const int64_t from = a.src_entry[r0 + t / 4], to = a.dst_entry[r0 + t / 4];
      if (from >= 0 && from < src_end && to >= 0 && to < dst_end) {
        const uint8_t *src = src_of(from);
        const int p = (int)(from % KV_BLOCK);
        const words_t c = *(const words_t *)(src + F::k_row(p) + 4 * J * i);
        const scales_t ks = *(const scales_t *)(src + F::k_scale(p, 0));
        kv4_k_store<T, J>(k + dst_of(to) + (int)(to % KV_BLOCK) * HD + 8 * i, c, ks);
      }
    }
    __syncthreads();
    const int quartets = counts[0], singles = counts[1];
    for (int i = t; i < ROWS / 4 * WORDS; i += 256) {
      const int q = i % (ROWS / 4), w = i / (ROWS / 4);
      if (q >= quartets) continue;
      const uint64_t from = a.src_entry[first[q]], to = a.dst_entry[first[q]];
      const uint8_t *src = src_of(from);
      const int p = (int)(from % KV_BLOCK);
      half4 vs[J];
#pragma unroll
      for (int j = 0; j < J; ++j) vs[j] = *(const half4 *)(src + F::v_scale(p, j));
      kv4_v_store<T, J>(v + dst_of(to) + (int)(to % KV_BLOCK), *(const u32x4_tt *)(src + F::v_word(p, w)), vs, w, 4,
                        false);
    }
    for (int i = t; i < singles * WORDS; i += 256) {
      // lanes are rows, whose places may be side by side
      const int w = i / singles, r = first[ROWS - 1 - (i - w * singles)];
      const uint64_t from = a.src_entry[r], to = a.dst_entry[r];
      const uint8_t *src = src_of(from);
      const int p = (int)(from % KV_BLOCK);
      const uint32_t c = *(const uint32_t *)(src + F::v_word(p, w));
      const f32x2_t y[4] = {kv4_pair32<0>(c), kv4_pair32<1>(c), kv4_pair32<2>(c), kv4_pair32<3>(c)};
      T *dst = v + dst_of(to) + (int)(to % KV_BLOCK);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float f = (float)*(const _Float16 *)(src + F::v_scale(p, b % J));
        const int dim = 32 * (b % J) + 2 * ((4 * w + b) / J);
        dst[dim * KV_BLOCK] = round_to<T>(y[b][0] * f);
        dst[(dim + 1) * KV_BLOCK] = round_to<T>(y[b][1] * f);
      }
    }
    __syncthreads();  // the lists have been used
  }
}

template <typename T>
void launch_kv4_read(const Kv4Read &a, T *k, T *v, hipStream_t s) {
  const auto run = [&](auto hd, auto rows) {
    constexpr int HD = decltype(hd)::value, ROWS = decltype(rows)::value;
    const unsigned wgs = (unsigned)ceil_div(a.rows, ROWS) * (unsigned)a.n_kv_heads;
    kv4_read_kernel<T, HD, ROWS><<<wgs, 256, 0, s>>>(a, k, v);
  };
  typedef std::integral_constant<int, 64> c64;
  typedef std::integral_constant<int, 16> c16;
  const bool large = (int64_t)ceil_div(a.rows, 64) * a.n_kv_heads >= 512;
  if (a.head_dim == 128)
    large ? run(std::integral_constant<int, 128>(), c64()) : run(std::integral_constant<int, 128>(), c16());
  else
    large ? run(c64(), c64()) : run(c64(), c16());
}

#define INST(T)                                                                        \
  template void launch_kv4_append<T>(const QkvAppend &, T *, uint8_t *, hipStream_t); \
  template void launch_kv4_read<T>(const Kv4Read &, T *, T *, hipStream_t);
INST(float)
INST(bf16_t)
INST(f16_t)
#undef INST

}  // namespace lp
