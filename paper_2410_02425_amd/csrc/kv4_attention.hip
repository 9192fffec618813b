// Attention over the cache held in 4 bits.
//
// Codes go to the matrix cores without their scales, exact in 16 bits:
//   score(t) = sum over groups j of sk[t][j] (q_j . c_tj): one MFMA over 32 dims is
//   a group's product, the scale multiplies its fp32 result;
//   out[d] = sum over t of (p_t sv[t][j]) c[t][d], d in group j: the scale goes into
//   the weight before that is rounded for the MFMA.
// So no value is dequantised, codes are finite whatever a stale place holds, and a
// row's mask clears its own weights alone.
// fp32: q and the weights as three bf16 parts each (8 bits and 8 and 8), products
// with codes exact, all sums fp32.
#include <algorithm>
#include <type_traits>

#include "batch.hpp"
#include "kv4.hpp"

namespace lp {

struct Kv4Args {
  PrefixBatch b;
  int G;                // query heads of a KV head
  int units;            // row tiles
  int splits, sblk;     // splits of a tile's blocks, blocks of a split
  Divisor by_g, by_hkv, by_units, by_per, by_sblk;
  float *po, *pml;      // partial o [rows][n_heads][splits][hd], (m, l) [rows][n_heads][splits][2]
};
// Blocks of a part: a context's are shared out evenly, by STEP, among as many parts as
// sblk asks for, so that items end together (8B heads, 48 rows of 1,500 tokens 31.9 us for
// 35.4, 64 of 2,300 48.5 for 49.5, 64 of 1,500 39.1 for 38.2).
template <int STEP>
__device__ __forceinline__ void part_blocks(const Kv4Args &a, int part, int top, int &e0, int &e1) {
  const int blocks = (top + KV_BLOCK - 1) / KV_BLOCK;
  int each = blocks;
  if (a.splits > 1 && blocks > a.sblk) {
    const unsigned parts = div_by(blocks + a.sblk - 1, a.by_sblk);
    each = (int)((blocks + parts - 1) / parts);
    each = min((each + STEP - 1) / STEP * STEP, a.sblk);
  }
  e0 = part * each;
  e1 = min(e0 + each, blocks);
}
// A part's m is the largest score before the scale 1/sqrt(hd), its weights are
// 2^((score - m) c2).
constexpr int KV4_UP = 15;  // fp16 weights of the rows' kernel go up to 2^15
template <int HD>
constexpr float KV4_C2 = (HD == 64 ? 0.125f : 0.08838834764831845f) * 1.44269504088896341f;

typedef unsigned int u32x2_tt __attribute__((ext_vector_type(2)));
typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));

// Eight codes (a word, the low half first) as an MFMA operand.
template <typename T>
__device__ __forceinline__ typename Mfma<T>::v8 codes8(uint32_t w) {
  const u32x4_tt v = {kv4_pair16<T, 0>(w), kv4_pair16<T, 1>(w), kv4_pair16<T, 2>(w), kv4_pair16<T, 3>(w)};
  return __builtin_bit_cast(typename Mfma<T>::v8, v);
}

// Two products of fp32 weights and fp16 scales (x the low half of sv's, y the high
// one's), each rounded once to fp16.  With 0 added a product is a fused step, which
// this GPU has with these types in one instruction; the compiler picks it, and so
// keeps the wait states before the MFMA that reads it.
__device__ __forceinline__ uint32_t mul_pair(float x, float y, uint32_t sv) {
  const half2_t s = __builtin_bit_cast(half2_t, sv);
  const half2_t d = {(_Float16)fmaf(x, (float)s[0], 0.f), (_Float16)fmaf(y, (float)s[1], 0.f)};
  return __builtin_bit_cast(uint32_t, d);
}

// Maximum / sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float quads_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return half_swap_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quads_sum(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return half_swap_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Up to 16 packed rows of a KV head over a range of blocks, on 16x16x32 MFMAs; the
// workgroup's waves take blocks in turn, each with LDS of its own for one block:
// its K half is copied there while the softmax and the values of the block before
// are worked on, its V half while the scores are.  S^T = K Q^T: a lane holds one
// row's scores of 8 consecutive keys of each 32, which is the operand of O^T +=
// V^T P^T as it lies; V's pairs of keys are made from its words of one key by
// exchanging halves of bytes.  ROOMY, for launches of at most two waves a SIMD, has
// registers for more loads and products at once (8B heads, one row of 613 tokens 8.5
// us on the GPU with 123 registers, 8.25 with 176; four waves a SIMD need 128).  A
// workgroup has the result's dims of one of DP parts.
// What bounds it: many rows, the memory (64 rows of 2,300, 170 MB, 48 us; 70B 64 of
// 8,000, 592 MB, 141 us, 4.2 TB/s of 4.7 that a copy reaches) with the rows' different
// ends, the join of their parts (5 and 7 us of these) and vector instructions
// behind it (45% and 54% of a SIMD's cycles); a row alone, its chain of loads (slot, ids,
// codes: 2.1 us) and one or two blocks of a wave (2 us each, half of it the values).
template <typename T, int HD, int NW, bool ROOMY, int DP>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(ROOMY ? 2 : sizeof(T) == 4 ? 3 : 4))) void
kv4_rows_kernel(const T *__restrict__ q, T *__restrict__ out, Kv4Args a) {
  typedef Kv4<HD> F;
  constexpr bool WIDE = sizeof(T) == 4;
  typedef std::conditional_t<WIDE, bf16_t, T> QT;      // operands of the scores
  typedef std::conditional_t<WIDE, bf16_t, f16_t> PT;  // of the values: fp16 has the finer weights
  typedef typename Mfma<QT>::v8 qv8;
  typedef typename Mfma<PT>::v8 pv8;
  constexpr int J = F::J, NP = WIDE ? 3 : 1;
  constexpr int JP = J / DP, HP = HD / DP;  // groups and dims of the result that this workgroup has
  float c2 = KV4_C2<HD>;
  constexpr int PART = 36 * HD, FULL = 32 * HD / 1024, TAIL = 4 * HD / 16;  // a half's bytes, copies, lanes of the last
  constexpr int ND = FULL + 1;
  __shared__ __attribute__((aligned(1024))) char lds[NW * F::BYTES];
  __shared__ float wm[NW * 16], wl[NW * 16];
  const int Hkv = a.b.kv.n_kv_heads, Hq = a.b.n_heads;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r16 = lane & 15, quad = lane >> 4;
  const int dp = blockIdx.x % DP, bid = blockIdx.x / DP;
  const int i0 = div_by(bid, a.by_hkv), g = bid - i0 * Hkv;
  const int part = div_by(i0, a.by_units);  // all rows' first splits, then their second ones
  int j_, r0;
  TileSeq ts;
  if (!own_tile<16>(a, i0 - part * a.units, j_, r0, ts)) return;
  r0 = __builtin_amdgcn_readfirstlane(r0);
  const int start = __builtin_amdgcn_readfirstlane(ts.start), n = __builtin_amdgcn_readfirstlane(ts.n);
  const int slot = __builtin_amdgcn_readfirstlane(ts.slot), p0 = __builtin_amdgcn_readfirstlane(ts.p0);
  const int top = row_ctx(a.b, slot, p0, min(div_by(r0 + 15, a.by_g), n - 1));  // the last row sees most
  int e0, e1;
  part_blocks<NW>(a, part, top, e0, e1);
  const bool direct = a.splits == 1;
  if (!direct && !a.b.seq_start && e0 >= e1) return;  // decode's join reads no such part
  auto row_live = [&](const PrefixRow &w) __attribute__((always_inline)) { return w.t < n; };
  const PrefixRow row = packed_row(a, start, r0, r16, g);
  const int ctx = row_live(row) ? row_ctx(a.b, slot, p0, row.t) : 0;
  // keys that every row of the tile sees; rows that see nothing get zeros at the end
  const int ctx_lo = (int)wave_min_u32(ctx ? (uint32_t)ctx : (uint32_t)INT_MAX);
  // Lane i: block id of entry win + i, -1 for none; left: those of them that are
  // there and this wave's still to take, every NW-th.
  int win = e0 - 64, id = -1;
  uint64_t left = 0;
  auto more = [&]() __attribute__((always_inline)) {
    while (!left && win + 64 < e1) {
      win += 64;
      id = -1;
      if (win + lane < e1 && win + lane < a.b.kv.max_blocks) {
        id = a.b.kv.block_table[(int64_t)slot * a.b.kv.max_blocks + win + lane];
        if (id >= a.b.kv.n_blocks) id = -1;
      }
      left = __ballot(id >= 0) & (~0ull / ((1ull << NW) - 1) << wave);
    }
    return left != 0;
  };

  char *ks = lds + wave * F::BYTES, *vs = ks + PART;
  const uint32_t kl = lds_addr(ks), vl = kl + PART;
  // Copies of 1 KB; 16-byte pieces of K rows are XOR-swizzled by the row against
  // bank conflicts.  Pieces past the last key repeat the last one before it.
  constexpr int KP = HD / 32;  // 16-byte pieces of a K row
  auto swz = [](int key) __attribute__((always_inline)) { return (key >> 3) & (KP - 1); };
  auto copy = [&](int i, bool is_k) __attribute__((always_inline)) {  // of entry win + i
    const int keys = min(KV_BLOCK, top - (win + i) * KV_BLOCK);
    const char *src = (const char *)a.b.kv.k +
                      ((int64_t)__builtin_amdgcn_readlane(id, i) * Hkv + g) * F::BYTES + (is_k ? 0 : PART);
    const uint32_t dst = is_k ? kl : vl;
    const uint32_t last = (is_k ? keys * (HD / 2) : (keys + 3) / 4 * 2 * HD) - 16;
    const uint32_t tail = __builtin_amdgcn_readfirstlane(dst + 32 * HD);  // kept scalar where lanes part
    if (lane < TAIL) dma16s(src, 32 * HD + lane * 16, tail);  // the scales
#pragma unroll
    for (int c = 0; c < FULL; ++c) {
      uint32_t off = c * 1024 + lane * 16;
      if (is_k) off ^= swz(off / (HD / 2)) * 16;
      dma16s(src, min(off, last), dst + c * 1024);
    }
  };

  // q: this lane's row, dims 32 j + 8 quad ..; looked at once the first copies are out
  typedef uint32_t words_t __attribute__((ext_vector_type(2 * sizeof(T))));
  words_t qx[J];
  {
    const T *qr = q + ((int64_t)(row_live(row) ? row.token : start) * Hq + row.head) * HD + quad * 8;
#pragma unroll
    for (int j = 0; j < J; ++j) qx[j] = *(const words_t *)(qr + 32 * j);
  }
  // o[2 j + x][i]: dim 32 j + 8 quad + 2 i + x of row r16, times 2^-ex
  floatx4_t o[2 * JP];
#pragma unroll
  for (int x = 0; x < 2 * JP; ++x) o[x] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  float mx = -INFINITY, sum = 0.f;  // of row r16; sum: this lane's keys alone
  int ex = -24 - KV4_UP;  // 16-bit types: V's largest scale so far is below 2^(ex + KV4_UP), at first the least of all
  // this lane's places in K's and V's halves, the rest of an address being constant
  int kat = (8 * (r16 >> 2) + (r16 & 3)) * (HD / 2) + (J == 4 ? quad : quad >> 1) * 16;
  kat = (kat ^ ((r16 >> 2) & (KP - 1)) * 16) + (J == 4 ? 0 : (quad & 1) * 8);
  int skat = F::k_scale(8 * quad, 0), vat = F::v_word(8 * quad, J == 4 ? r16 : r16 >> 1);
  int svat = F::v_scale(8 * quad, 0);
  asm volatile("" : "+v"(kat), "+v"(skat), "+v"(vat), "+v"(svat));
  int i = 0;
  bool go = more();
  if (go) {
    i = __builtin_ctzll(left);
    copy(i, true);
    copy(i, false);
  }
  qv8 qa[NP][J];  // Q^T as the B operand: this lane's row
  int up = 0;     // scores are taken by 2^-up of their row
  bool large = false;  // wave-uniform: values from 2^97 on, infinities or NaN among q
  if constexpr (!std::is_same_v<T, f16_t>) {
    // Products with codes are summed before the group's scale makes them small: a row of q
    // from 2^97 on is taken by a power of two to below it, and a sum over hd dims of codes up
    // to 6 and scales up to 10,752 then stays below 2^121.  (8B heads in bf16, one row of
    // 613 tokens 7.0 us, without the look at q 6.9.)
    typedef std::conditional_t<WIDE, uint32_t, uint16_t> bits_t;
    typedef bits_t lanes_t __attribute__((ext_vector_type(4 / sizeof(T))));
    constexpr uint32_t EXPS = WIDE ? 0x7F800000u : 0x7F807F80u;
    lanes_t most = 0;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int e = 0; e < 2 * (int)sizeof(T); ++e)
        most = __builtin_elementwise_max(most, __builtin_bit_cast(lanes_t, qx[j][e] & EXPS));
    uint32_t big = most[0];  // the largest exponent
    if constexpr (!WIDE) big = (uint32_t)max(most[0], most[1]) << 16;
    large = __any(big >= (127u + 97) << 23);
    if (__builtin_expect(large, 0)) {
      // that of the largest number stands for infinities and NaN
      up = max((int)(__float_as_uint(quads_max(__uint_as_float(min(big, 254u << 23)))) >> 23) - 127 - 96, 0);
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < 2 * (int)sizeof(T); ++e) {
          const float hi = __builtin_amdgcn_ldexpf(__uint_as_float(WIDE ? qx[j][e] : qx[j][e] & 0xFFFF0000u), -up);
          if constexpr (WIDE) {
            qx[j][e] = __float_as_uint(hi);
          } else {
            const float lo = __builtin_amdgcn_ldexpf(__uint_as_float(qx[j][e] << 16), -up);
            qx[j][e] = (uint32_t)round_to<bf16_t>(hi) << 16 | round_to<bf16_t>(lo);
          }
        }
      c2 = __builtin_amdgcn_ldexpf(c2, up);
    }
  }
#pragma unroll
  for (int j = 0; j < J; ++j) {
    if constexpr (!WIDE) {
      qa[0][j] = __builtin_bit_cast(qv8, qx[j]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = __uint_as_float(qx[j][e]);
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          const __bf16 part_ = (__bf16)v;
          qa[p][j][e] = part_;
          v -= (float)part_;
        }
      }
    }
  }
  if constexpr (WIDE)
    if (__builtin_expect(large, 0)) {  // an infinity is its first part alone: what it leaves is NaN
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if ((qx[j][e] & 0x7FFFFFFFu) == 0x7F800000u) qa[1][j][e] = qa[2][j][e] = (__bf16)0.f;
    }
  while (go) {
    const int base = (win + i) * KV_BLOCK;
    left &= left - 1;
    go = more();
    i = go ? __builtin_ctzll(left) : 0;  // the next one
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(ND) : "memory");  // K is there, V may not be
    float s[4][4];  // key 16 t + 8 (lane's quad) .. as p below: 32 (t / 2) + 8 quad + 4 (t % 2) + e
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      constexpr int ROW = HD / 2;
      const int tk = 32 * (t / 2) + 4 * (t & 1);  // the swizzle of a key is that of 8 (r16 / 4)
      uint32_t piece[J];
      if constexpr (J == 4) {
        const u32x4_tt v = *(const u32x4_tt *)(ks + kat + tk * ROW);
#pragma unroll
        for (int j = 0; j < J; ++j) piece[j] = v[j];
      } else {
        const u32x2_tt v = *(const u32x2_tt *)(ks + kat + tk * ROW);
#pragma unroll
        for (int j = 0; j < J; ++j) piece[j] = v[j];
      }
      _Float16 sk[4 * J];  // [key][group]
#pragma unroll
      for (int x = 0; x < J / 2; ++x)
        *(u32x4_tt *)(sk + 8 * x) =
            *(const u32x4_tt *)(ks + skat + tk * 2 * J + 16 * x);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[t][e] = 0.f;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const qv8 c = codes8<QT>(piece[j]);
        floatx4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < NP; ++p) acc = Mfma<QT>::m16(c, qa[p][j], acc);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[t][e] = fmaf((float)sk[e * J + j], acc[e], s[t][e]);
      }
      if constexpr (!ROOMY)
        asm volatile("" : "+v"(s[t][0]), "+v"(s[t][1]), "+v"(s[t][2]), "+v"(s[t][3]));  // products end here
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K has been read
    if (go) copy(i, true);
    const int end = min(KV_BLOCK, ctx - base) - 8 * quad;  // the row's keys, from the lane's first one on: those below
    const bool partly = base + KV_BLOCK > ctx_lo;
    if (partly) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (32 * (t / 2) + 4 * (t & 1) + e >= end) s[t][e] = -INFINITY;
    }
    float m = s[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, s[t][e]);
    m = fmaxf(mx, quads_max(m));
    int e = ex;
    if constexpr (!WIDE) {
      // Weights times scales are taken by 2^-ex: below 2^15 for values of any size,
      // and normal numbers of fp16 down to 2^-28 of the largest scale so far (of keys
      // that a row of the tile sees), so that large values elsewhere cost no bits.
      if (go)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(ND + FULL) : "memory");  // V's scales are there
      else
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(FULL) : "memory");
      // lane l: J scales from l J on, of keys l J mod 64 ..
      typedef uint32_t piece_t __attribute__((ext_vector_type(J / 2)));
      piece_t raw = *(const piece_t *)(vs + 32 * HD + lane * J * 2);
      const int keys = top - base - lane * J % 64;
      float big = 0.f;
#pragma unroll
      for (int x = 0; x < J / 2; ++x) {
        if (base + KV_BLOCK > top) raw[x] &= (2 * x < keys ? 0xFFFFu : 0u) | (2 * x + 1 < keys ? 0xFFFF0000u : 0u);
        big = fmaxf(big, (float)__builtin_bit_cast(_Float16, (uint16_t)raw[x]));
        big = fmaxf(big, (float)__builtin_bit_cast(_Float16, (uint16_t)(raw[x] >> 16)));
      }
      big = wave_max(big);
      e = __builtin_amdgcn_readfirstlane(big > 0.f ? __builtin_amdgcn_frexp_expf(fminf(big, 65504.f)) - KV4_UP : ex);
      e = max(e, ex);
    }
    if (e > ex || __any(m > mx && ctx > 0)) {
      const float corr = __builtin_amdgcn_exp2f((m == mx ? 0.f : (mx - m) * c2) + (float)(ex - e));
      mx = m;
      ex = e;
      sum *= corr;
#pragma unroll
      for (int x = 0; x < 2 * JP; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) o[x][y] *= corr;
    }
    const float m0 = mx == -INFINITY ? 0.f : mx;  // a row that has seen no key yet
    const float by = WIDE ? 0.f : (float)-ex;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        s[t][y] = __builtin_amdgcn_exp2f(fmaf(s[t][y] - m0, c2, by));
        sum += s[t][y];
      }
    if (go)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(ND) : "memory");  // V is there
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // words of keys 32 h + 8 quad .. + 7, then pairs of keys: lo the even dims', hi the odd ones'
      uint32_t x[8], lo[4], hi[4];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const u32x4_tt v = *(const u32x4_tt *)(ks + vat + (8 * h + y) * 2 * HD);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * y + e] = J == 4 ? v[e] : v[e] >> ((r16 & 1) * 16);
      }
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        lo[y] = (x[2 * y] & 0x0F0F0F0Fu) | ((x[2 * y + 1] << 4) & 0xF0F0F0F0u);
        hi[y] = ((x[2 * y] >> 4) & 0x0F0F0F0Fu) | (x[2 * y + 1] & 0xF0F0F0F0u);
      }
      auto group = [&](auto j_c) __attribute__((always_inline)) {
        constexpr int j = decltype(j_c)::value, l = j % JP;
        u32x4_tt raw = *(const u32x4_tt *)(ks + svat + 64 * h + 128 * j);
        if (partly) {
          // scales at places that the row does not see may be anything, and 0 * NaN is not 0
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int key = 32 * h + 2 * y;
            raw[y] &= (key < end ? 0xFFFFu : 0u) | (key + 1 < end ? 0xFFFF0000u : 0u);
          }
        }
        pv8 p[NP];
        if constexpr (!WIDE) {
          u32x4_tt pw;
#pragma unroll
          for (int y = 0; y < 4; ++y)
            pw[y] = mul_pair(s[2 * h + y / 2][y % 2 * 2], s[2 * h + y / 2][y % 2 * 2 + 1], raw[y]);
          p[0] = __builtin_bit_cast(pv8, pw);
        } else {
          _Float16 sv[8];
          *(u32x4_tt *)sv = raw;
#pragma unroll
          for (int y = 0; y < 8; ++y) {
            float v = s[2 * h + y / 4][y % 4] * (float)sv[y];
#pragma unroll
            for (int k = 0; k < NP; ++k) {
              const __bf16 part_ = (__bf16)v;
              p[k][y] = part_;
              v -= (float)part_;
            }
          }
        }
        const u32x4_tt c0 = {kv4_pair16<PT, j>(lo[0]), kv4_pair16<PT, j>(lo[1]), kv4_pair16<PT, j>(lo[2]),
                             kv4_pair16<PT, j>(lo[3])};
        const u32x4_tt c1 = {kv4_pair16<PT, j>(hi[0]), kv4_pair16<PT, j>(hi[1]), kv4_pair16<PT, j>(hi[2]),
                             kv4_pair16<PT, j>(hi[3])};
#pragma unroll
        for (int k = 0; k < NP; ++k) {
          o[2 * l] = Mfma<PT>::m16(__builtin_bit_cast(pv8, c0), p[k], o[2 * l]);
          o[2 * l + 1] = Mfma<PT>::m16(__builtin_bit_cast(pv8, c1), p[k], o[2 * l + 1]);
        }
        if constexpr (!ROOMY)
          __builtin_amdgcn_sched_barrier(0);  // a group's loads and operands at a time: 128 registers
      };
      if (dp == 0) group(std::integral_constant<int, 0>());
      if (dp == 1 / JP) group(std::integral_constant<int, 1>());
      if constexpr (J == 4) {
        if (dp == 2 / JP) group(std::integral_constant<int, 2>());
        if (dp == 3 / JP) group(std::integral_constant<int, 3>());
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V has been read
    if (go) copy(i, false);
  }
  const float back = WIDE ? 1.f : __builtin_amdgcn_ldexpf(1.f, ex);
  sum = quads_sum(sum) * back;
  const int nrows = a.b.seq_start ? 16 : min(16, a.G - r0);
  // o goes where K and V were, row r16's dims side by side
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  if (quad == 0) wm[wave * 16 + r16] = mx, wl[wave * 16 + r16] = sum;
  if (r16 < nrows) {
#pragma unroll
    for (int j = 0; j < JP; ++j)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const float4 v = make_float4(o[2 * j][2 * y] * back, o[2 * j + 1][2 * y] * back, o[2 * j][2 * y + 1] * back,
                                     o[2 * j + 1][2 * y + 1] * back);
        *(float4 *)(ks + (r16 * HP + 32 * j + 8 * quad + 4 * y) * 4) = v;
      }
  }
  __syncthreads();
  int l16 = r16;
  asm volatile("" : "+v"(l16));  // found again here, not held in registers over the walk
  const PrefixRow w = packed_row(a, start, r0, l16, g);
  const bool live = row_live(w);
  constexpr int VN = (HP + 63) / 64;
  // a wave a row: its lanes over the dims
  for (int r = wave; r < nrows; r += NW) {
    if (!__builtin_amdgcn_readlane((int)live, r)) continue;
    const int token = __builtin_amdgcn_readlane(w.token, r), h = __builtin_amdgcn_readlane(w.head, r);
    float M = -INFINITY, L = 0.f, v[VN];
    const float row_c2 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(c2), r));
#pragma unroll
    for (int k = 0; k < NW; ++k) M = fmaxf(M, wm[k * 16 + r]);
#pragma unroll
    for (int d = 0; d < VN; ++d) v[d] = 0.f;
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      const float m = wm[k * 16 + r], f = m == M ? 1.f : __builtin_amdgcn_exp2f((m - M) * row_c2);
      L += f * wl[k * 16 + r];
#pragma unroll
      for (int d = 0; d < VN; ++d) v[d] += f * ((const float *)(lds + k * F::BYTES))[r * HP + d * 64 + lane];
    }
    const bool none = __builtin_amdgcn_readlane(ctx, r) == 0;
    const int64_t row = (int64_t)token * Hq + h, rec = row * a.splits + part;
#pragma unroll
    for (int d = 0; d < VN; ++d) {
      if (none) v[d] = 0.f;
      if (direct && (HP >= 64 || lane < HP))
        out[row * HD + dp * HP + d * 64 + lane] = round_to<T>(L == 0.f ? 0.f : v[d] / L);
      else if (!direct && e0 < e1 && (HP >= 64 || lane < HP))
        a.po[rec * HD + dp * HP + d * 64 + lane] = v[d];
    }
    if (!direct && dp == 0 && lane == 0)
      *(float2 *)(a.pml + rec * 2) =
          none ? make_float2(-INFINITY, 0.f)
               : make_float2(__builtin_amdgcn_ldexpf(M, __builtin_amdgcn_readlane(up, r)), L);
  }
}

// Many rows of a 16-bit type, on 32x32x16 MFMAs in fp16: a workgroup owns 128 packed
// rows of a sequence, 32 to a wave, and walks the sequence's blocks.  Codes are
// turned into values once for all of its rows: a block's are loaded into
// registers while the one before is worked on, multiplied by their scales (exact:
// a value has 8 significant bits) and put into LDS, K by rows, V by dims, with the
// 16-byte pieces of a row XOR-swizzled against bank conflicts.  Two stages.
//   S^T = K Q^T: a lane holds one row's scores; the K row of MFMA row i is i with
//   bits 2 and 3 swapped, so that the eight weights a lane holds of each 16 keys
//   are consecutive keys, the operand of O^T += V^T P^T.
// bf16: a row of q is taken by its largest exponent, which the scores' factor
// brings back; its fp16 is then exact but for values below 2^-14 of the largest,
// whose rounding (2^-25 of the largest) is that of the fp32 sums (of rows whose large
// elements meet large keys: the rows' kernel keeps such values whole).
// Values at places that no row of the tile sees are 0.  Where V's scale is not of
// the format (NaN: the group held an infinity or NaN), the values are 0 as well, and the
// rows that see the place get NaN in the group's dims afterwards.
// Bound by the card's power: three prompts of 2,100 after 2,000 of 70B heads, 637
// GFLOP, 1.50 M cycles, 707 us at 2.1 GHz, 790 at 1.9; matrix cores are busy 41% of the
// cycles, vector units 56% (nine instructions a MFMA).  (Values turned before the
// matrix instructions instead of between them 817 us for 735; eight waves on 256 rows
// 820, with a half of them a phase behind 811; 64 rows a wave 1,068.)
// A reference within 2^8 of the maximum (735 us; following it exactly 773).
constexpr float KV4_LAZY = 8.f;
constexpr float KV4_TILE_UP = 7.f;  // weights are taken by 2^7: fp16's normal numbers are then those from 2^-21 to 2^8
constexpr float KV4_LARGE = 64.f;  // base-2 score up to which the rounded mc is within 2^-19: weights within 1.3e-6
template <typename T, int HD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void kv4_tile_kernel(
    const T *__restrict__ q, T *__restrict__ out, Kv4Args a) {
  typedef Kv4<HD> F;
  typedef f16x8_t v8;
  constexpr int RT = 128;
  constexpr int J = F::J, KS = HD / 16, NT = HD / 32;
  constexpr int CK = HD / 8;           // 16-byte pieces of a K row
  constexpr int PB = 64 * HD * 2, STAGE = 2 * PB;
  typedef uint32_t words_t __attribute__((ext_vector_type(J)));
  __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];
  __shared__ int odd_at[2];  // 1 + the block of a stage whose V scales are not all of the format
  const int Hkv = a.b.kv.n_kv_heads, Hq = a.b.n_heads;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int l32 = lane & 31, hh = lane >> 5;
  const int i0 = div_by(blockIdx.x, a.by_hkv), g = blockIdx.x - i0 * Hkv;
  const int part = div_by(i0, a.by_units);
  int j_, r0;
  TileSeq ts;
  if (!own_tile<RT>(a, i0 - part * a.units, j_, r0, ts)) return;
  r0 = __builtin_amdgcn_readfirstlane(r0);
  const int start = __builtin_amdgcn_readfirstlane(ts.start), n = __builtin_amdgcn_readfirstlane(ts.n);
  const int slot = __builtin_amdgcn_readfirstlane(ts.slot), p0 = __builtin_amdgcn_readfirstlane(ts.p0);
  const int top = row_ctx(a.b, slot, p0, min(div_by(r0 + RT - 1, a.by_g), n - 1));  // the last row sees most
  int e0, e1;
  part_blocks<1>(a, part, top, e0, e1);
  const PrefixRow w = packed_row(a, start, r0, wave * 32 + l32, g);
  const bool live = w.t < n;
  const int wctx = live ? row_ctx(a.b, slot, p0, w.t) : 0;
  // rows that do not exist or see nothing (zeros at the end, whatever is summed for them) ask for no mask
  const int ctx = wctx ? wctx : INT_MAX;
  const int ctx_lo = (int)wave_min_u32((uint32_t)ctx);
  const int ctx_top = (int)~wave_min_u32(~(uint32_t)wctx);

  // Block ids: lane i holds that of entry win + i, -1 for none.
  int win = e0, ids = -1;
  auto window = [&]() __attribute__((always_inline)) {
    ids = -1;
    if (win + lane < e1 && win + lane < a.b.kv.max_blocks) {
      ids = a.b.kv.block_table[(int64_t)slot * a.b.kv.max_blocks + win + lane];
      if (ids >= a.b.kv.n_blocks) ids = -1;
    }
  };
  // This thread's share of a block: K row kr, octets ki of its groups; V word vw of positions 4 vq ..
  const int kr = tid >> 2, ki = tid & 3, vq = tid & 15, vw = tid >> 4;
  const bool has_v = HD == 128 || vw < HD / 8;
  const uint32_t k_off = F::k_row(kr) + 4 * J * ki, ks_off = F::k_scale(kr, 0), v_off = F::v_word(4 * vq, vw),
                 vs_off = 8 * vq;
  words_t kc;
  _Float16 ksc[J];
  u32x4_tt vc;
  u32x2_tt vsc[J];
  auto head_of = [&](int id) __attribute__((always_inline)) {
    return (const char *)a.b.kv.k + ((int64_t)id * Hkv + g) * F::BYTES;
  };
  auto find = [&](int e) __attribute__((always_inline)) {  // block id of entry e, -1 past the last
    if (e >= win + 64) {
      win = e;
      window();
    }
    return e < e1 ? __builtin_amdgcn_readlane(ids, e - win) : -1;
  };
  // Loads of a block that is not there are left out: what the registers hold
  // then goes into a stage that is not read.
  auto load_k = [&](int id) __attribute__((always_inline)) {
    if (id < 0) return;
    const char *src = head_of(id);
    kc = *(const words_t *)(src + k_off);
    if constexpr (J == 4)
      *(u32x2_tt *)ksc = *(const u32x2_tt *)(src + ks_off);
    else
      *(uint32_t *)ksc = *(const uint32_t *)(src + ks_off);
  };
  auto load_v = [&](int id) __attribute__((always_inline)) {
    if (id < 0 || !has_v) return;
    const char *src = head_of(id);
    vc = *(const u32x4_tt *)(src + v_off);
#pragma unroll
    for (int j = 0; j < J; ++j) vsc[j] = *(const u32x2_tt *)(src + F::v_scale(0, j) + vs_off);
  };
  auto swz = [](int row) __attribute__((always_inline)) { return CK == 16 ? row & 15 : (row >> 1) & 7; };
  // V's scales of the loaded block as its values take them: 0 at places that no row
  // sees and where they are not of the format.
  auto check = [&](int e, int stage) __attribute__((always_inline)) {
    if (!has_v) return;
    if ((e + 1) * KV_BLOCK > top) {
      const int keys = top - e * KV_BLOCK - 4 * vq;  // that some row sees, of this thread's four
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int y = 0; y < 2; ++y)
          vsc[j][y] &= (2 * y < keys ? 0xFFFFu : 0u) | (2 * y + 1 < keys ? 0xFFFF0000u : 0u);
    }
    typedef uint16_t pair_t __attribute__((ext_vector_type(2)));
    pair_t big = {0, 0};
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int y = 0; y < 2; ++y)
        big = __builtin_elementwise_max(big, __builtin_bit_cast(pair_t, (uint32_t)vsc[j][y]));
    if (max(big[0], big[1]) > 0x7140) {  // past 10752, the largest scale, are the infinities and NaN
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t s = vsc[j][y];
          vsc[j][y] = ((s & 0xFFFFu) > 0x7140u ? 0 : s & 0xFFFFu) | (s >= 0x71410000u ? 0 : s & 0xFFFF0000u);
        }
      odd_at[stage] = e + 1;
    }
  };
  // The loaded block's values into a stage (where there is none, what the
  // registers hold: that stage is not read).
  auto fill_k = [&](int stage, int j) __attribute__((always_inline)) {  // group j
    const half2_t s = {ksc[j], ksc[j]};
    const half2_t y[4] = {__builtin_bit_cast(half2_t, kv4_pair16<f16_t, 0>(kc[j])) * s,
                          __builtin_bit_cast(half2_t, kv4_pair16<f16_t, 1>(kc[j])) * s,
                          __builtin_bit_cast(half2_t, kv4_pair16<f16_t, 2>(kc[j])) * s,
                          __builtin_bit_cast(half2_t, kv4_pair16<f16_t, 3>(kc[j])) * s};
    const u32x4_tt v = {__builtin_bit_cast(uint32_t, y[0]), __builtin_bit_cast(uint32_t, y[1]),
                        __builtin_bit_cast(uint32_t, y[2]), __builtin_bit_cast(uint32_t, y[3])};
    *(u32x4_tt *)(lds + stage * STAGE + kr * HD * 2 + (((4 * j + ki) ^ swz(kr)) * 16)) = v;
  };
  auto pair_v = [&]() __attribute__((always_inline)) {  // vc: bytes of even dims, of odd ones, each of two positions
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const uint32_t x0 = vc[2 * y], x1 = vc[2 * y + 1];
      vc[2 * y] = (x0 & 0x0F0F0F0Fu) | ((x1 << 4) & 0xF0F0F0F0u);
      vc[2 * y + 1] = ((x0 >> 4) & 0x0F0F0F0Fu) | (x1 & 0xF0F0F0F0u);
    }
  };
  auto fill_v = [&](int stage, int byte_) __attribute__((always_inline)) {  // byte of the word
    if (!has_v) return;
    char *vs = lds + stage * STAGE + PB;
    auto byte = [&](auto b_c) __attribute__((always_inline)) {
      constexpr int b = decltype(b_c)::value, j = b % J;
      const int d = 32 * j + 2 * ((4 * vw + b) / J);
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const half2_t y0 = __builtin_bit_cast(half2_t, kv4_pair16<f16_t, b>(vc[z])) *
                           __builtin_bit_cast(half2_t, (uint32_t)vsc[j][0]);
        const half2_t y1 = __builtin_bit_cast(half2_t, kv4_pair16<f16_t, b>(vc[2 + z])) *
                           __builtin_bit_cast(half2_t, (uint32_t)vsc[j][1]);
        const u32x2_tt v = {__builtin_bit_cast(uint32_t, y0), __builtin_bit_cast(uint32_t, y1)};
        *(u32x2_tt *)(vs + (d + z) * KV_BLOCK * 2 + (((vq >> 1) ^ ((d >> 1) & 7)) * 16) + (vq & 1) * 8) = v;
      }
    };
    if (byte_ == 0) byte(std::integral_constant<int, 0>());
    if (byte_ == 1) byte(std::integral_constant<int, 1>());
    if (byte_ == 2) byte(std::integral_constant<int, 2>());
    if (byte_ == 3) byte(std::integral_constant<int, 3>());
  };
  auto fill = [&](int stage) __attribute__((always_inline)) {
    pair_v();
#pragma unroll
    for (int j = 0; j < J; ++j) fill_k(stage, j);
#pragma unroll
    for (int b = 0; b < 4; ++b) fill_v(stage, b);
  };

  // ids of the blocks in the stage in use, in the registers, -1 for none
  int staged = -1, loaded = -1;
  if (e0 < e1) {
    window();
    staged = find(e0);
    load_k(staged);
    load_v(staged);
  }
  v8 qb[KS];  // Q^T as the operand: this lane's row, dims 16 k + 8 hh ..
  float c2 = KV4_C2<HD>, unit = 1.f;  // base-2 factor of a score, the row's power of two
  {
    const T *qr = q + ((int64_t)(live ? w.token : start) * Hq + w.head) * HD + hh * 8;
    if constexpr (std::is_same_v<T, f16_t>) {
#pragma unroll
      for (int k = 0; k < KS; ++k) qb[k] = load8<T>(qr + k * 16);
    } else {
      bf16x8_t x[KS];
      float big = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        x[k] = load8<T>(qr + k * 16);
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const float v = fabsf((float)x[k][y]);
          big = v < INFINITY ? fmaxf(big, v) : big;
        }
      }
      big = half_swap_max(big);
      const int ex = big > 0.f ? min(__builtin_amdgcn_frexp_expf(big), 127) : 0;  // 2^128 is no number
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int y = 0; y < 8; ++y) qb[k][y] = (_Float16)__builtin_amdgcn_ldexpf((float)x[k][y], -ex);
      unit = __builtin_amdgcn_ldexpf(1.f, ex);
      c2 *= unit;
    }
  }
  floatx16_t o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
  // running maximum (scores in the row's unit), its base-2 value, this half's share of the sum
  float mx = -INFINITY, mc = 0.f, lsum = 0.f;
  bool large = false;  // wave-uniform: a row's |mc| is past KV4_LARGE
  const int krow = (l32 & 0x13) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);
  const int kfb = krow * HD * 2, kfx = (hh ^ swz(krow)) << 4;
  const int vfb = l32 * KV_BLOCK * 2, vfx = (hh ^ ((l32 >> 1) & 7)) << 4;
  if (tid < 2) odd_at[tid] = 0;
  __syncthreads();  // odd_at is 0
  if (e0 < e1) {
    check(e0, 0);
    fill(0);
    loaded = find(e0 + 1);
    load_k(loaded);
    load_v(loaded);
  }
  __syncthreads();
  for (int e = e0; e < e1; ++e) {
    const int base = e * KV_BLOCK, stage = (e - e0) & 1;
    char *ks = lds + stage * STAGE, *vs = ks + PB;
    const int next = find(e + 2);
    const int odd = odd_at[stage];  // asked for long before its use
    if (staged >= 0 && base < ctx_top) {  // else no block, or wholly past this wave's rows
      floatx16_t s[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const v8 f = *(const v8 *)(ks + kfb + t * 32 * HD * 2 + (kfx ^ (k << 5)));
          s[t] = Mfma<f16_t>::m32(f, qb[k], s[t]);
          // the next block's values between the matrix instructions
          if (k % 4 == 3) fill_k(stage ^ 1, t * (KS / 4) + k / 4);
        }
      }
      // K's fragments four ahead of their MFMAs, which else wait for LDS one by one
      // (three long prompts 720 us)
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int i = 0; i < 2 * KS - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, 4, 0);
      load_k(next);  // a part of a walk's step ahead of their use, like V's below
      if (e + 1 < e1) check(e + 1, stage ^ 1);
      pair_v();
      // s[t][r]: key 32 t + 16 (r / 8) + 8 hh + r % 8 of the block
      const int end = min(KV_BLOCK, ctx - base);  // the row's keys: those below
      if (base + KV_BLOCK > ctx_lo || base + KV_BLOCK > top) {
        const int lim = min(end, top - base) - 8 * hh;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (t * 32 + (r >> 3) * 16 + (r & 7) >= lim) s[t][r] = -INFINITY;
      }
      float m = s[0][0];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) m = fmaxf(m, s[t][r]);
      m = half_swap_max(m);
      // The reference follows the maximum once that is past it by 2^8: weights up to
      // there are fp16 numbers like any others, and most blocks leave o alone.
      if (__any((m - mx) * c2 > KV4_LAZY)) {
        const float nm = fmaxf(mx, m);
        const float corr = nm == mx ? 1.f : __builtin_amdgcn_exp2f((mx - nm) * c2);
        mx = nm;
        lsum *= corr;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[t][r] *= corr;
        mc = nm == -INFINITY ? 0.f : fmaf(nm, c2, -KV4_TILE_UP);  // a row that has seen no key yet
        large = __any(fabsf(mc) > KV4_LARGE);
      }
      // s c2 - mc in one FMA is off 0 at the maximum by what mc's rounding left
      // out: large scores have the maximum taken off before the product instead
      float mo = mc;
      if (large) {
        const float m0 = mx == -INFINITY ? 0.f : mx;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[t][r] -= m0;
        mo = -KV4_TILE_UP;
      }
      v8 pb[4];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float p[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            p[r] = __builtin_amdgcn_exp2f(fmaf(s[t][u * 8 + r], c2, -mo));
            lsum += p[r];
          }
          // the one rounding below 32 bits before the result's: MFMA operands have 16 (the sum stays unrounded)
          pb[t * 2 + u] = pack8<f16_t>(p);
        }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const v8 f = *(const v8 *)(vs + vfb + t * 32 * KV_BLOCK * 2 + (vfx ^ (k << 5)));
          o[t] = Mfma<f16_t>::m32(f, pb[k], o[t]);
        }
        fill_v(stage ^ 1, k);
      }
      load_v(next);
      if (odd == e + 1) {
        const char *sc = head_of(staged);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint32_t x = *(const uint16_t *)(sc + F::v_scale(lane, t));
          const uint64_t bad = __ballot(x > 0x7140u);
          const uint64_t mine = end >= 64 ? ~0ull : end > 0 ? (1ull << end) - 1 : 0;
          if (bad & mine) {
#pragma unroll
            for (int r = 0; r < 16; ++r) o[t][r] = __uint_as_float(0x7FC00000u);
          }
        }
      }
    } else {
      if (e + 1 < e1) check(e + 1, stage ^ 1);
      fill(stage ^ 1);
      load_k(next);
      load_v(next);
    }
    staged = loaded;
    loaded = next;
    __syncthreads();
  }
  if (!wctx) {
    mx = -INFINITY;
    lsum = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
  }
  // o[t][r]: dim 32 t + 8 (r / 4) + 4 hh + r % 4 of this lane's row
  const float sum = half_swap_sum(lsum);
  const int64_t row = (int64_t)w.token * Hq + w.head;
  if (a.splits == 1) {
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
    for (int t = 0; t < NT; ++t) store_o32(out + row * HD + t * 32, o[t], inv, hh, live);
    return;
  }
  // Through LDS, so that a row's dims leave as one run of bytes: 16-byte pieces
  // XOR-swizzled by the row, the wave's 32 rows in a place of its own.
  constexpr int LR = HD / 4, RI = 64 / LR;  // lanes of a row, rows of a store
  char *own = lds + wave * 32 * HD * 4;
  if (live && hh == 0) *(float2 *)(a.pml + (row * a.splits + part) * 2) = make_float2(mx * unit, sum);
  const uint32_t rows_live = e0 < e1 ? (uint32_t)__ballot(live) : 0;  // the join skips o of empty parts
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int piece = t * 8 + r / 2 + hh;
      *(float4 *)(own + l32 * HD * 4 + ((piece ^ (l32 % LR)) * 16)) =
          make_float4(o[t][r], o[t][r + 1], o[t][r + 2], o[t][r + 3]);
    }
#pragma unroll 4
  for (int i = 0; i < 32 / RI; ++i) {
    const int x = i * RI + lane / LR;
    const float4 v = *(const float4 *)(own + x * HD * 4 + (((lane % LR) ^ (x % LR)) * 16));
    const PrefixRow y = packed_row(a, start, r0, wave * 32 + x, g);
    if (rows_live >> x & 1)
      *(float4 *)(a.po + (((int64_t)y.token * Hq + y.head) * a.splits + part) * HD + lane % LR * 4) = v;
  }
}

// ------------------------------------------------------------------ plan

// 16-row items.  A workgroup's waves share its blocks, so a row (or 16 packed ones)
// and KV head, a "pair", is one item of all blocks where there are pairs enough
// or few blocks, for which a second launch costs more than it brings; eight
// waves share it while that fills the GPU once.  Else items of a few blocks, about
// 1,365 of them for the longest rows' lengths, at most 24 blocks each, so that long
// rows end with the others.
// (Graphs of calls; an item's blocks with four waves, "all" with eight.  8B heads:
// one row of 300 tokens 4 8.4 us, all 7.4; four of 613, longest 16 blocks, 4 8.8, all
// 10.6; one of 2,000 4 9.2, 8 10.5, 16 14.7; one of 8,000 4 10.1, 8 12.0; 16 of 1,000 4
// 16.3, 8 15.2, all 17.3; 20 of 300, 160 pairs, 12 13.2, all 10.8; 24 of 800, 192, 16
// 17.7, all 15.6; 32 of 2,300, 256, 17 34.3, 23 39.9; 16 of 2,300 8 22.1, 10 24.3; 64
// of 1,000, 512, 16 28.8, all 28.0; 64 of 2,300 16 54.2, 24 49.8, 32 52.4, 48 54.5; 70B
// 64 of 8,000 16 152.7, 24 141.4, 32 141.6, 48 146.4; 13B 64 of 1,200, 2,560 pairs, 8
// 95.8, 16 91.5, all with four waves 87.2, with eight 91.3.)
struct Kv4Split {
  int blocks, waves;
};
static Kv4Split kv4_rows_split(int64_t pairs, int blocks) {
  if (blocks <= 12 || (blocks <= 40 && pairs >= 7 * blocks) || pairs >= 2048) return {blocks, pairs <= 512 ? 8 : 4};
  const int even = (int)std::min<int64_t>((blocks * std::min<int64_t>(pairs, 1024) * 3 + 4095) / 4096, 24);
  return {std::min(blocks, std::max(even, pairs < 64 ? 4 : 8)), 4};
}

// Prompts' tiles of 128 rows: blocks of a split, for about `items` tiles and KV heads
// of `live` sequences.  In us: a block takes 1.45 alone on a CU, 2.25 with a second tile
// beside it, which a launch of up to 480 tiles keeps to; more come as others end and
// take 1.1 each.  A tile takes 3.7 more, the join 2.6 and 1.7e-4 a row, head and part.
// Contexts of several sequences are taken to be 0.8 of the longest.  Fitted to (new +
// cached tokens, graphs of calls, blocks of a split): 8B 16 x 40 + 1,500 all 78.0, 25 65.5,
// 17 51.6, 13 57.1; 4 x 100 + 3,000 all 92.6, 21 56.5, 13 45.5, 11 54.2; 8 x 200 + 1,000
// all 63.7, 15 73.8; 8 x 60 + 2,000 all 81.8, 14 46.2, 11 54.3; 32 x 30 + 800 all 53.0,
// 14 48.3, 9 49.1; 2 x 300 + 4,000 all 123, 28 78.9, 21 88.8; 1 x 2,000 all 57.5, 16 74.5;
// 70B 1 x 100 + 2,000 all 50.8, 17 36.7, 9 27.0, 7 26.5; 7B 1 x 547 + 2,000 all 63.1, 20
// 54.9, 14 45.2, 10 54.5; 6 x 80 + 1,500 all 53.5, 11 44.9, 9 49.2; 13B 4 x 100 + 1,000
// all 50.9, 16 48.1, 11 40.1, 8 46.9.
static int kv4_tile_split(double items, int live, int blocks, int64_t rows_heads) {
  const double all = items * blocks * (live == 1 ? 1 : 0.8) * 1.1 / 256;  // at 1.1 a block
  int best = blocks;
  double least = 0;
  for (int s = 1; s <= ceil_div(blocks, 4) && (s == 1 || items * s <= 1024); ++s) {
    const int n = ceil_div(blocks, s);
    if (ceil_div(blocks, n) != s) continue;
    const double tiles = items * s;
    const double walk = tiles <= 256 ? n * 1.45 : tiles <= 480 ? n * 2.25 : std::max(n * 2.25, all + n * 0.7);
    const double t = 3.7 * std::max(1.0, tiles / 512) + walk + (s == 1 ? 0 : 2.6 + rows_heads * s * 1.7e-4);
    if (s == 1 || t < least) {
      least = t;
      best = n;
    }
  }
  return best;
}

// Partials (row, head and part) that a plan may have, ascending in rows and contexts
// so that a workspace for a batch's limits serves its smaller steps.  Plans stay
// within it by themselves but for batches with far more rows than their sequences
// can have: 16-row items split only below 2,048 pairs, 32,768 rows and heads, into
// parts of 24 blocks, or smaller ones (of four at least) up to about 1,365 items;
// tiles up to 1,024 items of 128 rows.
static int64_t kv4_partials(bool decode, int64_t rows_heads, int blocks) {
  const int64_t quarter = rows_heads * ((blocks + 3) / 4);
  return std::max(std::min<int64_t>(rows_heads, 32768) * ((blocks + 23) / 24),
                  std::min<int64_t>(quarter, decode ? 32768 : 131072));
}
size_t kv4_attention_ws_bytes(bool decode, int rows, int n_heads, int head_dim, int max_ctx) {
  return (size_t)kv4_partials(decode, (int64_t)rows * n_heads, ceil_div(max_ctx, KV_BLOCK)) * (head_dim + 2) *
         sizeof(float);
}

// Parts of the result's dims, a workgroup each, by the blocks of all items: scores
// are computed again on other CUs, the values' share of a wave's time shrinks.  (us
// with one part, two, a group of 32 dims each: 8B heads, one row of 613 tokens, 80
// blocks, 8.3 7.5 7.0, eight, 640, 8.4 7.9 9.8, one of 2,000 in items of four, 256, 8.9 -
// 8.4, of 4,000, 504, 8.9 9.5; 7B one of 613, 320, 7.8 7.0 7.8, three, 1,056, 8.0 9.3; 70B
// one of 3,000 in items, 376, 9.9 9.3; 8B in fp32, whose values cost three times as much,
// one of 613 12.2 10.4 9.1, four in items, 512, 10.2 9.8.)
static int kv4_dim_parts(int64_t blocks, bool split16, int groups) {
  return blocks <= 288 ? groups : blocks <= (split16 ? 400 : 720) ? 2 : 1;
}

template <typename T, int HD>
static bool launch_kv4_hd(const T *q, T *out, const PrefixBatch &b, float *ws, hipStream_t s) {
  Kv4Args a{};
  a.b = b;
  const bool decode = !b.seq_start;
  const int Hkv = b.kv.n_kv_heads, blocks = ceil_div(b.max_ctx, KV_BLOCK), live = std::min(b.n_seq, b.rows);
  a.G = b.n_heads / Hkv;
  const auto units = [&](int rt) {  // row tiles at most, of rt rows
    if (decode) return b.rows * ceil_div(a.G, rt);
    return (int)std::min((int64_t)live * ceil_div((int64_t)std::min(b.max_new, b.rows) * a.G, rt),
                         (int64_t)b.rows * a.G / rt + live);
  };
  // Few rows over more than two blocks take 16-row items, as fp32 does (new + cached
  // tokens, 16-row items against tiles, at their best splits: 8B 30 + 2,000, 64 pairs,
  // 13.2 us and 15.5, 100 + 500, 200 pairs, 12.7 and 14.8, 30 alone 7.9 and 7.0; 70B
  // 16 + 1,000, 64, 13.4 and 15.6, 100 + 2,000, 400, 31.8 and 27.9; 7B 547, 1,120, 20.2
  // and 18.8).
  const bool tile = sizeof(T) == 2 && !decode && ((int64_t)units(16) * Hkv > 256 || blocks <= 2);
  a.units = units(tile ? 128 : 16);
  const int64_t pairs = (int64_t)a.units * Hkv;
  // sequences' last tiles taken to be half full
  const double items = std::min<double>(pairs, ((double)b.rows * a.G / 128 + live / 2.0) * Hkv);
  const Kv4Split split = tile ? Kv4Split{kv4_tile_split(items, live, blocks, (int64_t)b.rows * b.n_heads), 4}
                              : kv4_rows_split(pairs, blocks);
  const int64_t most = std::max<int64_t>(1, kv4_partials(decode, (int64_t)b.rows * b.n_heads, blocks) /
                                                ((int64_t)b.rows * b.n_heads));
  a.sblk = std::max(split.blocks, ceil_div(blocks, most));
  a.splits = ceil_div(blocks, a.sblk);
  a.po = ws;
  a.pml = ws + (size_t)b.rows * b.n_heads * a.splits * HD;
  a.by_g = divisor(a.G);
  a.by_hkv = divisor(Hkv);
  a.by_units = divisor(a.units);
  a.by_sblk = divisor(a.sblk);
  a.by_per = divisor(ceil_div(a.G, 16));
  const int64_t wgs = pairs * a.splits;
  if (std::max(wgs, attention_join_wgs(b, a.splits)) >= 1 << 23) return false;  // a launch has fewer than 2^32 threads
  const unsigned grid = (unsigned)wgs;
  if constexpr (sizeof(T) == 2)
    if (tile) kv4_tile_kernel<T, HD><<<grid, 256, 0, s>>>(q, out, a);
  const auto rows = [&](auto nw, auto roomy, auto parts) {
    constexpr int NW = decltype(nw)::value, DP = decltype(parts)::value;
    kv4_rows_kernel<T, HD, NW, decltype(roomy)::value, DP><<<grid * DP, NW * 64, 0, s>>>(q, out, a);
  };
  const auto plan = [&](auto nw) {
    const int parts = kv4_dim_parts(wgs * a.sblk, a.splits > 1 && sizeof(T) == 2, HD / 32);
    if (wgs * split.waves > 2048)  // more than two waves a SIMD
      rows(nw, std::false_type(), std::integral_constant<int, 1>());
    else if (parts == 1)
      rows(nw, std::true_type(), std::integral_constant<int, 1>());
    else if (parts == 2)
      rows(nw, std::true_type(), std::integral_constant<int, 2>());
    else
      rows(nw, std::true_type(), std::integral_constant<int, HD / 32>());
  };
  if (!tile && split.waves == 8)
    plan(std::integral_constant<int, 8>());
  else if (!tile)
    plan(std::integral_constant<int, 4>());
  if (a.splits > 1) launch_attention_join<T>(out, b, a.splits, a.sblk, a.po, a.pml, s);
  return true;
}

template <typename T>
bool launch_kv4_attention(const T *q, T *out, const PrefixBatch &b, float *ws, hipStream_t s) {
  return b.kv.head_dim == 128 ? launch_kv4_hd<T, 128>(q, out, b, ws, s) : launch_kv4_hd<T, 64>(q, out, b, ws, s);
}

#define INST(T) template bool launch_kv4_attention<T>(const T *, T *, const PrefixBatch &, float *, hipStream_t);
INST(float)
INST(bf16_t)
INST(f16_t)
#undef INST

}  // namespace lp
