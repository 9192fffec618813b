// Attention for a batch whose sequences begin with the same prefix.
//
// softmax over a row's keys = (keys of the prefix) joined with (its own keys):
// with (m, l, o) = (largest score, sum of weights, weighted values) of a set of
// keys, two sets join as m = max(m1, m2), l = l1 e^(m1 - m) + l2 e^(m2 - m),
// o likewise.  The prefix's keys are the same for every row, so one workgroup
// takes many rows of the batch (packed rows: token by token, each with the G
// query heads of one KV head) over a range of the prefix's blocks; the rows'
// own keys are walked sequence by sequence.  Both leave (m, l, o) in the
// workspace, and a last pass joins a row's parts.
//
// Keys are walked as a list of cache blocks ("entries"): entry e < nP is block
// e of the prefix, entry nP + i is own block F + i of the sequence, F =
// floor(P / 64) being the first that is not all prefix.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "device.hpp"

namespace lp {

// n / d for n >= 0 with m = floor(2^32 / d) (all ones for d = 1): n m / 2^32 is
// at most one short, which the remainder shows.
struct Divisor {
  uint32_t d, m;
};
__device__ __forceinline__ int div_by(int n, Divisor x) {
  const uint32_t k = __umulhi((uint32_t)n, x.m);
  return (int)(k + ((uint32_t)n - k * x.d >= x.d ? 1 : 0));
}
static Divisor divisor(int d) {
  const uint32_t u = (uint32_t)std::max(d, 1);
  return {u, u > 1 ? (uint32_t)((1ull << 32) / u) : 0xFFFFFFFFu};
}

struct PrefixArgs {
  PrefixBatch b;
  int G;                      // query heads of a KV head
  int nP, F;                  // prefix entries, first own block
  int tiles, splits, sblk;    // shared items: row tiles, splits of the prefix, entries of a split
  int shared_rows;            // 16-row tiles of the shared items that take rows_item (tiles is 0 then)
  int otiles, osplits, oblk;  // own items: row tiles, splits of the own entries, entries of a split
  int own_log, units;         // decode: waves of a row's own item (log 2), workgroups of a split of them
  int parts;                  // splits + osplits
  int direct;                 // one part, written to out by the tile kernel itself
  int whole;                  // decode: a workgroup takes all keys of a row
  Divisor by_g, by_hkv, by_splits, by_osplits, by_units, by_shared, by_per;
  float *po, *pml;            // partial o [rows][n_heads][parts][hd], (m, l) [rows][n_heads][parts][2]
};
// A part's m is the largest score before the scale 1/sqrt(hd), its weights are
// 2^((score - m) c2).
template <int HD>
constexpr float SCORE_C2 = (HD == 64 ? 0.125f : 0.08838834764831845f) * 1.44269504088896341f;

struct PrefixRow {
  int token, head, t;  // t: the token's place in its sequence, or in the batch
};

// Row l of the packed rows from r0 (uniform) on: of all tokens, or of a sequence
// whose first token is `start`.
__device__ __forceinline__ PrefixRow packed_row(const PrefixArgs &a, int start, int r0, int l, int g) {
  const int t0 = div_by(r0, a.by_g), x = r0 - t0 * a.G + l, dt = div_by(x, a.by_g);
  return PrefixRow{start + t0 + dt, g * a.G + x - dt * a.G, t0 + dt};
}

// Sequence j's first row and row count, inside the batch's rows.
__device__ __forceinline__ void seq_rows(const PrefixBatch &b, int j, int &start, int &n) {
  if (!b.seq_start) {
    start = j;
    n = 1;
    return;
  }
  start = min(max(b.seq_start[j], 0), b.rows);
  n = min(max(b.seq_start[j + 1], start), b.rows) - start;
}

// Keys that row i of sequence j sees.
__device__ __forceinline__ int row_ctx(const PrefixBatch &b, int j, int i) {
  const int slot = b.seq_slot[j], p0 = b.seq_pos[j];
  if (slot < 0 || slot >= b.n_slots) return 0;
  const int64_t ctx = (int64_t)p0 + i + 1;
  return p0 < 0 ? 0 : (int)min(ctx, (int64_t)b.max_ctx);
}

// Keys that a packed row sees, -1 if the row does not exist: token t of sequence
// j (which has n rows), or with j < 0 token t of the batch.
__device__ __forceinline__ int packed_ctx(const PrefixArgs &a, int j, int t, int n) {
  if (j >= 0) return t < n && t < a.b.max_new ? row_ctx(a.b, j, t) : -1;
  if (!a.b.seq_start) return t < a.b.rows ? row_ctx(a.b, t, 0) : -1;
  // the last sequence that starts at or before the token, 64 sequences at a time
  const int lane = threadIdx.x & 63;
  int at = -1;
  for (int base = 0; base < a.b.n_seq; base += 64) {
    const int s = base + lane < a.b.n_seq ? a.b.seq_start[base + lane] : INT_MAX;
    if (!__any(__builtin_amdgcn_readlane(s, 0) <= t)) break;
    int k = -1;
#pragma unroll
    for (int step = 32; step; step >>= 1)
      if (__shfl(s, k + step, 64) <= t) k += step;
    if (k == 62 && __shfl(s, 63, 64) <= t) k = 63;
    if (k >= 0) at = base + k;
  }
  if (at < 0 || t >= a.b.rows) return -1;
  int start;
  seq_rows(a.b, at, start, n);
  t -= start;
  return t >= 0 && t < n && t < a.b.max_new ? row_ctx(a.b, at, t) : -1;
}

// Own tile u of RT packed rows: sequence by sequence, each with as many tiles as
// its rows need.  Each wave finds it on its own: an inclusive sum over 64
// sequences at a time, the first whose sum exceeds u.  False past the last.
template <int RT>
__device__ __forceinline__ bool own_tile(const PrefixArgs &a, int u, int &j, int &r0) {
  const int lane = threadIdx.x & 63;
  if (!a.b.seq_start) {  // one row a sequence
    j = div_by(u, a.by_per);
    r0 = (u - j * (int)a.by_per.d) * RT;
    return j < a.b.n_seq;
  }
  for (int base = 0; base < a.b.n_seq; base += 64) {
    int start, n = 0;
    if (base + lane < a.b.n_seq) seq_rows(a.b, base + lane, start, n);
    const int tiles = (int)(((int64_t)min(n, a.b.max_new) * a.G + RT - 1) / RT);
    const int incl = (int)wave_scan((uint64_t)tiles);
    const int total = __builtin_amdgcn_readlane(incl, 63);
    if (u < total) {
      const int k = __popcll(__ballot(incl <= u));  // sequences wholly before the tile
      j = base + k;
      r0 = (__shfl(incl, k, 64) - 1 - u) * RT;  // from the last, whose rows see most
      return true;
    }
    u -= total;
  }
  return false;
}

// An entry's block id, -1 for none.
__device__ __forceinline__ int prefix_entry(const PrefixArgs &a, int slot, int e) {
  int id = -1;
  if (e < a.nP) {
    id = a.b.prefix_blocks[e];
  } else {
    const int blk = a.F + e - a.nP;
    if (slot >= 0 && slot < a.b.n_slots && blk < a.b.kv.max_blocks)
      id = a.b.kv.block_table[(int64_t)slot * a.b.kv.max_blocks + blk];
  }
  return id < a.b.kv.n_blocks ? id : -1;
}

// Operands come in 16-byte pieces: lane l has row (or column) l % 16, elements
// E (l / 16) .. of a run of 4 E.  16-bit types: E = 8, one MFMA over 32; fp32: E =
// 4, four over 4 each, the run taken in the same other order on both sides.
template <typename T>
struct Piece {
  static constexpr int E = 16 / (int)sizeof(T);
  static __device__ __forceinline__ floatx4_t mma(u32x4_tt a, u32x4_tt b, floatx4_t c) {
    if constexpr (sizeof(T) == 2) {
      typedef typename Mfma<T>::v8 v8;
      return Mfma<T>::m16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
      return c;
    }
  }
  // word y of a piece of keys k0 ..: the bits of those in [lo, hi)
  static __device__ __forceinline__ uint32_t keep(int k0, int y, int lo, int hi) {
    if constexpr (sizeof(T) == 2) {
      const int key = k0 + 2 * y;
      return (key >= lo && key < hi ? 0xFFFFu : 0u) | (key + 1 >= lo && key + 1 < hi ? 0xFFFF0000u : 0u);
    } else {
      return k0 + y >= lo && k0 + y < hi ? ~0u : 0u;
    }
  }
  // whether a word holds an infinity or NaN
  static __device__ __forceinline__ bool odd(uint32_t w) {
    if constexpr (std::is_same_v<T, float>) return (w & 0x7F800000u) == 0x7F800000u;
    constexpr uint32_t X = std::is_same_v<T, bf16_t> ? 0x7F80u : 0x7C00u;
    return (w & X) == X || (w & X << 16) == X << 16;
  }
};

// Base-2 score past which a tile takes the maximum off before the scale.  Up to
// here its rounded mc is within 2^-19, which moves the sums of a block or part
// by 1.3e-6 against those of the others, as they meet at the maximum itself: no
// more than the rounding of fp32 scores does.  (Three prompts of 2,100 over 4,096
// tokens, 70B heads: scores past it 703 us, under it 698; sums corrected for mc's
// rounding at every new maximum 686 and 703.)
constexpr float TILE_LARGE = 64.f;

// Many rows of a 16-bit type over a range of entries, on 32x32x16 MFMAs: a
// workgroup owns 128 packed rows, 32 to a wave, and walks its entries' blocks,
// which are copied into LDS for all its waves (two stages: the next block lands while the
// current one is used) in the cache's own order, with the 16-byte pieces of a
// row XOR-swizzled against bank conflicts.
//   S^T = K Q^T: a lane holds one row's scores, so the softmax's maximum and sum
//   run in its registers and meet the wave's other half once a block.  The K row
//   of MFMA row i is i with bits 2 and 3 swapped: then the eight weights a lane
//   holds of each 16 keys are consecutive keys, the B operand of O^T += V^T P^T,
//   and P never leaves the registers.
//   The running maximum moves in every block that raises it for a row of the
//   wave, so the largest weight is 1 (within TILE_LARGE's 1.3e-6) before it is
//   rounded to 16 bits.
// V at places that no row of the tile sees is cleared in LDS (stale entries may
// hold anything, and 0 * NaN is not 0).  Places that only some of its rows see
// are not: their weight is 0 for the others, which is enough unless V is
// infinite or NaN there.  A tile whose result is not finite is therefore
// computed again with every row's own V (`careful`), once.
template <typename T, int HD>
__device__ __forceinline__ void tile_item(const T *__restrict__ q, T *__restrict__ out, const PrefixArgs &a, int idx,
                                          int g, char *lds) {
  typedef typename Mfma<T>::v8 v8;
  constexpr int QW = 4, RT = QW * 32;  // waves, rows
  constexpr int KS = HD / 16;         // contraction steps of S over head_dim
  constexpr int NT = HD / 32;         // 32-dim tiles of O^T
  constexpr int CK = HD / 8;          // 16-byte pieces of a K row
  constexpr int PB = 64 * HD * 2;     // bytes of a K (or V) block
  constexpr int STAGE = 2 * PB;
  constexpr int ND = PB / 1024 / QW;  // 1 KB copies per wave and block, K and V each
  constexpr float c2 = SCORE_C2<HD>;
  const int Hkv = a.b.kv.n_kv_heads, Hq = a.b.n_heads, P = a.b.prefix_len;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l32 = lane & 31, hh = lane >> 5;
  floatx16_t o[NT];
  float mref, lsum;
  int r0 = 0, part = 0, start = 0, seen = -1;
  bool walked = false;
  PrefixRow w{};
  int *again = (int *)(lds + 2 * STAGE);
  // The item from its index to its (m, l, o); returns whether some rows of the
  // wave saw a block only in part, or leaves early (a tile past the last).
  // Called again for a tile whose result is not finite, it reads everything
  // anew: what it kept over the first walk would cost that one's registers.
  auto item = [&](auto careful_, int idx, bool &none) __attribute__((always_inline)) {
    constexpr bool careful = decltype(careful_)::value;
    int j = -1, e0, e1, most = INT_MAX, slot = -1, n = a.b.rows;
    start = 0;
    none = false;
    if (idx < a.tiles * a.splits) {
      const int tile = div_by(idx, a.by_splits);
      part = idx - tile * a.splits;
      r0 = tile * RT;
      e0 = part * a.sblk;
      e1 = min(a.nP, e0 + a.sblk);
    } else {
      idx -= a.tiles * a.splits;
      const int u = div_by(idx, a.by_osplits), s = idx - u * a.osplits;
      if (!own_tile<RT>(a, u, j, r0)) {
        none = true;
        return false;
      }
      part = a.splits + s;
      slot = a.b.seq_slot[j];
      seq_rows(a.b, j, start, n);
      most = row_ctx(a.b, j, min(div_by(r0 + RT - 1, a.by_g), n - 1));  // the last row sees most
      e0 = (a.splits ? a.nP : 0) + s * a.oblk;
      const int blocks = (most + KV_BLOCK - 1) / KV_BLOCK;
      e1 = min(e0 + a.oblk, most > P ? a.nP + blocks - a.F : blocks);
    }
    walked = e0 < e1;
    // What the first copies wait for is requested first, with the rows' q: a
    // walk of few blocks is one memory round trip after the other.
    w = packed_row(a, start, r0, wave * 32 + l32, g);
    v8 qb[KS];  // Q^T as the B operand: this lane's row, dims 16 k + 8 hh ..
    {
      const T *qr = q + ((int64_t)(w.t < n ? w.token : 0) * Hq + w.head) * HD + hh * 8;
#pragma unroll
      for (int k = 0; k < KS; ++k) qb[k] = load8<T>(qr + k * 16);
    }
    // Byte offsets of the entries' blocks (head included), -1 for none: lane i
    // holds that of entry win + i, the wave reads them back with readlane.
    int win = e0, off_lo, off_hi;
    auto window = [&]() __attribute__((always_inline)) {
      int64_t off = -1;
      if (win + lane < e1) {
        const int id = prefix_entry(a, slot, win + lane);
        if (id >= 0) off = ((int64_t)id * Hkv + g) * PB;
      }
      off_lo = (int)off;
      off_hi = (int)(off >> 32);
      asm volatile("" : "+v"(off_lo), "+v"(off_hi));  // the wait for the load stands here
    };
    auto offset = [&](int e) __attribute__((always_inline)) {
      return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_hi, e - win) << 32) |
                       (uint32_t)__builtin_amdgcn_readlane(off_lo, e - win));
    };
    constexpr int KR = 1024 / (HD * 2);
    const uint32_t lds0 = lds_addr(lds) + wave * ND * 1024;
    auto swz = [](int row) __attribute__((always_inline)) { return CK == 16 ? row & 15 : (row >> 1) & 7; };
    uint32_t ko[ND], vo[ND];  // byte offsets of this lane's pieces inside a block
#pragma unroll
    for (int c = 0; c < ND; ++c) {
      const int m = wave * ND + c, kr = m * KR + lane / CK, vr = m * 8 + (lane >> 3);
      ko[c] = kr * HD * 2 + ((lane % CK) ^ swz(kr)) * 16;
      vo[c] = vr * KV_BLOCK * 2 + ((lane & 7) ^ ((vr >> 1) & 7)) * 16;
    }
    bool have[2];  // the stage holds a block
    auto issue = [&](int e) __attribute__((always_inline)) {
      if (e >= win + 64) {
        win = e;
        window();
      }
      const int64_t off = offset(e);
      const int b = (e - e0) & 1;
      have[0] = b ? have[0] : off >= 0;
      have[1] = b ? off >= 0 : have[1];
      if (off < 0) return;
      const uint32_t st = lds0 + b * STAGE;
#pragma unroll
      for (int c = 0; c < ND; ++c) {
        dma16s((const char *)a.b.kv.k + off, ko[c], st + c * 1024);
        dma16s((const char *)a.b.kv.v + off, vo[c], st + PB + c * 1024);
      }
    };
    if (e0 < e1) {  // the first two blocks
      window();
      issue(e0);
      if (e0 + 1 < e1) issue(e0 + 1);
    }
    seen = packed_ctx(a, j, w.t, n);
    const int wctx = max(seen, 0);
    // rows that do not exist or see nothing (zeros at the end, whatever is summed
    // for them) ask for no mask
    const int ctx = wctx ? wctx : INT_MAX;
    const int ctx_lo = (int)wave_min_u32((uint32_t)ctx);
    const int ctx_top = (int)~wave_min_u32(~(uint32_t)wctx);
    const int krow = (l32 & 0x13) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);
    const int kfb = krow * HD * 2, kfx = (hh ^ swz(krow)) << 4;
    const int vfb = l32 * KV_BLOCK * 2, vfx = (hh ^ ((l32 >> 1) & 7)) << 4;

#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
    // running maximum (raw scores), its base-2 value, this half's share of the sum
    float mc = 0.f;
    mref = -INFINITY;
    lsum = 0.f;
    bool large = false;   // wave-uniform: a row's |mc| is past TILE_LARGE
    bool masked = false;  // wave-uniform: a block that only some rows see whole
    for (int e = e0; e < e1; ++e) {
      const bool mine = e < a.nP;
      const int base = mine ? e * KV_BLOCK : (a.F + e - a.nP) * KV_BLOCK;
      const int lo = mine ? 0 : max(0, P - base);
      const int hi = min(KV_BLOCK, (mine ? min(P, most) : most) - base);
      // this wave's copies of the block have landed; after the barrier everyone's
      // have, and the stage of the block before is free
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      const int stage = (e - e0) & 1;
      char *ks = lds + stage * STAGE, *vs = ks + PB;
      const bool there = stage ? have[1] : have[0];
      if (there && (lo > 0 || hi < KV_BLOCK)) {  // clear V outside [lo, hi)
#pragma unroll
        for (int i = threadIdx.x; i < HD * 8; i += QW * 64) {
          const int row = i >> 3, k0 = (i & 7) * 8;
          if (k0 >= lo && k0 + 8 <= hi) continue;
          char *p = vs + row * KV_BLOCK * 2 + ((i & 7) ^ ((row >> 1) & 7)) * 16;
          u32x4_tt v = u32x4_tt{0, 0, 0, 0};
          if (k0 + 8 > lo && k0 < hi) {
            v = *(const u32x4_tt *)p;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int k = k0 + 2 * x;
              v[x] &= (k >= lo && k < hi ? 0xFFFFu : 0u) | (k + 1 >= lo && k + 1 < hi ? 0xFFFF0000u : 0u);
            }
          }
          *(u32x4_tt *)p = v;
        }
        __syncthreads();
      }
      if (e > e0 && e + 1 < e1) issue(e + 1);
      if (!there || base + lo >= ctx_top) continue;  // no block, or wholly past this wave's rows
      floatx16_t s[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const v8 f = *(const v8 *)(ks + kfb + t * 32 * HD * 2 + (kfx ^ (k << 5)));
          s[t] = Mfma<T>::m32(f, qb[k], s[t]);
        }
      }
      // s[t][r]: key 32 t + 16 (r / 8) + 8 hh + r % 8 of the block
      const bool partly = lo > 0 || base + hi > ctx_lo || hi < KV_BLOCK;
      const int end = min(hi, max(ctx - base, 0));  // the row's keys: [lo, end)
      if (base + hi > ctx_lo) masked = true;
      if (partly) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = t * 32 + (r >> 3) * 16 + hh * 8 + (r & 7);
            if (key < lo || key >= end) s[t][r] = -INFINITY;
          }
      }
      float mx = s[0][0];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r]);
      mx = half_swap_max(mx);
      if (__any(mx > mref)) {
        const float nm = fmaxf(mref, mx);
        const float corr = nm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((mref - nm) * c2);
        mref = nm;
        mc = nm == -INFINITY ? 0.f : nm * c2;  // a row that has seen no key yet
        large = __any(fabsf(mc) > TILE_LARGE);
        lsum *= corr;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[t][r] *= corr;
      }
      // s c2 - mc in one FMA is off 0 at the maximum by what mc's rounding left
      // out: large scores have the maximum taken off before the product instead
      float mo = mc;
      if (large) {
        const float m0 = mref == -INFINITY ? 0.f : mref;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[t][r] -= m0;
        mo = 0.f;
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
          // the one rounding below 32 bits before the result's: the matrix instruction
          // of 16-bit V takes 16-bit weights (their sum stays fp32 and unrounded)
          pb[t * 2 + u] = pack8<T>(p);
        }
      if (careful && partly) {
        // row by row, each with V of its own keys alone
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll 1
          for (int i = 0; i < 32; ++i) {
            const int lim = __builtin_amdgcn_readlane(end, i);
            int at = vfb;
            asm volatile("" : "+v"(at));  // not held in registers over the rows
            floatx16_t acc = o[t];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              u32x4_tt f = *(const u32x4_tt *)(vs + at + t * 32 * KV_BLOCK * 2 + (vfx ^ (k << 5)));
#pragma unroll
              for (int x = 0; x < 4; ++x) f[x] &= Piece<T>::keep(k * 16 + hh * 8, x, 0, lim);
              acc = Mfma<T>::m32(__builtin_bit_cast(v8, f), pb[k], acc);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) o[t][r] = l32 == i ? acc[r] : o[t][r];
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const v8 f = *(const v8 *)(vs + vfb + t * 32 * KV_BLOCK * 2 + (vfx ^ (k << 5)));
            o[t] = Mfma<T>::m32(f, pb[k], o[t]);
          }
      }
    }
    return masked;
  };
  if (threadIdx.x == 0) *again = 0;  // before the walk's first barrier, or the one below
  bool none;
  const bool masked = item(std::false_type(), idx, none);
  if (none) return;
  __syncthreads();
  if (masked) {
    float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r & 3] = fmaf(o[t][r], 0.f, z[r & 3]);
    if (seen > 0 && !(z[0] + z[1] + (z[2] + z[3]) == 0.f)) *again = 1;
  }
  __syncthreads();  // the last block is used by now: LDS is free below
  if (*again) {
    int opaque = idx;
    asm volatile("" : "+s"(opaque));
    item(std::true_type(), opaque, none);
    __syncthreads();
  }
  const bool live = seen >= 0;
  const int wctx = max(seen, 0);
  if (!wctx) {
    mref = -INFINITY;
    lsum = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
  }
  // o[t][r]: dim 32 t + 8 (r / 4) + 4 hh + r % 4 of this lane's row
  const float sum = half_swap_sum(lsum);
  const int64_t row = (int64_t)w.token * Hq + w.head;
  if (a.direct) {
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
    for (int t = 0; t < NT; ++t) store_o32(out + row * HD + t * 32, o[t], inv, hh, live);
  } else {
    // Through LDS, so that a row's dims leave as one run of bytes: 16-byte
    // pieces XOR-swizzled by the row, the wave's 32 rows in a place of its own.
    constexpr int LR = HD / 4, RI = 64 / LR;  // lanes of a row, rows of a store
    char *own = lds + wave * 32 * HD * 4;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int piece = t * 8 + r / 2 + hh;
        *(float4 *)(own + l32 * HD * 4 + ((piece ^ (l32 % LR)) * 16)) =
            make_float4(o[t][r], o[t][r + 1], o[t][r + 2], o[t][r + 3]);
      }
    if (live && hh == 0) *(float2 *)(a.pml + (row * a.parts + part) * 2) = make_float2(mref, sum);
    const uint32_t rows_live = walked ? (uint32_t)__ballot(live) : 0;  // the join skips o of empty parts
#pragma unroll 4
    for (int i = 0; i < 32 / RI; ++i) {
      const int x = i * RI + lane / LR;
      const float4 v = *(const float4 *)(own + x * HD * 4 + (((lane % LR) ^ (x % LR)) * 16));
      const PrefixRow y = packed_row(a, start, r0, wave * 32 + x, g);
      if (rows_live >> x & 1)
        *(float4 *)(a.po + (((int64_t)y.token * Hq + y.head) * a.parts + part) * HD + lane % LR * 4) = v;
    }
  }
}

template <typename T, int HD>
constexpr int TILE_LDS = 4 * 64 * HD * 2 + 16;  // two stages of K and V, a flag

// Prefill in 16-bit types.  Bound by the matrix cores with the softmax's vector
// work beside them: three prompts of 2,100 over 4,096 tokens, 70B heads in bf16,
// 690 us, 956 TFLOP/s (a large library product on the same card 1,252).
template <typename T, int HD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void prefix_tile_kernel(
    const T *__restrict__ q, T *__restrict__ out, PrefixArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[TILE_LDS<T, HD>];
  // KV head fastest: with 8 of them each XCD's L2 holds one head's blocks
  const int i = div_by(blockIdx.x, a.by_hkv);
  tile_item<T, HD>(q, out, a, i, blockIdx.x - i * a.b.kv.n_kv_heads, lds);
}

// Few rows over a range of entries, on 16x16 MFMAs: up to 16 packed rows of a KV
// head, walked 32 keys at a time; waves that share an item take half blocks in turn.
// Each wave has its own LDS for K and V of 32 keys: K is copied there while the
// softmax of the keys before runs, V while the scores do.  (Fragments loaded
// straight from the cache ask for 16 rows with every four lanes on four lines:
// 21 bytes a clock and CU, 6,200 clocks per 32 keys with eight waves, against
// 1,900 with one.)  Online softmax per wave; P goes through LDS into the A
// operand's layout; the waves' (m, l, o) meet in LDS at the end.  Own items: the
// query heads of one row, or in fp32 prefill 16 packed rows of a sequence.
// Shared items (batches of few rows, and fp32): packed rows.

template <typename T, int HD>
constexpr int ROWS_KV = 32 * HD * (int)sizeof(T);  // bytes of 32 keys, K or V
template <typename T>
constexpr int ROWS_LP = 32 + 16 / (int)sizeof(T);  // a row of P in LDS
template <typename T, int HD, int NW>
constexpr int ROWS_LDS = NW * (2 * ROWS_KV<T, HD> + 16 * ROWS_LP<T> * (int)sizeof(T) + 2 * 16 * 4);

// With WHOLE an item is all that the query heads of one row see, prefix and own
// entries, and its result goes to out.
template <typename T, int HD, int NW, bool WHOLE>
__device__ __forceinline__ void rows_item(const T *__restrict__ q, T *__restrict__ out, const PrefixArgs &a, int idx,
                                          int g, char *lds) {
  constexpr int S = (int)sizeof(T), E = Piece<T>::E;
  constexpr int KS = HD / (4 * E), NT = HD / 16, PS = 32 / (4 * E), LP = ROWS_LP<T>;
  constexpr float c2 = SCORE_C2<HD>;
  constexpr int KV = ROWS_KV<T, HD>, ND = KV / 1024;         // copies of 1 KB
  constexpr int CK = HD / E, KR = 64 / CK;                   // pieces of a K row, rows of a copy
  constexpr int CV = 32 / E, VR = 64 / CV;                   // pieces of a V row (32 keys of a dim), rows of a copy
  constexpr int KX = CK < 16 ? CK - 1 : 15;                  // pieces are XOR-swizzled by the row's low bits
  static_assert(16 * HD * 4 <= 2 * KV, "o of a wave in the place of its K and V");
  auto vx = [](int row) __attribute__((always_inline)) { return CV == 4 ? (row >> 1) & 3 : row & 7; };
  float *wm = (float *)(lds + NW * 2 * KV), *wl = wm + NW * 16;  // [NW][16] each
  T(*pls)[LP] = (T(*)[LP])(lds + NW * (2 * KV + 2 * 16 * 4));    // [NW * 16][LP]
  const int Hkv = a.b.kv.n_kv_heads, Hq = a.b.n_heads, P = a.b.prefix_len;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r16 = lane & 15, quad = lane >> 4;
  pls += wave * 16;
  int j = -1, r0, e0, e1, part = 0, slot = -1, start = 0, n = 1;
  const int shared = WHOLE ? 0 : a.shared_rows * a.splits;
  // waves that share an item's entries: all, or of a row's own ones 2^own_log
  int log = NW == 8 ? 3 : 2;
  if (idx < shared) {
    part = div_by(idx, a.by_shared);
    r0 = (idx - part * a.shared_rows) * 16;
    e0 = part * a.sblk;
    e1 = min(a.nP, e0 + a.sblk);
  } else {
    idx -= shared;
    if (!WHOLE) log = a.own_log;
    // all rows' first splits, then their second ones: the grid ends with what few have
    const int s = WHOLE ? 0 : div_by(idx, a.by_units);
    const int u = ((idx - s * a.units) << (WHOLE ? 0 : 2 - log)) + (wave >> log);
    // past the last tile (prefill's bound of them is loose): nothing, but for the barrier
    bool some = u < a.otiles && own_tile<16>(a, u, j, r0);
    if (!some) j = 0, r0 = 0;
    part = a.splits + s;
    slot = a.b.seq_slot[j];
    seq_rows(a.b, j, start, n);
    if (!some) n = 0;
    // the last row sees most
    const int ctx = some ? row_ctx(a.b, j, min(div_by(r0 + 15, a.by_g), n - 1)) : 0;
    const int blocks = (ctx + KV_BLOCK - 1) / KV_BLOCK;
    const int end = ctx > P ? a.nP + blocks - a.F : WHOLE ? blocks : 0;
    e0 = WHOLE ? 0 : a.nP + s * a.oblk;
    e1 = WHOLE ? end : min(e0 + a.oblk, end);
  }
  const bool own = j >= 0;
  const int nth = wave & ((1 << log) - 1);  // the wave's place among them
  // Byte offsets of the entries' blocks (head included), -1 for none: lane i
  // holds that of entry e0 + i (an item has at most 64).
  int64_t off = -1;
  if (e0 + lane < e1) {
    const int id = prefix_entry(a, slot, e0 + lane);
    if (id >= 0) off = ((int64_t)id * Hkv + g) * (KV_BLOCK * HD * S);
  }
  const int off_lo = (int)off, off_hi = (int)(off >> 32);
  const PrefixRow w = packed_row(a, start, r0, r16, g);
  const int seen_ = packed_ctx(a, j, w.t, n), ctx = max(seen_, 0);
  const bool live = seen_ >= 0;
  const int ctx_top = (int)~wave_min_u32(~(uint32_t)ctx);
  // rows that see nothing get zeros at the end, whatever is summed for them
  const int ctx_lo = (int)wave_min_u32(ctx ? (uint32_t)ctx : (uint32_t)INT_MAX);
  // Entries with a block of which some row sees the first half, the second half,
  // of those that are this wave's: all of the item's, or where waves share it one
  // half of every 2^(log - 1)-th.
  const bool pre = e0 + lane < a.nP;
  const int first = pre ? (e0 + lane) * KV_BLOCK : (a.F + e0 + lane - a.nP) * KV_BLOCK;
  const int from = pre ? 0 : P, to = min(pre ? P : INT_MAX, ctx_top);  // its positions [from, to)
  const uint64_t mine = log ? ~0ull / ((1ull << (1 << (log - 1))) - 1) << (nth >> 1) : ~0ull;
  const bool some_key = off >= 0 && first < to && from < to;
  const uint64_t half0 = log && nth & 1 ? 0 : __ballot(some_key && from < first + 32) & mine;
  const uint64_t half1 = log && !(nth & 1) ? 0 : __ballot(some_key && first + 32 < to) & mine;
  uint64_t left = half0 | half1;
  // copies into this wave's LDS
  char *ks = lds + wave * 2 * KV, *vs = ks + KV;
  const uint32_t kl = lds_addr(ks), vl = kl + KV;
  uint32_t ko[16 / KR];  // byte offsets of this lane's pieces, rows 0 .. 15
#pragma unroll
  for (int c = 0; c < 16 / KR; ++c) {
    const int row = c * KR + lane / CK;
    ko[c] = row * HD * S + ((lane % CK) ^ (row & KX)) * 16;
  }
  const uint32_t vo = lane / CV * KV_BLOCK * S + ((lane % CV) ^ vx(lane / CV)) * 16;
  int64_t at;
  auto place = [&](int i, int h) __attribute__((always_inline)) {  // half h of entry e0 + i
    at = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_hi, i) << 32) |
                   (uint32_t)__builtin_amdgcn_readlane(off_lo, i));
    return __builtin_amdgcn_readlane(first, i) + h * 32;
  };
  auto copy_k = [&](int h) __attribute__((always_inline)) {
    const char *kb = (const char *)a.b.kv.k + at + h * KV;
#pragma unroll
    for (int c = 0; c < ND; ++c) dma16s(kb + c / (16 / KR) * 16 * HD * S, ko[c % (16 / KR)], kl + c * 1024);
  };
  auto copy_v = [&](int h) __attribute__((always_inline)) {
    const char *vb = (const char *)a.b.kv.v + at + h * 32 * S;
#pragma unroll
    for (int c = 0; c < ND; ++c) dma16s(vb + c * VR * KV_BLOCK * S, vo, vl + c * 1024);
  };
  u32x4_tt qa[KS];
  const T *qrow = q + ((int64_t)(live ? w.token : 0) * Hq + w.head) * HD + quad * E;
#pragma unroll
  for (int k = 0; k < KS; ++k) qa[k] = *(const u32x4_tt *)(qrow + k * 4 * E);
  // row 4 quad + i: running maximum (raw scores) and this lane's share of the
  // sum; o[nt][i]: its dim nt * 16 + r16
  float mx[4], sm[4];
  int rctx[4];
  floatx4_t o[NT], s[2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) o[nt] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) mx[i] = -INFINITY, sm[i] = 0.f, rctx[i] = __shfl(ctx, 4 * quad + i, 64);
  if (left) {
    int i = __builtin_ctzll(left), h = (int)(~half0 >> i & 1), base = place(i, h);
    copy_k(h);
    copy_v(h);
    for (int halves = __builtin_popcountll(half0) + __builtin_popcountll(half1); halves > 0; --halves) {
      // keys [lo, hi) of the 32 at `base` are there
      const int lo = max(0, __builtin_amdgcn_readlane(from, i) - base);
      const int hi = min(32, __builtin_amdgcn_readlane(to, i) - base);
      const int here = base;
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(ND) : "memory");  // K is there, V may not be
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) s[nt] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          const char *f = ks + (nt * 16 + r16) * HD * S + (((k * 4 + quad) ^ (r16 & KX)) * 16);
          s[nt] = Piece<T>::mma(qa[k], *(const u32x4_tt *)f, s[nt]);
        }
      if (halves > 1) {
        h = (int)(half1 >> i & 1) & (h ^ 1);
        if (!h) {
          left &= left - 1;
          i = __builtin_ctzll(left);
          h = (int)(~half0 >> i & 1);
        }
        base = place(i, h);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K has been read
        copy_k(h);
      }
      // s[nt][y]: row 4 quad + y, key nt * 16 + r16, to weights in LDS
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int end = min(hi, rctx[y] - here);
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          const int key = nt * 16 + r16;
          s[nt][y] = key >= lo && key < end ? s[nt][y] : -INFINITY;
        }
        const float v = fmaxf(mx[y], row16_max(fmaxf(s[0][y], s[1][y])));
        const float m0 = v == -INFINITY ? 0.f : v;
        const float corr = mx[y] == v ? 1.f : __builtin_amdgcn_exp2f((mx[y] - v) * c2);
        mx[y] = v;
        sm[y] *= corr;
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          const float p = __builtin_amdgcn_exp2f((s[nt][y] - m0) * c2);
          sm[y] += p;
          pls[4 * quad + y][nt * 16 + r16] = round_to<T>(p);  // as in tile_item; fp32 keeps all bits
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[nt][y] *= corr;
      }
      u32x4_tt pa[PS];
#pragma unroll
      for (int k = 0; k < PS; ++k) pa[k] = *(const u32x4_tt *)&pls[r16][(k * 4 + quad) * E];
      if (halves > 1)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(ND) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      // V outside [lo, hi) is stale and may hold anything, and 0 * NaN is not 0.
      // Inside, where rows see different keys, a weight of 0 cancels V unless it
      // is infinite or NaN: then row by row, each with V of its own keys alone.
      bool odd = false;
      if (ctx_lo < here + hi) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < PS; ++k) {
            const int dim = nt * 16 + r16;
            const u32x4_tt f = *(const u32x4_tt *)(vs + dim * 32 * S + (((k * 4 + quad) ^ vx(dim)) * 16));
#pragma unroll
            for (int y = 0; y < 4; ++y) odd |= Piece<T>::odd(f[y]);
          }
        odd = __any(odd);
      }
      if (odd) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          int dim = nt * 16 + r16;
#pragma unroll 1
          for (int r = 0; r < 16; ++r) {
            const int lim = min(hi, __builtin_amdgcn_readlane(ctx, r) - here);
            asm volatile("" : "+v"(dim));  // V is read anew, not held in registers over the rows
            floatx4_t acc = o[nt];
#pragma unroll
            for (int k = 0; k < PS; ++k) {
              u32x4_tt f = *(const u32x4_tt *)(vs + dim * 32 * S + (((k * 4 + quad) ^ vx(dim)) * 16));
#pragma unroll
              for (int y = 0; y < 4; ++y) f[y] &= Piece<T>::keep((k * 4 + quad) * E, y, lo, lim);
              acc = Piece<T>::mma(pa[k], f, acc);
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) o[nt][y] = 4 * quad + y == r ? acc[y] : o[nt][y];
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < PS; ++k) {
          u32x4_tt keep;
#pragma unroll
          for (int y = 0; y < 4; ++y) keep[y] = Piece<T>::keep((k * 4 + quad) * E, y, lo, hi);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const int dim = nt * 16 + r16;
            const u32x4_tt f = *(const u32x4_tt *)(vs + dim * 32 * S + (((k * 4 + quad) ^ vx(dim)) * 16));
            o[nt] = Piece<T>::mma(pa[k], f & keep, o[nt]);
          }
        }
      }
      if (halves > 1) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V has been read
        copy_v(h);
      }
    }
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // o goes where K and V were
  const int nrows = own && !a.b.seq_start ? min(16, a.G - r0) : 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * quad + i;
    const float t = row16_sum(sm[i]);
    if (r16 == 0) wm[wave * 16 + r] = mx[i], wl[wave * 16 + r] = t;
    if (r < nrows) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) ((float *)ks)[r * HD + nt * 16 + r16] = o[nt][i];
    }
  }
  __syncthreads();
  if (!WHOLE && !a.b.seq_start && e0 >= e1) return;  // decode's join reads no such part
  // a wave a row: its lanes over the dims
  const int w0 = wave - nth;
  for (int r = nth; r < nrows; r += 1 << log) {
    const int token = __builtin_amdgcn_readlane(w.token, r), h = __builtin_amdgcn_readlane(w.head, r);
    if (!__builtin_amdgcn_readlane((int)live, r)) continue;
    float M = -INFINITY, L = 0.f, v[HD / 64];
    for (int k = w0; k < w0 + (1 << log); ++k) M = fmaxf(M, wm[k * 16 + r]);
#pragma unroll
    for (int d = 0; d < HD / 64; ++d) v[d] = 0.f;
    for (int k = w0; k < w0 + (1 << log); ++k) {
      const float m = wm[k * 16 + r], f = m == M ? 1.f : __builtin_amdgcn_exp2f((m - M) * c2);
      L += f * wl[k * 16 + r];
#pragma unroll
      for (int d = 0; d < HD / 64; ++d) v[d] += f * ((const float *)(lds + k * 2 * KV))[r * HD + d * 64 + lane];
    }
    const bool none = __builtin_amdgcn_readlane(ctx, r) == 0;
    const int64_t row = (int64_t)token * Hq + h, rec = row * a.parts + part;
#pragma unroll
    for (int d = 0; d < HD / 64; ++d) {
      if (none) v[d] = 0.f;
      if constexpr (WHOLE)
        out[row * HD + d * 64 + lane] = round_to<T>(L == 0.f ? 0.f : v[d] / L);
      else if (e0 < e1)
        a.po[rec * HD + d * 64 + lane] = v[d];
    }
    if (!WHOLE && lane == 0) *(float2 *)(a.pml + rec * 2) = none ? make_float2(-INFINITY, 0.f) : make_float2(M, L);
  }
}

// Decode in 16-bit types: shared items of 128 rows, which the matrix cores
// bound, and items of few rows (the rows' own, and the shared ones of small
// batches), which memory bounds; the longer ones first.  64 rows, 8B heads in
// fp16 over 2,000 + 300 tokens: 26.6 us, 3.3 TB/s; 70B heads in bf16 over 16,000 +
// 150: 56 us, 600 TFLOP/s.
template <typename T, int HD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void prefix_decode_kernel(
    const T *__restrict__ q, T *__restrict__ out, PrefixArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[std::max(TILE_LDS<T, HD>, ROWS_LDS<T, HD, 4>)];
  const int i = div_by(blockIdx.x, a.by_hkv), g = blockIdx.x - i * a.b.kv.n_kv_heads, tiles = a.tiles * a.splits;
  if (i < tiles)
    tile_item<T, HD>(q, out, a, i, g, lds);
  else
    rows_item<T, HD, 4, false>(q, out, a, i - tiles, g, lds);
}

// Items of few rows alone (fp32, in both phases); latency at the sizes fp32
// serves: five prompts of 20 over 64 tokens, four heads of 64, 9.3 us.
template <typename T, int HD>
__global__ __launch_bounds__(256) void prefix_rows_kernel(const T *__restrict__ q, T *__restrict__ out, PrefixArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[ROWS_LDS<T, HD, 4>];
  const int i = div_by(blockIdx.x, a.by_hkv);
  rows_item<T, HD, 4, false>(q, out, a, i, blockIdx.x - i * a.b.kv.n_kv_heads, lds);
}

// Small decode batches: a workgroup of eight waves (four where LDS holds no
// more) per row and KV head takes all of its keys, the prefix's too.  Every row
// reads the prefix for itself, from the L2, and no second launch joins anything.
// Bound by one memory trip after another (slot, block id, K and V, three half
// blocks a wave): one row over 553 + 60 tokens, 8B heads, 10.2 us.
template <typename T, int HD>
constexpr int WHOLE_WAVES = HD * sizeof(T) <= 256 ? 8 : 4;
template <typename T, int HD>
__global__ __launch_bounds__(512) void prefix_row_kernel(const T *__restrict__ q, T *__restrict__ out,
                                                           PrefixArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[ROWS_LDS<T, HD, WHOLE_WAVES<T, HD>>];
  const int i = div_by(blockIdx.x, a.by_hkv);
  rows_item<T, HD, WHOLE_WAVES<T, HD>, true>(q, out, a, i, blockIdx.x - i * a.b.kv.n_kv_heads, lds);
}

// Joins the parts of a (token, head), a wave each, or with more than 16 parts
// four: its lanes hold the weights of 64 parts first, then the dims of U parts
// at a time; of four waves each takes 16 of the 64, and they add up in LDS (one
// row of 32 heads, 66 parts: the call 26.2 -> 22.3 us).  Bound by memory: 633
// rows of 32 heads, three parts each, 9.2 us, 4.0 TB/s.
template <typename T, int HD, int U, int W>
__global__ __launch_bounds__(256) void prefix_join_kernel(T *__restrict__ out, PrefixArgs a) {
  static_assert(W == 1 || (W == 4 && U == 16), "a fourth of 64 parts in one step");
  constexpr int DPL = HD / 64;
  constexpr float c2 = SCORE_C2<HD>;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t row = W == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  const int64_t t = row / a.b.n_heads;
  if (t >= a.b.rows) return;
  int parts = a.parts;
  if (a.b.seq_start) {
    if (t < a.b.seq_start[0] || t >= a.b.seq_start[a.b.n_seq]) return;
  } else if (a.osplits) {  // decode: a row has as many own parts as its context needs
    const int ctx = row_ctx(a.b, (int)t, 0);
    const int own = ctx > a.b.prefix_len ? (ctx + KV_BLOCK - 1) / KV_BLOCK - a.F : 0;
    parts = a.splits + (own + a.oblk - 1) / a.oblk;
  }
  const float2 *ml = (const float2 *)a.pml + row * a.parts;
  const float *po = a.po + row * a.parts * HD + lane * DPL;
  float M = -INFINITY, L = 0.f, o[DPL];
#pragma unroll
  for (int d = 0; d < DPL; ++d) o[d] = 0.f;
  for (int p0 = 0; p0 < parts; p0 += 64) {
    const int n = min(64, parts - p0);
    const float2 x = lane < n ? ml[p0 + lane] : make_float2(-INFINITY, 0.f);
    const float mn = fmaxf(M, wave_max(x.x));
    const float f0 = M == mn ? 1.f : __builtin_amdgcn_exp2f((M - mn) * c2);
    const uint64_t filled = __ballot(x.x != -INFINITY);  // a part without keys has no o
    const float f = x.x == -INFINITY ? 0.f : x.x == mn ? 1.f : __builtin_amdgcn_exp2f((x.x - mn) * c2);
    L = L * f0 + wave_sum(f * x.y);
    M = mn;
#pragma unroll
    for (int d = 0; d < DPL; ++d) o[d] *= f0;
    for (int p = W == 1 ? 0 : wave * U; p < n; p += W * U) {
      // all requested before any is used, and before it is known which parts have
      // keys (half a microsecond a call); past the last part: 0 of that part again
      float v[U][DPL];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int d = 0; d < DPL; ++d) v[u][d] = po[(int64_t)(p0 + min(p + u, n - 1)) * HD + d];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float fu = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), p + u));
#pragma unroll
        for (int d = 0; d < DPL; ++d) o[d] += fu * (filled >> (p + u) & 1 ? v[u][d] : 0.f);
      }
    }
  }
  if constexpr (W > 1) {
    __shared__ float sums[W - 1][HD];
#pragma unroll
    for (int d = 0; d < DPL; ++d)
      if (wave) sums[wave - 1][lane * DPL + d] = o[d];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int d = 0; d < DPL; ++d)
#pragma unroll
      for (int w = 0; w < W - 1; ++w) o[d] += sums[w][lane * DPL + d];
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
#pragma unroll
  for (int d = 0; d < DPL; ++d) out[row * HD + lane * DPL + d] = round_to<T>(o[d] * inv);
}

// ------------------------------------------------------------------ plan

static int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// A decode batch whose rows each see at most WHOLE_ENTRIES blocks, and whose rows
// and KV heads are at most WHOLE_ITEMS, takes a workgroup per row and KV head
// (graphs of calls, 8B heads: 32 rows over 553 + 60 tokens, 12 blocks, 12.2 us
// against 14.9 in two launches, over 1,000 + 100, 19 blocks, 16.5 against 15.6; one
// row over 300 + 60 8.2 against 9.7, 553 + 60 9.8 against 9.5, 1,000 + 60, 18
// blocks, 11.9 against 10.0; 64 rows over 553 + 60, 512 workgroups, 22.4 against
// 20.5; 7B heads, 4 rows over 553 + 60, 128 workgroups, 11.0 against 12.2).
constexpr int WHOLE_ENTRIES = 12, WHOLE_ITEMS = 256;

// Splits of a prefix of nP blocks at most: of two blocks, but for longer prefixes
// of four, as parts cost the join (graphs of calls: 8B 32 rows over 1,000 tokens
// 2 blocks 15.6 us, 4 17.3; fp32 32 small rows over 1,000 13.4 and 15.9; 8B 8 rows
// over 2,000 14.5 and 15.1; one row over 6,000 14.8 and 13.4).
static int most_splits(int nP) { return nP <= 32 ? ceil_div(nP, 2) : std::max(16, ceil_div(nP, 4)); }

// Blocks of a split of the prefix for `items` tiles and KV heads.  In units of a
// block's time where two workgroups share a CU (about 2 us), an item of n blocks
// takes n + 4, 512 run at once, the work spread over them ends half the shortest
// item after its mean, and a split costs its partials' way to memory and back (the
// 4 and PART, per row and head, are fitted to the batches below).
// Splits are even, or the last one is half as long, so that other items begin
// where it ends.  Measured (graphs of calls; prompts' rows x tokens of prefix,
// blocks of a split): 8B 640 x 1,500 6 blocks 53.4 us, 8 46.7, 12 44.0, 24 55.5;
// 7B 547 x 4,000 16 blocks 96.8, 21 87.4, 24 76.0, 32 82.5; 8B 200 x 2,000 4 blocks
// 28.7, 8 28.8, 11 32.1; 13B 240 x 1,000 4 blocks 32.6, 6 27.9, 8 29.3; 64 decode
// rows, 8B x 8,000 6 blocks 50.3, 10 40.3, 16 46.2; 70B x 16,000 10 74.7, 16 77.5,
// 20 63.1, 25 69.3.
static int tile_split(int nP, int64_t items, int64_t rows_heads, int64_t own_items, int own_blocks, double &least) {
  constexpr double FIXED = 4, PART = 1.3e-4;
  int best = nP;
  least = 0;
  for (int s = 1; s <= most_splits(nP) && (s == 1 || items * s <= 512); ++s) {
    if (s > 1 && items * (s * FIXED + nP) / 512 + s * rows_heads * PART > least) break;  // more only cost more
    for (const int n : {ceil_div(nP, s), (int)(nP / (s - 0.5))}) {
      if (n > nP || n < 1 || ceil_div(nP, n) != s) continue;
      const double work = (items * (s * FIXED + nP) + own_items * (FIXED + own_blocks)) / 512;
      const double last = nP - (s - 1) * n;
      const double t = std::max(n + FIXED, work + (last + FIXED) / 2) + s * rows_heads * PART;
      if (least == 0 || t < least) {
        least = t;
        best = n;
      }
    }
  }
  return best;
}

// Row tiles and splits.
static void prefix_plan(PrefixArgs &a, bool decode, bool half, int rows, int n_heads, int n_kv_heads, int prefix_len,
                        int max_ctx, int n_seq) {
  a.G = n_heads / n_kv_heads;
  a.nP = ceil_div(std::min(prefix_len, max_ctx), KV_BLOCK);
  a.F = prefix_len / KV_BLOCK;
  int own = max_ctx > prefix_len ? ceil_div(max_ctx, KV_BLOCK) - a.F : 0;
  const int64_t packed = (int64_t)rows * a.G;
  // Shared items of 16 rows in fp32 (prefix_rows_kernel), and for up to two of
  // them (graphs of calls, packed rows: 16-row items against 128-row ones): 8B 8
  // rows over 2,000 tokens (32) 15.5 us against 16.9; 8B 16 rows (64) 18.6 and
  // 18.8; 13B 64 rows over 8,000 (64) 101 and 79; 70B 16 rows over 8,000 (128) 32 and 24.
  const bool few = !half || (decode && packed <= 32);
  const int rt = few ? 16 : 128;
  bool walk = false;
  const int tiles = a.nP ? ceil_div(packed, rt) : 0;
  if (decode && a.nP + own <= WHOLE_ENTRIES && (int64_t)rows * ceil_div(a.G, 16) * n_kv_heads <= WHOLE_ITEMS) {
    a.whole = 1;
    return;
  }
  a.tiles = few ? 0 : tiles;
  a.shared_rows = few ? tiles : 0;
  a.own_log = 2;
  if (decode) {
    const int64_t pairs = (int64_t)rows * ceil_div(a.G, 16) * n_kv_heads;
    while (a.own_log && (1 << a.own_log > own || (a.own_log == 2 && pairs > 256))) --a.own_log;
    const int want = std::max(1, 512 / (int)std::min((int64_t)rows * n_kv_heads, (int64_t)512));
    a.oblk = std::max(1, ceil_div(own, std::min(want, std::max(1, ceil_div(own, 4)))));
    // Two waves an item (four in batches of up to 256 rows and KV heads), of
    // six blocks (eight), so that long rows end with the others; at most 16 parts
    // a row while an item's 64 blocks allow, for max_ctx far above the rows'
    // contexts.  Waves x blocks: 8B heads, 64 rows of 300 over 2,000 tokens 1 x 4
    // 31.5 us, 2 x 6 29.8, 2 x 8 32.4, 4 x 8 32.7; 64 of 2,000 over 64 138, 125, 125,
    // 123; 13B, 64 of 300 over 2,000 108, 104; 70B, 48 of 300 over 4,000 33.5, 33.3,
    // 33.8, 38.0; 8B, 32 of 600 over 500, 256 pairs, -, 24.5, -, 23.9.
    a.oblk = std::min(std::max(std::min(a.oblk, 4 + 2 * a.own_log), ceil_div(own, 16)), 64);
  } else {
    // Prompts' own blocks are split where their tiles leave half the GPU idle,
    // to four blocks, past 64 tiles to 16.  New + cached tokens, whole against
    // split: 8B one prompt of 30 + 4,000 116 us and 24, 50 + 400 25 and 18, 500 + 400
    // (128 tiles) 52 and 62 in halves of 8; eight of 50 + 2,000 (104 tiles) 108 and
    // 68; one of 1,000 (256 tiles) 63 and 68; fp32 20 + 3,000 67 and 16.
    const int items = (int)std::min((int64_t)ceil_div(packed, rt) * n_kv_heads, (int64_t)512);
    const int want = std::max(1, 256 / items);
    a.oblk = std::max(std::min(own, items <= 64 ? 4 : 16), ceil_div(own, want));
    a.oblk = std::max(1, half ? a.oblk : std::min(a.oblk, 64));
  }
  if (a.nP && few) {
    // Up to 512 workgroups, and up to 24 parts while a part is at most 32 blocks:
    // 8B, graphs of calls, one row over 6,000 tokens 2 blocks 14.8 us, 4 13.4, 8
    // 15.4; one over 16,000 4 blocks 22.3, 8 19.8, 12 19.5, 20 24.6.
    const int want = std::max(1, 512 / std::max(1, tiles * n_kv_heads));
    const int most = std::min(most_splits(a.nP), std::max(24, a.nP / 32));
    a.sblk = std::min(ceil_div(a.nP, std::min(want, most)), 64);
  } else if (a.nP) {
    // own items: a row's (as above), or the sequences' tiles, half of the longest's blocks each
    const int64_t items = (int64_t)tiles * n_kv_heads, rows_heads = (int64_t)rows * n_heads;
    const int64_t of_rows = (((int64_t)rows * n_kv_heads) << a.own_log) / 4 * ceil_div(own, a.oblk);
    double split;
    a.sblk = tile_split(a.nP, items, rows_heads, decode ? of_rows : items * ceil_div(own, a.oblk),
                        decode ? std::min(own, a.oblk) >> a.own_log : (std::min(own, a.oblk) + 1) / 2, split);
    // Prompts may instead walk the prefix and their own blocks in one item, and
    // nothing is joined: in the units of tile_split, every round of 512 items takes
    // the prefix, the first (or with more, about half) the longest own context; a
    // sequence's last tile is half full.  The 3 and 1.05 are fitted: right for 30 of
    // 33 batches measured, the others within 11% (walk against splits): 70B three prompts of 2,100 over 4,096
    // tokens 686 us and 800, 8 of 100 over 1,000 50 and 69, 32 of 30 over 2,000 125 and
    // 109; 13B two of 800 over 3,000 149 and 165; 8B 16 of 120 over 2,000 135 and 115,
    // one of 2,500 over 4,000 313 and 283 (taken for 304 and 313).
    const double rounds = std::ceil((tiles + (n_seq - 1) / 2.0) * n_kv_heads / 512);
    walk = !decode && rounds * (a.nP + 3) + (rounds > 1 ? own / 2 : own) < 1.05 * split;
  }
  a.splits = a.nP ? ceil_div(a.nP, a.sblk) : 0;
  if (walk) {
    a.splits = a.tiles = 0;
    own += a.nP;
    a.oblk = own;
  }
  a.osplits = ceil_div(own, a.oblk);
  a.parts = a.splits + a.osplits;
  a.direct = a.parts == 1 && !few && (!decode || a.splits);
}

// Partials of any plan of at most these rows and contexts, so that a workspace
// for a batch's limits serves its smaller steps.  A row has at most one part per
// four blocks, or one per two up to 16.  Splits times row tiles are up to 512
// workgroups over the KV heads, so rows times splits stay under 512 x 128 /
// n_heads where splits are more than one, or, of 64 blocks an item, than nP / 64
// (prefill's own: than own / 64).  A decode row's own: at most 16, or own / 64.
size_t prefix_attention_ws_bytes(bool decode, int rows, int n_heads, int n_kv_heads, int head_dim, int prefix_len,
                                 int max_ctx) {
  const int64_t nP = ceil_div(std::min(prefix_len, max_ctx), KV_BLOCK);
  const int64_t own = max_ctx > prefix_len ? ceil_div(max_ctx, KV_BLOCK) - prefix_len / KV_BLOCK : 0;
  const int64_t r = rows, quarter = (own + 3) / 4, each = (own + 63) / 64;
  const int64_t shared = std::min(r * most_splits((int)nP),
                                  std::max(r * std::max<int64_t>(1, (nP + 63) / 64), (int64_t)65536 / n_heads));
  const int64_t of_rows = decode ? r * std::min(quarter, std::max<int64_t>(16, each))
                                 : std::min(r * quarter, std::max(r * each, (int64_t)65536 / n_heads));
  return (size_t)(shared + of_rows) * n_heads * (head_dim + 2) * sizeof(float);
}

template <typename T, int HD>
static bool launch_prefix_hd(const T *q, T *out, const PrefixBatch &b, float *ws, hipStream_t s) {
  PrefixArgs a{};
  a.b = b;
  const int Hkv = b.kv.n_kv_heads;
  constexpr bool half = sizeof(T) == 2;
  const bool decode = !b.seq_start;
  // Sequences that can have rows: a batch of fixed size may hold many more places,
  // and each that owned a tile would cost a search through all of seq_start (8B
  // heads, five prompts of 40 over 1,500 tokens: in 5 places 22 us, in 8,192 124;
  // with a tile for every place 4,221).
  const int live = std::min(b.n_seq, b.rows);
  prefix_plan(a, decode, half, b.rows, b.n_heads, Hkv, b.prefix_len, b.max_ctx, live);
  a.po = ws;
  a.pml = ws + (size_t)b.rows * b.n_heads * a.parts * HD;
  const int rto = decode || !half ? 16 : 128;
  a.otiles = decode ? b.rows * ceil_div(a.G, rto)
                    : (int)std::min((int64_t)live * ceil_div((int64_t)std::min(b.max_new, b.rows) * a.G, rto),
                                    (int64_t)b.rows * a.G / rto + live);
  a.units = decode ? ceil_div((int64_t)a.otiles << a.own_log, 4) : a.otiles;
  a.by_g = divisor(a.G);
  a.by_hkv = divisor(Hkv);
  a.by_splits = divisor(a.splits);
  a.by_osplits = divisor(a.osplits);
  a.by_units = divisor(a.units);
  a.by_shared = divisor(a.shared_rows);
  a.by_per = divisor(ceil_div(a.G, rto));
  const int64_t items = ((int64_t)(a.tiles + a.shared_rows) * a.splits + (int64_t)a.units * a.osplits) * Hkv;
  const int64_t joins = a.parts <= 16 ? ((int64_t)b.rows * b.n_heads + 3) / 4 : (int64_t)b.rows * b.n_heads;
  if (std::max(items, joins) >= 1 << 23) return false;  // a launch has fewer than 2^32 threads, 512 to a workgroup
  auto grid = [](int64_t n) { return dim3((unsigned)n); };
  if (a.whole) {
    prefix_row_kernel<T, HD><<<grid((int64_t)a.otiles * Hkv), WHOLE_WAVES<T, HD> * 64, 0, s>>>(q, out, a);
  } else if constexpr (half) {
    if (decode)
      prefix_decode_kernel<T, HD><<<grid(items), 256, 0, s>>>(q, out, a);
    else
      prefix_tile_kernel<T, HD><<<grid(items), 256, 0, s>>>(q, out, a);
  } else {
    prefix_rows_kernel<T, HD><<<grid(items), 256, 0, s>>>(q, out, a);
  }
  if (!a.direct && !a.whole) {
    if (a.parts <= 4)
      prefix_join_kernel<T, HD, 4, 1><<<grid(joins), 256, 0, s>>>(out, a);
    else if (a.parts <= 16)
      prefix_join_kernel<T, HD, 16, 1><<<grid(joins), 256, 0, s>>>(out, a);
    else
      prefix_join_kernel<T, HD, 16, 4><<<grid(joins), 256, 0, s>>>(out, a);
  }
  return true;
}

template <typename T>
bool launch_prefix_attention(const T *q, T *out, const PrefixBatch &b, float *ws, hipStream_t s) {
  return b.kv.head_dim == 128 ? launch_prefix_hd<T, 128>(q, out, b, ws, s) : launch_prefix_hd<T, 64>(q, out, b, ws, s);
}

#define INST(T) template bool launch_prefix_attention<T>(const T *, T *, const PrefixBatch &, float *, hipStream_t);
INST(float)
INST(bf16_t)
INST(f16_t)
#undef INST

}  // namespace lp
