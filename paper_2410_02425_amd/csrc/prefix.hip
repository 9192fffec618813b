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
#include <type_traits>

#include "device.hpp"

namespace lp {

struct PrefixArgs {
  PrefixBatch b;
  int G;                      // query heads of a KV head
  int nP, F;                  // prefix entries, first own block
  int tiles, splits, sblk;    // shared items: row tiles, splits of the prefix, entries of a split
  int otiles, osplits, oblk;  // own items: row tiles, splits of the own entries, entries of a split
  int parts;                  // splits + osplits
  int direct;                 // one part, written to out by the tile kernel itself
  float *po, *pml;            // partial o [rows][n_heads][parts][hd], (m, l) [rows][n_heads][parts][2]
};
// A part's m is the largest score before the scale 1/sqrt(hd), its weights are
// 2^((score - m) c2).
template <int HD>
constexpr float SCORE_C2 = (HD == 64 ? 0.125f : 0.08838834764831845f) * 1.44269504088896341f;

struct PrefixRow {
  int token, head, ctx;  // ctx: keys the row sees, 0 for a row that does not exist or sees none
  bool live;             // the row exists: its result (or partial) is written
};

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

// Packed row r of all tokens (j < 0), or of sequence j alone.
__device__ __forceinline__ PrefixRow packed_row(const PrefixArgs &a, int j, int r, int g) {
  PrefixRow w{0, g * a.G + r % a.G, 0, false};
  int t = r / a.G, start, n;
  if (j < 0) {
    if (t >= a.b.rows) return w;
    if (!a.b.seq_start) {
      j = t;
    } else {  // the last sequence that starts at or before the token
      int lo = 0, hi = a.b.n_seq - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.b.seq_start[mid] <= t) lo = mid;
        else hi = mid - 1;
      }
      j = lo;
    }
    seq_rows(a.b, j, start, n);
    t -= start;
  } else {
    seq_rows(a.b, j, start, n);
  }
  if (t < 0 || t >= n || t >= a.b.max_new) return w;
  w.token = start + t;
  w.ctx = row_ctx(a.b, j, t);
  w.live = true;
  return w;
}

// Own tile u of RT packed rows: sequence by sequence, each with as many tiles as
// its rows need.  Each wave finds it on its own: an inclusive sum over 64
// sequences at a time, the first whose sum exceeds u.  False past the last.
template <int RT>
__device__ __forceinline__ bool own_tile(const PrefixArgs &a, int u, int &j, int &r0) {
  const int lane = threadIdx.x & 63;
  if (!a.b.seq_start) {  // one row a sequence
    const int per = (a.G + RT - 1) / RT;
    j = u / per;
    r0 = u % per * RT;
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

// An entry's block id (-1: none), first position and valid places [lo, hi).
struct PrefixEntry {
  int id, base, lo, hi;
};
__device__ __forceinline__ PrefixEntry prefix_entry(const PrefixArgs &a, int slot, int e) {
  PrefixEntry x;
  if (e < a.nP) {
    x.base = e * KV_BLOCK;
    x.lo = 0;
    x.hi = min(KV_BLOCK, a.b.prefix_len - x.base);
    x.id = a.b.prefix_blocks[e];
  } else {
    const int blk = a.F + e - a.nP;
    x.base = blk * KV_BLOCK;
    x.lo = max(0, a.b.prefix_len - x.base);
    x.hi = KV_BLOCK;
    x.id = slot >= 0 && slot < a.b.n_slots && blk < a.b.kv.max_blocks
               ? a.b.kv.block_table[(int64_t)slot * a.b.kv.max_blocks + blk]
               : -1;
  }
  if (x.id < 0 || x.id >= a.b.kv.n_blocks) x.id = -1;
  return x;
}

// One workgroup per (64 packed rows, KV head, entry range); four threads hold a
// row's dims, the keys go through LDS block by block, with a running maximum.
template <typename T, int HD>
__global__ __launch_bounds__(256) void prefix_attn_kernel(const T *__restrict__ q, PrefixArgs a) {
  constexpr int Q4 = HD / 4;  // dims per thread
  __shared__ T ks[64][HD + 2];
  __shared__ T vs[64][HD + 2];
  const int Hkv = a.b.kv.n_kv_heads, Hq = a.b.n_heads;
  int idx = blockIdx.x, j = -1, r0, e0, e1, part;
  const int g = idx % Hkv;
  idx /= Hkv;
  if (idx < a.tiles * a.splits) {
    part = idx % a.splits;
    r0 = idx / a.splits * 64;
    e0 = part * a.sblk;
    e1 = min(a.nP, e0 + a.sblk);
  } else {
    idx -= a.tiles * a.splits;
    const int s = idx % a.osplits;
    if (!own_tile<64>(a, idx / a.osplits, j, r0)) return;
    part = a.splits + s;
    e0 = a.nP + s * a.oblk;
    e1 = e0 + a.oblk;
  }
  const int slot = j < 0 ? -1 : a.b.seq_slot[j];
  const int qi = threadIdx.x >> 2, qq = threadIdx.x & 3;
  const PrefixRow w = packed_row(a, j, r0 + qi, g);
  __shared__ int top;  // the largest context of the tile
  if (threadIdx.x == 0) top = 0;
  __syncthreads();
  atomicMax(&top, w.ctx);
  __syncthreads();
  const int most = top;
  float qv[Q4], o[Q4];
  const T *qr = q + ((int64_t)w.token * Hq + w.head) * HD + qq * Q4;
#pragma unroll
  for (int t = 0; t < Q4; ++t) {
    qv[t] = w.live ? Act<T>::ld(qr[t]) : 0.f;
    o[t] = 0.f;
  }
  float mx = -INFINITY, l = 0.f;
  constexpr float c2 = SCORE_C2<HD>;
  for (int e = e0; e < e1; ++e) {
    const PrefixEntry x = prefix_entry(a, slot, e);
    if (x.base + x.lo >= most) break;
    if (x.id < 0) continue;
    const int64_t base = ((int64_t)x.id * Hkv + g) * KV_BLOCK * HD;
    const T *kbp = (const T *)a.b.kv.k + base;
    const T *vbp = (const T *)a.b.kv.v + base;
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * HD; i += 256) {
      ks[i / HD][i % HD] = kbp[i];
      vs[i % 64][i / 64] = vbp[i];
    }
    __syncthreads();
    const int end = min(x.hi, most - x.base);
    for (int p = x.lo; p < end; ++p) {
      float sc = 0.f;
#pragma unroll
      for (int t = 0; t < Q4; ++t) sc += qv[t] * Act<T>::ld(ks[p][qq * Q4 + t]);
      sc += __shfl_xor(sc, 1, 64);
      sc += __shfl_xor(sc, 2, 64);
      if (x.base + p >= w.ctx) continue;  // uniform across the 4 threads of a row
      const float mn = fmaxf(mx, sc);
      const float corr = mx == mn ? 1.f : __builtin_amdgcn_exp2f((mx - mn) * c2);
      const float pe = mn == -INFINITY && sc == sc ? 0.f : __builtin_amdgcn_exp2f((sc - mn) * c2);
      l = l * corr + pe;
#pragma unroll
      for (int t = 0; t < Q4; ++t) o[t] = o[t] * corr + pe * Act<T>::ld(vs[p][qq * Q4 + t]);
      mx = mn;
    }
  }
  if (w.live) {
    const int64_t rec = ((int64_t)w.token * Hq + w.head) * a.parts + part;
    float *dst = a.po + rec * HD + qq * Q4;
#pragma unroll
    for (int t = 0; t < Q4; ++t) dst[t] = o[t];
    if (qq == 0) *(float2 *)(a.pml + rec * 2) = make_float2(mx, l);
  }
}

// ------------------------------------------------------------------ 16-bit types

// Many rows over a range of entries, on 32x32x16 MFMAs: a workgroup owns 32 QW
// packed rows, 32 to a wave, and walks its entries' blocks, which are copied
// into LDS for all its waves (two stages: the next block lands while the
// current one is used) in the cache's own order, with the 16-byte pieces of a
// row XOR-swizzled against bank conflicts.
//   S^T = K Q^T: a lane holds one row's scores, so the softmax's maximum and sum
//   run in its registers and meet the wave's other half once a block.  The K row
//   of MFMA row i is i with bits 2 and 3 swapped: then the eight weights a lane
//   holds of each 16 keys are consecutive keys, the B operand of O^T += V^T P^T,
//   and P never leaves the registers.
//   The running maximum moves in every block that raises it for a row of the
//   wave, so the largest weight is exactly 1 before it is rounded to 16 bits.
// V at places that no row of the tile sees is cleared in LDS (stale entries may
// hold anything, and 0 * NaN is not 0).  Places that only some of its rows see
// are not: their weight is 0 for the others, which is enough unless V is
// infinite or NaN there.  A tile whose result is not finite is therefore
// computed again with every row's own V (`careful`), once.
template <typename T, int HD, int QW>
__global__ __launch_bounds__(QW * 64) __attribute__((amdgpu_waves_per_eu(2))) void prefix_tile_kernel(
    const T *__restrict__ q, T *__restrict__ out, PrefixArgs a) {
  typedef typename Mfma<T>::v8 v8;
  constexpr int RT = QW * 32;
  constexpr int KS = HD / 16;         // contraction steps of S over head_dim
  constexpr int NT = HD / 32;         // 32-dim tiles of O^T
  constexpr int CK = HD / 8;          // 16-byte pieces of a K row
  constexpr int PB = 64 * HD * 2;     // bytes of a K (or V) block
  constexpr int STAGE = 2 * PB;
  constexpr int ND = PB / 1024 / QW;  // 1 KB copies per wave and block, K and V each
  constexpr float c2 = SCORE_C2<HD>;
  __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];
  const int Hkv = a.b.kv.n_kv_heads, Hq = a.b.n_heads, P = a.b.prefix_len;
  // KV head fastest: with 8 of them each XCD's L2 holds one head's blocks
  int idx = blockIdx.x, j = -1, r0, e0, e1, part, most = INT_MAX, slot = -1;
  const int g = idx % Hkv;
  idx /= Hkv;
  if (idx < a.tiles * a.splits) {
    part = idx % a.splits;
    r0 = idx / a.splits * RT;
    e0 = part * a.sblk;
    e1 = min(a.nP, e0 + a.sblk);
  } else {
    idx -= a.tiles * a.splits;
    const int s = idx % a.osplits;
    if (!own_tile<RT>(a, idx / a.osplits, j, r0)) return;
    part = a.splits + s;
    slot = a.b.seq_slot[j];
    int start, n;
    seq_rows(a.b, j, start, n);
    most = row_ctx(a.b, j, min((r0 + RT - 1) / a.G, n - 1));  // the last row sees most
    e0 = (a.splits ? a.nP : 0) + s * a.oblk;
    e1 = min(e0 + a.oblk, most > P ? a.nP + (most + KV_BLOCK - 1) / KV_BLOCK - a.F : (most + KV_BLOCK - 1) / KV_BLOCK);
  }
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l32 = lane & 31, hh = lane >> 5;
  const PrefixRow w = packed_row(a, j, r0 + wave * 32 + l32, g);
  // rows that do not exist see everything (no mask on their account)
  const int ctx = w.live ? w.ctx : INT_MAX;
  const int ctx_lo = (int)wave_min_u32((uint32_t)ctx);
  const int ctx_hi = w.live ? w.ctx : 0;
  const int ctx_top = (int)~wave_min_u32(~(uint32_t)ctx_hi);

  v8 qb[KS];  // Q^T as the B operand: this lane's row, dims 16 k + 8 hh ..
  {
    const T *qr = q + ((int64_t)w.token * Hq + w.head) * HD + hh * 8;
#pragma unroll
    for (int k = 0; k < KS; ++k) qb[k] = load8<T>(qr + k * 16);
  }
  // Byte offsets of the entries' blocks (head included), -1 for none: lane i
  // holds that of entry win + i, the wave reads them back with readlane.
  int win = e0, off_lo, off_hi;
  auto window = [&]() __attribute__((always_inline)) {
    int64_t off = -1;
    if (win + lane < e1) {
      const int id = prefix_entry(a, slot, win + lane).id;
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
    const int n = wave * ND + c, kr = n * KR + lane / CK, vr = n * 8 + (lane >> 3);
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
  const int krow = (l32 & 0x13) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);
  const int kfb = krow * HD * 2, kfx = (hh ^ swz(krow)) << 4;
  const int vfb = l32 * KV_BLOCK * 2, vfx = (hh ^ ((l32 >> 1) & 7)) << 4;

  floatx16_t o[NT];
  float mref, lsum;
  // the entries' walk; returns whether a block was seen whole by some rows of
  // the wave only
  auto walk = [&](auto careful_) __attribute__((always_inline)) {
    constexpr bool careful = decltype(careful_)::value;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
    // running maximum (raw scores), its base-2 value, this half's share of the sum
    float mc = 0.f;
    mref = -INFINITY;
    lsum = 0.f;
    bool large = false;   // wave-uniform: a row's |mc| is past PFA_LARGE
    bool masked = false;  // wave-uniform: a block that only some rows see whole
    if (e0 < e1) {
      win = e0;
      window();
      issue(e0);
    }
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
      if (e + 1 < e1) issue(e + 1);
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
      if (partly) {
        masked = true;
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
        large = __any(fabsf(mc) > PFA_LARGE);
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
          pb[t * 2 + u] = pack8<T>(p);
        }
      if (careful && partly) {
        // row by row, each with V of its own keys alone
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll 1
          for (int i = 0; i < 32; ++i) {
            const int lim = __builtin_amdgcn_readlane(end, i);
            floatx16_t acc = o[t];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              u32x4_tt f = *(const u32x4_tt *)(vs + vfb + t * 32 * KV_BLOCK * 2 + (vfx ^ (k << 5)));
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const int key = k * 16 + hh * 8 + 2 * x;
                f[x] &= (key < lim ? 0xFFFFu : 0u) | (key + 1 < lim ? 0xFFFF0000u : 0u);
              }
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
  const bool masked = walk(std::false_type());
  float z = 0.f;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) z = fmaf(o[t][r], 0.f, z);
  if (__syncthreads_or(masked && w.live && !(z == 0.f))) walk(std::true_type());
  // o[t][r]: dim 32 t + 8 (r / 4) + 4 hh + r % 4 of this lane's row
  const float sum = half_swap_sum(lsum);
  const int64_t row = (int64_t)w.token * Hq + w.head;
  if (a.direct) {
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
    for (int t = 0; t < NT; ++t) store_o32(out + row * HD + t * 32, o[t], inv, hh, w.live);
  } else if (w.live) {
    const int64_t rec = row * a.parts + part;
    float *dst = a.po + rec * HD + 4 * hh;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *(float4 *)(dst + t * 32 + 2 * r) = make_float4(o[t][r], o[t][r + 1], o[t][r + 2], o[t][r + 3]);
    if (hh == 0) *(float2 *)(a.pml + rec * 2) = make_float2(mref, sum);
  }
}

// Few rows over four entries, on 16x16x32 MFMAs: up to 16 packed rows of a KV
// head, a wave per entry, which requests its K fragments at once from the cache
// and then its V fragments.  P goes through LDS into the A operand's layout;
// the waves' (m, l, o) meet in LDS.  Own items: the query heads of one row.
// Shared items (a batch of few rows): packed rows.
template <typename T, int HD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3))) void prefix_chunk_kernel(const T *__restrict__ q, PrefixArgs a) {
  typedef typename Mfma<T>::v8 v8;
  constexpr int KS = HD / 32, NT = HD / 16;
  constexpr float c2 = SCORE_C2<HD>;
  __shared__ T pls[4][16][64 + 8];
  __shared__ float wm[4][16], wl[4][16];
  __shared__ float wo[4][16][HD];
  const int Hkv = a.b.kv.n_kv_heads, Hq = a.b.n_heads, P = a.b.prefix_len;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r16 = lane & 15, quad = lane >> 4, kq = quad * 8;
  int idx = blockIdx.x, j = -1, r0, e, part, slot = -1;
  const int g = idx % Hkv;
  idx /= Hkv;
  if (idx < a.tiles * a.splits) {
    part = idx % a.splits;
    r0 = idx / a.splits * 16;
    e = part * a.sblk + wave;
  } else {
    idx -= a.tiles * a.splits;
    const int s = idx / a.otiles;  // all rows' first chunks, then their second ones: the grid ends with what few have
    own_tile<16>(a, idx % a.otiles, j, r0);
    part = a.splits + s;
    slot = a.b.seq_slot[j];
    e = a.nP + s * a.oblk + wave;
    const int ctx = row_ctx(a.b, j, 0);
    if (ctx <= P || (a.F + s * a.oblk) * KV_BLOCK >= ctx) return;
  }
  const PrefixRow w = packed_row(a, j, r0 + r16, g);
  const bool own = j >= 0;
  const bool live = w.live && (!own || r0 + r16 < a.G);
  const int ctx_top = (int)~wave_min_u32(~(uint32_t)(live ? w.ctx : 0));
  const int base = own ? (a.F + e - a.nP) * KV_BLOCK : e * KV_BLOCK;
  const int lo = own ? max(0, P - base) : 0;
  const int hi = min(KV_BLOCK, min(own ? INT_MAX : P, ctx_top) - base);
  const PrefixEntry x = lo < hi ? prefix_entry(a, slot, e) : PrefixEntry{-1, 0, 0, 0};
  const bool there = x.id >= 0;
  const int64_t off = there ? ((int64_t)x.id * Hkv + g) * KV_BLOCK * HD : 0;
  v8 qa[KS], kf[4][KS], vf[NT][2];
  const T *qrow = q + ((int64_t)w.token * Hq + w.head) * HD;
#pragma unroll
  for (int k = 0; k < KS; ++k) qa[k] = live ? load8<T>(qrow + k * 32 + kq) : zero8<T>();
  floatx4_t sacc[4], oacc[NT];
  float mx[4], sm[4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) oacc[nt] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) mx[i] = -INFINITY, sm[i] = 0.f;
  if (there) {
    const T *kb = (const T *)a.b.kv.k + off, *vb = (const T *)a.b.kv.v + off;
#pragma unroll
    for (int nt = 0; nt < 4; ++nt)
#pragma unroll
      for (int k = 0; k < KS; ++k) kf[nt][k] = load8<T>(kb + (nt * 16 + r16) * HD + k * 32 + kq);
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
      sacc[nt] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) sacc[nt] = Mfma<T>::m16(qa[k], kf[nt][k], sacc[nt]);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int k = 0; k < 2; ++k) vf[nt][k] = load8<T>(vb + (nt * 16 + r16) * KV_BLOCK + k * 32 + kq);
    // sacc[nt][i]: row 4 quad + i, key nt * 16 + r16
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int end = min(hi, __shfl(live ? w.ctx : 0, 4 * quad + i, 64) - base);
      float v = -INFINITY;
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        const int key = nt * 16 + r16;
        sacc[nt][i] = key >= lo && key < end ? sacc[nt][i] : -INFINITY;
        v = fmaxf(v, sacc[nt][i]);
      }
      v = row16_max(v);
      mx[i] = v;
      const float m0 = v == -INFINITY ? 0.f : v;
      float t = 0.f;
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        const float p = __builtin_amdgcn_exp2f((sacc[nt][i] - m0) * c2);
        t += p;
        pls[wave][4 * quad + i][nt * 16 + r16] = Act<T>::st(p);
      }
      sm[i] = row16_sum(t);
    }
  }
  __syncthreads();
  if (there) {
    v8 pa[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) pa[k] = load8<T>(&pls[wave][r16][k * 32 + kq]);
    // keys [from, to) of the V fragments, others 0 (stale entries hold anything)
    auto keep = [&](v8 f, int k, int from, int to) __attribute__((always_inline)) {
      u32x4_tt m = __builtin_bit_cast(u32x4_tt, f);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int key = k * 32 + kq + 2 * y;
        m[y] &= (key >= from && key < to ? 0xFFFFu : 0u) | (key + 1 >= from && key + 1 < to ? 0xFFFF0000u : 0u);
      }
      return __builtin_bit_cast(v8, m);
    };
    if (lo > 0 || hi < KV_BLOCK) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k) vf[nt][k] = keep(vf[nt][k], k, lo, hi);
    }
    float z = 0.f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int k = 0; k < 2; ++k) oacc[nt] = Mfma<T>::m16(pa[k], vf[nt][k], oacc[nt]);
#pragma unroll
      for (int i = 0; i < 4; ++i) z = fmaf(oacc[nt][i], 0.f, z);
    }
    if (!own && __any(!(z == 0.f))) {
      // V is not finite at a key that perhaps not every row sees: row by row
#pragma unroll 1
      for (int rr = 0; rr < 16; ++rr) {
        const int end = min(hi, __builtin_amdgcn_readlane(live ? w.ctx : 0, rr) - base);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          floatx4_t acc = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < 2; ++k) acc = Mfma<T>::m16(pa[k], keep(vf[nt][k], k, 0, end), acc);
#pragma unroll
          for (int i = 0; i < 4; ++i) oacc[nt][i] = 4 * quad + i == rr ? acc[i] : oacc[nt][i];
        }
      }
    }
  }
  if (r16 == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      wm[wave][4 * quad + i] = mx[i];
      wl[wave][4 * quad + i] = sm[i];
    }
  }
  const int nrows = own ? min(16, a.G - r0) : 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (4 * quad + i < nrows) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) wo[wave][4 * quad + i][nt * 16 + r16] = oacc[nt][i];
    }
  }
  __syncthreads();
  // a wave a row: its lanes over the dims
  for (int r = wave; r < nrows; r += 4) {
    const int token = __builtin_amdgcn_readlane(w.token, r), h = __builtin_amdgcn_readlane(w.head, r);
    if (!__builtin_amdgcn_readlane((int)live, r)) continue;
    float M = -INFINITY, f[4], L = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) M = fmaxf(M, wm[k][r]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f[k] = wm[k][r] == M ? 1.f : __builtin_amdgcn_exp2f((wm[k][r] - M) * c2);
      L += f[k] * wl[k][r];
    }
    const int64_t rec = ((int64_t)token * Hq + h) * a.parts + part;
    for (int d = lane; d < HD; d += 64)
      a.po[rec * HD + d] = (f[0] * wo[0][r][d] + f[1] * wo[1][r][d]) + (f[2] * wo[2][r][d] + f[3] * wo[3][r][d]);
    if (lane == 0) *(float2 *)(a.pml + rec * 2) = make_float2(M, L);
  }
}

// Joins the parts of a (token, head), a wave each: its lanes hold the parts'
// weights first, then the dims.
template <typename T, int HD>
__global__ __launch_bounds__(256) void prefix_join_kernel(T *__restrict__ out, PrefixArgs a) {
  constexpr int DPL = HD / 64, U = 4;
  constexpr float c2 = SCORE_C2<HD>;
  const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
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
    const float f = x.x == mn ? 1.f : __builtin_amdgcn_exp2f((x.x - mn) * c2);
    L = L * f0 + wave_sum(f * x.y);
    M = mn;
#pragma unroll
    for (int d = 0; d < DPL; ++d) o[d] *= f0;
    for (int p = 0; p < n; p += U) {
      float v[U][DPL];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int d = 0; d < DPL; ++d) v[u][d] = po[(int64_t)(p0 + min(p + u, n - 1)) * HD + d];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p + u >= n) break;
        const float fu = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), p + u));
#pragma unroll
        for (int d = 0; d < DPL; ++d) o[d] += fu * v[u][d];
      }
    }
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
#pragma unroll
  for (int d = 0; d < DPL; ++d) out[row * HD + lane * DPL + d] = Act<T>::st(o[d] * inv);
}

// ------------------------------------------------------------------ plan

static int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

enum PrefixKernel : int { PK_SIMPLE, PK_CHUNK, PK_TILE };

// The shared items' row tile and kernel, the splits of both parts.  16-bit
// types: batches of at most 16 packed rows take the chunk kernel (the rows of a
// KV head are one tile of it), larger ones the tile kernel; a decode batch's own
// parts take the chunk kernel.
struct PrefixPlan {
  int shared, own;  // kernels
  int rt;           // rows of a shared tile
};
static PrefixPlan prefix_plan(PrefixArgs &a, bool decode, bool half, int rows, int n_heads, int n_kv_heads,
                              int prefix_len, int max_ctx) {
  a.G = n_heads / n_kv_heads;
  a.nP = ceil_div(std::min(prefix_len, max_ctx), KV_BLOCK);
  a.F = prefix_len / KV_BLOCK;
  int own = max_ctx > prefix_len ? ceil_div(max_ctx, KV_BLOCK) - a.F : 0;
  const int64_t packed = (int64_t)rows * a.G;
  PrefixPlan p{PK_SIMPLE, PK_SIMPLE, 64};
  if (half) {
    p.shared = decode && packed <= 16 ? PK_CHUNK : PK_TILE;
    p.own = decode ? PK_CHUNK : PK_TILE;
    p.rt = p.shared == PK_CHUNK ? 16 : !decode || packed > 64 ? 128 : packed > 32 ? 64 : 32;
  }
  a.tiles = a.nP ? ceil_div(packed, p.rt) : 0;
  a.splits = a.sblk = 0;
  if (a.nP) {
    if (p.shared == PK_CHUNK) {
      a.sblk = 4;
    } else {
      const int want = std::max(1, 512 / std::max(1, a.tiles * n_kv_heads));
      a.sblk = ceil_div(a.nP, std::min(want, ceil_div(a.nP, 4)));
    }
    a.splits = ceil_div(a.nP, a.sblk);
  }
  a.oblk = std::max(1, decode ? std::min(own, 4) : own);
  if (p.own == PK_TILE && a.tiles * n_kv_heads >= 512) {
    a.splits = 0;
    a.tiles = 0;
    own += a.nP;
    a.oblk = own;
  }
  a.osplits = ceil_div(own, a.oblk);
  a.parts = a.splits + a.osplits;
  a.direct = a.parts == 1 && (a.splits ? p.shared : p.own) == PK_TILE;
  return p;
}

size_t prefix_attention_ws_bytes(bool decode, int rows, int n_heads, int n_kv_heads, int head_dim, int prefix_len,
                                 int max_ctx) {
  size_t most = 0;
  for (bool half : {false, true}) {
    PrefixArgs a{};
    prefix_plan(a, decode, half, rows, n_heads, n_kv_heads, prefix_len, max_ctx);
    most = std::max(most, (size_t)rows * n_heads * a.parts * (head_dim + 2) * sizeof(float));
  }
  return most;
}

template <typename T, int HD>
static void launch_prefix_hd(const T *q, T *out, const PrefixBatch &b, float *ws, hipStream_t s) {
  PrefixArgs a{};
  a.b = b;
  const int Hkv = b.kv.n_kv_heads;
  const bool decode = !b.seq_start;
  const PrefixPlan p =
      prefix_plan(a, decode, sizeof(T) == 2, b.rows, b.n_heads, Hkv, b.prefix_len, b.max_ctx);
  a.po = ws;
  a.pml = ws + (size_t)b.rows * b.n_heads * a.parts * HD;
  const int rto = p.own == PK_CHUNK ? 16 : p.own == PK_TILE ? 128 : 64;
  a.otiles = decode ? b.rows * ceil_div(a.G, rto)
                    : (int)std::min((int64_t)b.n_seq * ceil_div((int64_t)std::min(b.max_new, b.rows) * a.G, rto),
                                    (int64_t)b.rows * a.G / rto + b.n_seq);
  const int64_t shared = (int64_t)a.tiles * a.splits * Hkv, own = (int64_t)a.otiles * a.osplits * Hkv;
  auto grid = [](int64_t n) { return dim3((unsigned)n); };
  if constexpr (sizeof(T) == 2) {
    const auto tile = [&](int64_t n, const PrefixArgs &x) {
      if (p.rt == 32)
        prefix_tile_kernel<T, HD, 1><<<grid(n), 64, 0, s>>>(q, out, x);
      else if (p.rt == 64)
        prefix_tile_kernel<T, HD, 2><<<grid(n), 128, 0, s>>>(q, out, x);
      else
        prefix_tile_kernel<T, HD, 4><<<grid(n), 256, 0, s>>>(q, out, x);
    };
    if (p.shared == p.own) {
      if (p.own == PK_TILE)
        tile(shared + own, a);
      else
        prefix_chunk_kernel<T, HD><<<grid(shared + own), 256, 0, s>>>(q, a);
    } else {
      if (shared) tile(shared, a);
      PrefixArgs x = a;
      x.tiles = 0;  // own items alone
      if (own) prefix_chunk_kernel<T, HD><<<grid(own), 256, 0, s>>>(q, x);
    }
  } else {
    prefix_attn_kernel<T, HD><<<grid(shared + own), 256, 0, s>>>(q, a);
  }
  if (!a.direct)
    prefix_join_kernel<T, HD><<<grid(ceil_div((int64_t)b.rows * b.n_heads, 4)), 256, 0, s>>>(out, a);
}

template <typename T>
void launch_prefix_attention(const T *q, T *out, const PrefixBatch &b, float *ws, hipStream_t s) {
  if (b.kv.head_dim == 128)
    launch_prefix_hd<T, 128>(q, out, b, ws, s);
  else
    launch_prefix_hd<T, 64>(q, out, b, ws, s);
}

#define INST(T) template void launch_prefix_attention<T>(const T *, T *, const PrefixBatch &, float *, hipStream_t);
INST(float)
INST(bf16_t)
INST(f16_t)
#undef INST

}  // namespace lp
