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

#include "device.hpp"

namespace lp {

struct PrefixArgs {
  PrefixBatch b;
  int G;                      // query heads of a KV head
  int nP, F;                  // prefix entries, first own block
  int tiles, splits, sblk;    // shared items: row tiles, splits of the prefix, entries of a split
  int otiles, osplits, oblk;  // own items: row tiles of a sequence, splits of its entries, entries of a split
  int parts;                  // splits + osplits
  float *po, *pml;            // partial o [rows][n_heads][parts][hd], (m, l) [rows][n_heads][parts][2]
};

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
    idx /= a.osplits;
    j = idx / a.otiles;
    r0 = idx % a.otiles * 64;
    int start, n;
    seq_rows(a.b, j, start, n);
    if (r0 >= n * a.G) return;
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
  const float scale = rsqrtf((float)HD);
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
      sc *= scale;
      const float mn = fmaxf(mx, sc);
      const float corr = mx == mn ? 1.f : __expf(mx - mn);
      const float pe = mn == -INFINITY && sc == sc ? 0.f : __expf(sc - mn);
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

// Joins the parts of a (token, head): a wave each, its lanes over the dims.
template <typename T, int HD>
__global__ __launch_bounds__(256) void prefix_join_kernel(T *__restrict__ out, PrefixArgs a) {
  constexpr int DPL = HD / 64;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int64_t t = row / a.b.n_heads;
  if (t >= a.b.rows) return;
  if (a.b.seq_start && (t < a.b.seq_start[0] || t >= a.b.seq_start[a.b.n_seq])) return;
  const float *ml = a.pml + row * a.parts * 2, *po = a.po + row * a.parts * HD + lane * DPL;
  float M = -INFINITY, L = 0.f, o[DPL];
#pragma unroll
  for (int d = 0; d < DPL; ++d) o[d] = 0.f;
  for (int p = 0; p < a.parts; ++p) {
    const float m = ml[2 * p], l = ml[2 * p + 1];
    if (m == -INFINITY && l == 0.f) continue;  // no key in this part
    const float mn = fmaxf(M, m);
    const float f0 = M == mn ? 1.f : __expf(M - mn), f1 = m == mn ? 1.f : __expf(m - mn);
    L = L * f0 + l * f1;
#pragma unroll
    for (int d = 0; d < DPL; ++d) o[d] = o[d] * f0 + po[(int64_t)p * HD + d] * f1;
    M = mn;
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
#pragma unroll
  for (int d = 0; d < DPL; ++d) out[row * HD + lane * DPL + d] = Act<T>::st(o[d] * inv);
}

static int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Splits of the prefix and of the own entries: about 512 workgroups, four
// blocks each at least.
static void prefix_plan(PrefixArgs &a, bool decode, int rows, int n_heads, int n_kv_heads, int prefix_len, int max_ctx) {
  a.G = n_heads / n_kv_heads;
  a.nP = ceil_div(prefix_len < max_ctx ? prefix_len : max_ctx, KV_BLOCK);
  a.F = prefix_len / KV_BLOCK;
  const int own = max_ctx > prefix_len ? ceil_div(max_ctx, KV_BLOCK) - a.F : 0;
  a.tiles = a.nP ? ceil_div((int64_t)rows * a.G, 64) : 0;
  a.splits = a.sblk = 0;
  if (a.nP) {
    const int want = std::max(1, 512 / std::max(1, a.tiles * n_kv_heads));
    a.sblk = ceil_div(a.nP, std::min(want, ceil_div(a.nP, 4)));
    a.splits = ceil_div(a.nP, a.sblk);
  }
  a.oblk = std::max(1, decode ? std::min(own, 4) : own);
  a.osplits = ceil_div(own, a.oblk);
  a.parts = a.splits + a.osplits;
}

size_t prefix_attention_ws_bytes(bool decode, int rows, int n_heads, int n_kv_heads, int head_dim, int prefix_len,
                                 int max_ctx) {
  PrefixArgs a{};
  prefix_plan(a, decode, rows, n_heads, n_kv_heads, prefix_len, max_ctx);
  return (size_t)rows * n_heads * a.parts * (head_dim + 2) * sizeof(float);
}

template <typename T, int HD>
static void launch_prefix_hd(const T *q, T *out, const PrefixBatch &b, float *ws, hipStream_t s) {
  PrefixArgs a{};
  a.b = b;
  prefix_plan(a, !b.seq_start, b.rows, b.n_heads, b.kv.n_kv_heads, b.prefix_len, b.max_ctx);
  a.otiles = ceil_div((int64_t)std::min(b.max_new, b.rows) * a.G, 64);
  a.po = ws;
  a.pml = ws + (size_t)b.rows * b.n_heads * a.parts * HD;
  const int64_t items = (int64_t)a.tiles * a.splits + (int64_t)b.n_seq * a.otiles * a.osplits;
  prefix_attn_kernel<T, HD><<<dim3((unsigned)(items * b.kv.n_kv_heads)), 256, 0, s>>>(q, a);
  prefix_join_kernel<T, HD><<<dim3((unsigned)ceil_div((int64_t)b.rows * b.n_heads, 4)), 256, 0, s>>>(out, a);
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
