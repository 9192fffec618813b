// What comes before attention over a paged cache in a step that the caller
// plans: block tables and cache entries from lengths, and the QKV projection's
// K and V into those entries.
#include <algorithm>
#include <type_traits>

#include "device.hpp"

namespace lp {

// ------------------------------------------------------------------ block tables

// Of one sequence: new rows, entries held before the step, entries needed.
struct SeqNeed {
  int64_t rows;
  int have, need;
};
__device__ __forceinline__ int blocks_of(int n) { return n / KV_BLOCK + (n % KV_BLOCK != 0); }
__device__ __forceinline__ SeqNeed seq_need(const TableStep &t, int j) {
  const int c = max(t.cached[j], 0), n = max(t.lengths[j], 0);
  SeqNeed s;
  s.rows = n > c ? n - c : 0;
  s.have = c > t.prefix_len ? blocks_of(c) : t.prefix_len / KV_BLOCK;
  // a length inside the prefix needs none of its own, also where the prefix ends inside a block
  s.need = min(n > t.prefix_len ? blocks_of(n) : min(blocks_of(n), t.prefix_len / KV_BLOCK), t.max_blocks);
  return s;
}

__device__ __forceinline__ int free_block(const TableStep &t, int64_t i) {
  return i >= 0 && i < t.n_free ? t.free_blocks[i] : -1;
}
__device__ __forceinline__ int saturated(int64_t v) { return (int)min(v, (int64_t)INT32_MAX); }

// A step is a scan over the sequences (rows and blocks) and independent stores:
// nothing but latency at any size that a service has (256 requests, 65,000 rows:
// 1.1 MB, 5.2 us; 64 requests of one row 3.8 us).  So one launch: every workgroup
// scans all sequences for itself, keeps what it needs of each in LDS, and takes
// its share of the table rows (a wave a sequence) and of the packed rows (a
// thread each, its sequence by bisection).
// With WHOLE = false the sums come from a launch of their own (table_scan_kernel)
// and the sequences are read again: more sequences than LDS holds, or a free_head
// inside free_start, which workgroups that start late would find updated.
constexpr int TABLE_SEQS = 1024, TABLE_THREADS = 1024;

struct TableSeq {
  int start[TABLE_SEQS], taken[TABLE_SEQS], cached[TABLE_SEQS], have[TABLE_SEQS], slot[TABLE_SEQS];
};

// Exclusive sums over one value per thread of the workgroup, and the totals.
__device__ __forceinline__ void table_scan(uint64_t rows, uint64_t take, uint64_t &r0, uint64_t &b0, uint64_t &rt,
                                           uint64_t &bt) {
  __shared__ uint64_t wsum[2][TABLE_THREADS / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t r = wave_scan(rows), b = wave_scan(take);
  __syncthreads();  // the sums before are read
  if (lane == 63) {
    wsum[0][wave] = r;
    wsum[1][wave] = b;
  }
  __syncthreads();
  const uint64_t vr = row16_scan(wsum[0][lane & 15]), vb = row16_scan(wsum[1][lane & 15]);
  rt = readlane_u64(vr, 15);
  bt = readlane_u64(vb, 15);
  const int w = __builtin_amdgcn_readfirstlane(wave);
  r0 = (w ? readlane_u64(vr, w - 1) : 0) + r - rows;
  b0 = (w ? readlane_u64(vb, w - 1) : 0) + b - take;
}

__global__ __launch_bounds__(TABLE_THREADS) void table_scan_kernel(TableStep t) {
  int64_t rows = 0, blocks = *t.free_head;
  for (int j0 = 0; j0 < t.n_seq; j0 += TABLE_THREADS) {
    const int j = j0 + threadIdx.x;
    const SeqNeed n = j < t.n_seq ? seq_need(t, j) : SeqNeed{0, 0, 0};
    uint64_t r0, b0, rt, bt;
    table_scan(n.rows, max(0, n.need - n.have), r0, b0, rt, bt);  // its barriers: free_head is read by all
    if (j < t.n_seq) {
      t.seq_start[j] = saturated(rows + (int64_t)r0);
      t.free_start[j] = saturated(blocks + (int64_t)b0);
    }
    rows += rt;
    blocks += bt;
  }
  if (threadIdx.x == 0) {
    t.seq_start[t.n_seq] = saturated(rows);
    t.free_start[t.n_seq] = saturated(blocks);
  }
}

template <bool WHOLE>
__global__ __launch_bounds__(TABLE_THREADS) void table_kernel(TableStep t) {
  __shared__ TableSeq s;
  const int lane = threadIdx.x & 63;
  if constexpr (WHOLE) {
    const int j = threadIdx.x, head = *t.free_head;
    const SeqNeed n = j < t.n_seq ? seq_need(t, j) : SeqNeed{0, 0, 0};
    const int cached = j < t.n_seq ? max(t.cached[j], 0) : 0, slot = j < t.n_seq ? t.seq_slot[j] : -1;
    uint64_t r0, b0, rt, bt;
    table_scan(n.rows, max(0, n.need - n.have), r0, b0, rt, bt);
    const int start = saturated((int64_t)r0), taken = saturated(head + (int64_t)b0);
    s.start[j] = j < t.n_seq ? start : saturated((int64_t)rt);  // [n_seq]: the total
    s.taken[j] = taken;
    s.cached[j] = cached;
    s.have[j] = n.have;
    s.slot[j] = slot;
    if (blockIdx.x == 0) {
      if (j < t.n_seq) {
        t.seq_start[j] = start;
        t.free_start[j] = taken;
      }
      if (j == 0) {
        t.seq_start[t.n_seq] = saturated((int64_t)rt);
        t.free_start[t.n_seq] = saturated(head + (int64_t)bt);
      }
    }
    __syncthreads();
  }
  const int F = t.prefix_len / KV_BLOCK;
  for (int j = blockIdx.x * (TABLE_THREADS / 64) + (threadIdx.x >> 6); j < t.n_seq;
       j += gridDim.x * (TABLE_THREADS / 64)) {
    const int slot = WHOLE ? s.slot[j] : t.seq_slot[j];
    if (slot < 0 || slot >= t.n_slots) continue;
    const SeqNeed n = seq_need(t, j);
    int32_t *row = t.block_table + (int64_t)slot * t.max_blocks;
    const int64_t f0 = (int64_t)(WHOLE ? s.taken[j] : t.free_start[j]) - n.have;
    for (int b = lane; b < n.need; b += 64)
      if (b < F)
        row[b] = t.prefix_blocks[b];
      else if (b >= n.have)
        row[b] = free_block(t, f0 + b);
  }
  const int total = WHOLE ? s.start[t.n_seq] : t.seq_start[t.n_seq];
  for (int64_t r_ = blockIdx.x * TABLE_THREADS + threadIdx.x; r_ < t.max_rows; r_ += gridDim.x * TABLE_THREADS) {
    const int r = (int)r_;
    int slot = -1, pos = -1;
    int64_t entry = -1;
    if (r < total) {
      int lo = 0, hi = t.n_seq - 1;  // the last sequence that starts at or before the row
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((WHOLE ? s.start[mid] : t.seq_start[mid]) <= r) lo = mid;
        else hi = mid - 1;
      }
      slot = WHOLE ? s.slot[lo] : t.seq_slot[lo];
      pos = (WHOLE ? s.cached[lo] : max(t.cached[lo], 0)) + r - (WHOLE ? s.start[lo] : t.seq_start[lo]);
      const int b = pos / KV_BLOCK, have = WHOLE ? s.have[lo] : seq_need(t, lo).have;
      int id = -1;
      if (slot < 0 || slot >= t.n_slots) id = -1;
      else if (pos < t.prefix_len) id = t.prefix_blocks[b];
      else if (b >= t.max_blocks) id = -1;
      else if (b >= have) id = free_block(t, (int64_t)(WHOLE ? s.taken[lo] : t.free_start[lo]) + b - have);
      else id = t.block_table[(int64_t)slot * t.max_blocks + b];
      if (id >= 0) entry = (int64_t)id * KV_BLOCK + pos % KV_BLOCK;
    }
    t.row_slot[r] = slot;
    t.row_pos[r] = pos;
    t.row_entry[r] = entry;
  }
}

void launch_block_tables(const TableStep &t, hipStream_t s) {
  // a row for every thread, or a sequence for every wave, up to two workgroups a CU
  const int64_t by_rows = ((int64_t)t.max_rows + TABLE_THREADS - 1) / TABLE_THREADS;
  const int64_t by_seqs = ((int64_t)t.n_seq * 64 + TABLE_THREADS - 1) / TABLE_THREADS;
  const unsigned wgs = (unsigned)std::min<int64_t>(std::max(by_rows, by_seqs), 512);
  const bool in_place = t.free_head >= t.free_start && t.free_head <= t.free_start + t.n_seq;
  if (t.n_seq < TABLE_SEQS && (!in_place || wgs == 1)) {
    table_kernel<true><<<wgs, TABLE_THREADS, 0, s>>>(t);
  } else {
    table_scan_kernel<<<1, TABLE_THREADS, 0, s>>>(t);
    table_kernel<false><<<wgs, TABLE_THREADS, 0, s>>>(t);
  }
}

// ------------------------------------------------------------------ QKV append

// W values from / to consecutive places, in one access.
template <int W>
struct Floats {
  typedef float type __attribute__((ext_vector_type(W)));
};
template <typename T, int W>
__device__ __forceinline__ void store_w(T *dst, const float *v) {
  typedef T vec __attribute__((ext_vector_type(W)));
  vec x;
#pragma unroll
  for (int i = 0; i < W; ++i) x[i] = round_to<T>(v[i]);
  *(vec *)dst = x;
}

// Memory-bound: every projected value is read once and written once in its type.
//   * q and k heads: a thread takes W pairs (dims i .. and i + hd/2 ..) of a
//     row and head.
//   * v heads: the cache holds V transposed, 64 positions of one dim side by
//     side.  A workgroup takes TR rows of one head through LDS, so that a store's
//     lanes are rows: consecutive positions of a prompt leave as runs (a thread
//     per value stores 2 bytes to a line of its own each time: a prompt step of
//     about 4,200 rows, 8B heads, bf16, 53.8 us against 23.8, 5.25 TB/s).
template <typename T, int HD, int W, int TR>
__global__ __launch_bounds__(256) void qkv_append_kernel(QkvAppend a, T *__restrict__ q, T *__restrict__ k,
                                                         T *__restrict__ v, int v_wgs) {
  typedef typename Floats<W>::type vec;
  constexpr int HALF = HD / 2;
  if ((int)blockIdx.x >= v_wgs) {
    constexpr int TH = HALF / W;  // threads of a head
    const int heads = a.n_heads + a.n_kv_heads;
    const int per = (heads * TH + 255) / 256, b = blockIdx.x - v_wgs;
    const int r = b / per, e = (b - r * per) * 256 + threadIdx.x, h = e / TH, i = e % TH * W;
    if (h >= heads) return;
    const float *x = a.qkv + r * a.ld + h * HD + i;
    const vec x0 = *(const vec *)x, x1 = *(const vec *)(x + HALF);
    const int pos = a.row_pos[r];
    const int64_t entry = a.row_entry[r];
    if (pos < 0 || pos >= a.n_pos) return;
    T *dst;
    if (h < a.n_heads) {
      dst = q + ((int64_t)r * a.n_heads + h) * HD + i;
    } else {
      if (entry < 0 || entry >= a.n_blocks * KV_BLOCK) return;
      dst = k + ((entry / KV_BLOCK * a.n_kv_heads + h - a.n_heads) * KV_BLOCK + entry % KV_BLOCK) * HD + i;
    }
    const vec cs = *(const vec *)(a.rope_cos + (int64_t)pos * HALF + i);
    const vec sn = *(const vec *)(a.rope_sin + (int64_t)pos * HALF + i);
    float r0[W], r1[W];
#pragma unroll
    for (int e = 0; e < W; ++e) rope_rotate(x0[e], x1[e], cs[e], sn[e], r0[e], r1[e]);
    store_w<T, W>(dst, r0);
    store_w<T, W>(dst + HALF, r1);
    return;
  }
  // rows of the tile an odd number of 4-byte words apart: lanes that read one
  // dim of 64 rows meet no bank twice
  constexpr int LD = HD + 4 / sizeof(T);
  __shared__ T tile[TR * LD];
  const int h = blockIdx.x % a.n_kv_heads, r0 = blockIdx.x / a.n_kv_heads * TR;
  const float *x = a.qkv + (int64_t)r0 * a.ld + (int64_t)(a.n_heads + a.n_kv_heads + h) * HD;
  constexpr int RW = HD / W;  // threads of a row
  const int row = threadIdx.x % TR, r = r0 + row;
  const bool there = r < a.rows;
  const int pos = there ? a.row_pos[r] : -1;
  const int64_t entry = there ? a.row_entry[r] : -1;
#pragma unroll
  for (int e = 0; e < TR * RW / 256; ++e) {
    const int y = (e * 256 + threadIdx.x) / RW, d = (e * 256 + threadIdx.x) % RW * W;
    if (r0 + y < a.rows) {
      const vec f = *(const vec *)(x + (int64_t)y * a.ld + d);
#pragma unroll
      for (int i = 0; i < W; ++i) tile[y * LD + d + i] = round_to<T>(f[i]);
    }
  }
  __syncthreads();
  if (pos < 0 || pos >= a.n_pos || entry < 0 || entry >= a.n_blocks * KV_BLOCK) return;
  T *dst = v + (entry / KV_BLOCK * a.n_kv_heads + h) * KV_BLOCK * HD + entry % KV_BLOCK;
  constexpr int STEP = 256 / TR;
#pragma unroll 8
  for (int d = threadIdx.x / TR; d < HD; d += STEP) dst[d * KV_BLOCK] = tile[row * LD + d];
}

template <typename T, int HD, int W>
static void launch_append(const QkvAppend &a, T *q, T *k, T *v, hipStream_t s) {
  const int per = ((a.n_heads + a.n_kv_heads) * (HD / 2 / W) + 255) / 256;
  const auto run = [&](auto tr) {
    constexpr int TR = decltype(tr)::value;
    const int v_wgs = (a.rows + TR - 1) / TR * a.n_kv_heads;
    qkv_append_kernel<T, HD, W, TR><<<v_wgs + a.rows * per, 256, 0, s>>>(a, q, k, v, v_wgs);
  };
  // 64-row tiles of V store whole 128-byte runs; 16-row ones are four times the
  // workgroups, until there is a large one for each CU (graphs of calls, 16-row
  // against 64-row tiles: 8B heads 64 decode rows 4.0 us against 8.1, 1,000 rows of
  // four prompts, 128 large tiles, 7.2 and 8.3, 1,500 rows, 190, 10.8 and 10.9,
  // 2,600, 330, 15.0 and 14.4, 4,200, 528, 25.7 and 24.7; 7B heads 500 rows, 256, 8.1
  // and 8.4, 800, 400, 11.3 and 11.3)
  if ((int64_t)((a.rows + 63) / 64) * a.n_kv_heads >= 256)
    run(std::integral_constant<int, 64>());
  else
    run(std::integral_constant<int, 16>());
}

template <typename T>
void launch_qkv_append(const QkvAppend &a, T *q, T *k, T *v, hipStream_t s) {
  // 16-byte reads where the rows and tables allow them, else 8-byte ones
  const bool w4 = a.ld % 4 == 0 && (((uintptr_t)a.qkv | (uintptr_t)a.rope_cos | (uintptr_t)a.rope_sin) & 15) == 0;
  if (a.head_dim == 128)
    w4 ? launch_append<T, 128, 4>(a, q, k, v, s) : launch_append<T, 128, 2>(a, q, k, v, s);
  else
    w4 ? launch_append<T, 64, 4>(a, q, k, v, s) : launch_append<T, 64, 2>(a, q, k, v, s);
}

#define INST(T) template void launch_qkv_append<T>(const QkvAppend &, T *, T *, T *, hipStream_t);
INST(float)
INST(bf16_t)
INST(f16_t)
#undef INST

}  // namespace lp
