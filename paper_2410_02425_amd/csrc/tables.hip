// What comes before attention over a paged cache in a step that the caller
// plans: block tables and cache entries from lengths, and the QKV projection's
// K and V into those entries.
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

// Exclusive sums of the sequences' rows and blocks, 1,024 sequences at a time.
__global__ __launch_bounds__(1024) void table_scan_kernel(TableStep t) {
  __shared__ uint64_t wsum[2][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t rows = 0, blocks = *t.free_head;
  __syncthreads();  // free_head may be the last element of free_start
  for (int j0 = 0; j0 < t.n_seq; j0 += 1024) {
    const int j = j0 + threadIdx.x;
    const SeqNeed n = j < t.n_seq ? seq_need(t, j) : SeqNeed{0, 0, 0};
    const uint64_t take = max(0, n.need - n.have);
    const uint64_t r = wave_scan((uint64_t)n.rows), b = wave_scan(take);
    if (lane == 63) {
      wsum[0][wave] = r;
      wsum[1][wave] = b;
    }
    __syncthreads();
    uint64_t r0 = 0, b0 = 0, rt = 0, bt = 0;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) r0 += wsum[0][w], b0 += wsum[1][w];
      rt += wsum[0][w], bt += wsum[1][w];
    }
    if (j < t.n_seq) {
      t.seq_start[j] = (int)min(rows + (int64_t)(r0 + r - n.rows), (int64_t)INT32_MAX);
      t.free_start[j] = (int)min(blocks + (int64_t)(b0 + b - take), (int64_t)INT32_MAX);
    }
    rows += rt;
    blocks += bt;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    t.seq_start[t.n_seq] = (int)min(rows, (int64_t)INT32_MAX);
    t.free_start[t.n_seq] = (int)min(blocks, (int64_t)INT32_MAX);
  }
}

__device__ __forceinline__ int free_block(const TableStep &t, int64_t i) {
  return i >= 0 && i < t.n_free ? t.free_blocks[i] : -1;
}

// Table rows, a wave per sequence, and the packed rows, a thread each.
__global__ __launch_bounds__(256) void table_fill_kernel(TableStep t, int table_wgs) {
  if ((int)blockIdx.x < table_wgs) {
    const int j = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (j >= t.n_seq) return;
    const int slot = t.seq_slot[j];
    if (slot < 0 || slot >= t.n_slots) return;
    const SeqNeed n = seq_need(t, j);
    int32_t *row = t.block_table + (int64_t)slot * t.max_blocks;
    const int whole = min(t.prefix_len / KV_BLOCK, n.need);
    for (int b = lane; b < whole; b += 64) row[b] = t.prefix_blocks[b];
    const int64_t f0 = t.free_start[j];
    for (int b = n.have + lane; b < n.need; b += 64) row[b] = free_block(t, f0 + b - n.have);
    return;
  }
  const int r = (blockIdx.x - table_wgs) * 256 + threadIdx.x;
  if (r >= t.max_rows) return;
  int slot = -1, pos = -1;
  int64_t entry = -1;
  if (r < t.seq_start[t.n_seq]) {
    int lo = 0, hi = t.n_seq - 1;  // the last sequence that starts at or before the row
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (t.seq_start[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    const SeqNeed n = seq_need(t, lo);
    slot = t.seq_slot[lo];
    pos = max(t.cached[lo], 0) + r - t.seq_start[lo];
    const int b = pos / KV_BLOCK;
    int id = -1;
    if (slot < 0 || slot >= t.n_slots) id = -1;
    else if (pos < t.prefix_len) id = t.prefix_blocks[b];
    else if (b >= t.max_blocks) id = -1;
    else if (b >= n.have) id = free_block(t, (int64_t)t.free_start[lo] + b - n.have);
    else id = t.block_table[(int64_t)slot * t.max_blocks + b];
    if (id >= 0) entry = (int64_t)id * KV_BLOCK + pos % KV_BLOCK;
  }
  t.row_slot[r] = slot;
  t.row_pos[r] = pos;
  t.row_entry[r] = entry;
}

void launch_block_tables(const TableStep &t, hipStream_t s) {
  table_scan_kernel<<<1, 1024, 0, s>>>(t);
  const int table_wgs = (t.n_seq + 3) / 4;
  table_fill_kernel<<<table_wgs + (t.max_rows + 255) / 256, 256, 0, s>>>(t, table_wgs);
}

// ------------------------------------------------------------------ QKV append

// One workgroup per row, a thread per pair of elements.
template <typename T>
__global__ __launch_bounds__(256) void qkv_append_kernel(QkvAppend a, T *__restrict__ q, T *__restrict__ k,
                                                         T *__restrict__ v) {
  const int r = blockIdx.x, hd = a.head_dim, half = hd / 2;
  const int pos = a.row_pos[r];
  if (pos < 0 || pos >= a.n_pos) return;
  const int64_t entry = a.row_entry[r];
  const bool kept = entry >= 0 && entry < a.n_blocks * KV_BLOCK;
  const int64_t blk = entry / KV_BLOCK;
  const int off = (int)(entry % KV_BLOCK);
  const float *x = a.qkv + r * a.ld;
  const int pairs = (a.n_heads + 2 * a.n_kv_heads) * half;
  for (int p = threadIdx.x; p < pairs; p += 256) {
    const int h = p / half, i = p % half;
    if (h < a.n_heads + a.n_kv_heads) {
      float r0, r1;
      rope_rotate(x[h * hd + i], x[h * hd + i + half], a.rope_cos[(int64_t)pos * half + i],
                  a.rope_sin[(int64_t)pos * half + i], r0, r1);
      T *dst;
      if (h < a.n_heads) {
        dst = q + ((int64_t)r * a.n_heads + h) * hd;
      } else {
        if (!kept) continue;
        dst = k + ((blk * a.n_kv_heads + h - a.n_heads) * KV_BLOCK + off) * hd;
      }
      dst[i] = Act<T>::st(r0);
      dst[i + half] = Act<T>::st(r1);
    } else if (kept) {
      T *dst = v + (blk * a.n_kv_heads + h - a.n_heads - a.n_kv_heads) * KV_BLOCK * hd + off;
      dst[(int64_t)(2 * i) * KV_BLOCK] = Act<T>::st(x[h * hd + 2 * i]);
      dst[(int64_t)(2 * i + 1) * KV_BLOCK] = Act<T>::st(x[h * hd + 2 * i + 1]);
    }
  }
}

template <typename T>
void launch_qkv_append(const QkvAppend &a, T *q, T *k, T *v, hipStream_t s) {
  qkv_append_kernel<T><<<a.rows, 256, 0, s>>>(a, q, k, v);
}

#define INST(T) template void launch_qkv_append<T>(const QkvAppend &, T *, T *, T *, hipStream_t);
INST(float)
INST(bf16_t)
INST(f16_t)
#undef INST

}  // namespace lp
