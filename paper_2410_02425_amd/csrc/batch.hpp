// Rows of a batch whose sequences and positions are on the device (PrefixBatch),
// shared by the kernels of such batches.
#pragma once
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <algorithm>

#include "kernels.hpp"

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

static int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

}  // namespace lp
