// Rows of a batch whose sequences and positions are on the device (PrefixBatch),
// shared by the kernels of such batches.
#pragma once
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <algorithm>

#include "device.hpp"
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

// Keys that row i of sequence j sees, of a sequence in `slot` from position p0 on.
__device__ __forceinline__ int row_ctx(const PrefixBatch &b, int slot, int p0, int i) {
  if (slot < 0 || slot >= b.n_slots) return 0;
  const int64_t ctx = (int64_t)p0 + i + 1;
  return p0 < 0 ? 0 : (int)min(ctx, (int64_t)b.max_ctx);
}
__device__ __forceinline__ int row_ctx(const PrefixBatch &b, int j, int i) {
  return row_ctx(b, b.seq_slot[j], b.seq_pos[j], i);
}

// Rows are packed: a sequence's tokens, each with the G query heads of a KV head.
// The arguments A of a kernel hold the batch b, G, and divisors by G (by_g) and by
// the tiles of a decode row's G heads (by_per).

struct PrefixRow {
  int token, head, t;  // t: the token's place in its sequence, or in the batch
};

// Row l of the packed rows from r0 (uniform) on: of all tokens, or of a sequence
// whose first token is `start`.
template <typename A>
__device__ __forceinline__ PrefixRow packed_row(const A &a, int start, int r0, int l, int g) {
  const int t0 = div_by(r0, a.by_g), x = r0 - t0 * a.G + l, dt = div_by(x, a.by_g);
  return PrefixRow{start + t0 + dt, g * a.G + x - dt * a.G, t0 + dt};
}

// Own tile u of RT packed rows: sequence by sequence, each with as many tiles as
// its rows need.  Each wave finds it on its own: an inclusive sum over 64
// sequences at a time, the first whose sum exceeds u.  False past the last.  The
// sequence's rows (those with a result, max_new at most), slot and position come from
// the same lanes, requested together.
struct TileSeq {
  int start, n, slot, p0;
};
template <int RT, typename A>
__device__ __forceinline__ bool own_tile(const A &a, int u, int &j, int &r0, TileSeq &s) {
  const int lane = threadIdx.x & 63;
  if (!a.b.seq_start) {  // one row a sequence
    j = __builtin_amdgcn_readfirstlane(div_by(u, a.by_per));  // its loads stay scalar
    r0 = (u - j * (int)a.by_per.d) * RT;
    if (j >= a.b.n_seq) return false;
    s = TileSeq{j, 1, a.b.seq_slot[j], a.b.seq_pos[j]};
    return true;
  }
  for (int base = 0; base < a.b.n_seq; base += 64) {
    int start = 0, n = 0, slot = -1, p0 = -1;
    if (base + lane < a.b.n_seq) {
      seq_rows(a.b, base + lane, start, n);
      n = min(n, a.b.max_new);
      slot = a.b.seq_slot[base + lane];
      p0 = a.b.seq_pos[base + lane];
    }
    const int tiles = (int)(((int64_t)n * a.G + RT - 1) / RT);
    const int incl = (int)wave_scan((uint64_t)tiles);
    const int total = __builtin_amdgcn_readlane(incl, 63);
    if (u < total) {
      const int k = __popcll(__ballot(incl <= u));  // sequences wholly before the tile
      j = base + k;
      r0 = (__shfl(incl, k, 64) - 1 - u) * RT;  // from the last, whose rows see most
      s = TileSeq{__shfl(start, k, 64), __shfl(n, k, 64), __shfl(slot, k, 64), __shfl(p0, k, 64)};
      return true;
    }
    u -= total;
  }
  return false;
}

template <int RT, typename A>
__device__ __forceinline__ bool own_tile(const A &a, int u, int &j, int &r0) {
  TileSeq s;
  return own_tile<RT>(a, u, j, r0, s);
}

static int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

}  // namespace lp
