// Arithmetic of the paged cache's kernels that the host checks and the CPU tests share with the device: how many rows a
// sequence has, and who walks which key steps of the attention.
#pragma once
#include <stdint.h>

namespace amph {

constexpr int PAGED_MAX_SEQ = 1024;           // a workgroup lists the sequences' lengths in LDS: four a thread
constexpr int PAGED_WAVES = 4;                // waves of an attention workgroup; they take a walk's key steps in turn
constexpr int PAGED_WGS = 512;                // attention workgroups: two a compute unit

// Rows of a sequence: len of them before this step, new_rows of it; -1 where they do not fit cap rows or are no lengths at all.
__host__ __device__ inline int paged_rows(int len, int new_rows, int cap) {
  return (len < 0 || len > cap || new_rows > cap - len) ? -1 : len + new_rows;
}
__host__ __device__ inline int paged_new(int n_new, int valid) { return valid < 0 ? 0 : valid < n_new ? valid : n_new; }

// The key steps of all walks in one line (sequence by sequence; the walks of a sequence, one for each key head and query group,
// one after the other) are dealt out in equal pieces, whatever the lengths: piece w begins at begin(w).  The first `rem` pieces have
// base + 1 steps, the others base; with few steps in all, a step for every wave and fewer pieces.
struct PagedDeal {
  int base, rem;
  __host__ __device__ long long begin(int w) const { return (long long)w * base + (w < rem ? w : rem); }
  __host__ __device__ int piece(long long step) const {                // the piece that a step is in
    const long long big = (long long)rem * (base + 1);
    const bool first = step < big;
    const unsigned long long off = first ? step : step - big;
    const unsigned n = first ? base + 1 : base;
    return (off >> 32 ? (int)(off / n) : (int)((unsigned)off / n)) + (first ? 0 : rem);     // (64-bit division: some hundred instructions)
  }
};
__host__ __device__ inline PagedDeal paged_deal(long long total) {
  if (total < (long long)PAGED_WAVES * PAGED_WGS) return {PAGED_WAVES, 0};
  return {(int)(total / PAGED_WGS), (int)(total % PAGED_WGS)};
}
// Of one walk [first, first + steps) of that line: the pieces that reach into it, and where piece w leaves its partial result.
// A piece has at most two walks that it does not hold whole: the one it begins with (place 0) and the one it ends with (place 1).
struct PagedWalk {
  int w0, w1;
  bool begins;                                // piece w0 begins with this walk
  __host__ __device__ int place(int w) const { return 2 * w + (w == w0 && !begins ? 1 : 0); }
};
__host__ __device__ inline PagedWalk paged_walk(long long first, int steps, PagedDeal d) {
  PagedWalk p;
  p.w0 = d.piece(first);
  p.w1 = d.piece(first + steps - 1);
  p.begins = first == d.begin(p.w0);
  return p;
}

}  // namespace amph
