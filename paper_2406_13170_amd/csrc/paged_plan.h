// Arithmetic of the paged cache's kernels that the host checks and the CPU tests share with the device: how many rows a
// sequence has, and who walks which key steps of the attention.
#pragma once
#include <stdint.h>

namespace amph {

constexpr int PAGED_MAX_SEQ = 1024;           // a workgroup lists the sequences' lengths in LDS: four a thread
constexpr int PAGED_WAVES = 4;                // waves of an attention workgroup; they take a walk's key steps in turn
constexpr int PAGED_WGS = 512;                // attention workgroups: two a compute unit, what its registers allow

// Rows of a sequence: len of them before this step, new_rows of it; -1 where they do not fit cap rows or are no lengths at all.
__host__ __device__ inline int paged_rows(int len, int new_rows, int cap) {
  return (len < 0 || len > cap || new_rows > cap - len) ? -1 : len + new_rows;
}
__host__ __device__ inline int paged_new(int n_new, int valid) { return valid < 0 ? 0 : valid < n_new ? valid : n_new; }

// The key steps of all walks in one line (sequence by sequence; the walks of a sequence, one for each key head and query group,
// one after the other) are dealt out in equal pieces, whatever the lengths: piece w has the steps [w * chunk, (w + 1) * chunk).
__host__ __device__ inline int paged_chunk(long long total, int wgs) {
  const long long c = (total + wgs - 1) / wgs;
  const int r = (int)((c + PAGED_WAVES - 1) / PAGED_WAVES) * PAGED_WAVES;
  return r < PAGED_WAVES ? PAGED_WAVES : r;
}
// Of one walk [first, first + steps) of that line: the pieces that reach into it, and where piece w leaves its partial result.
// A piece has at most two walks that it does not hold whole: the one it begins with (place 0) and the one it ends with (place 1).
struct PagedWalk {
  int w0, w1;
  bool begins;                                // piece w0 begins with this walk
  __host__ __device__ int place(int w) const { return 2 * w + (w == w0 && !begins ? 1 : 0); }
};
__host__ __device__ inline PagedWalk paged_walk(long long first, int steps, int chunk) {
  PagedWalk p;
  const unsigned long long last = (unsigned long long)first + steps - 1;
  if (last >> 32) {                           // (a 64-bit division costs some hundred instructions)
    p.w0 = (int)(first / chunk);
    p.w1 = (int)(last / chunk);
  } else {
    p.w0 = (int)((unsigned)first / (unsigned)chunk);
    p.w1 = (int)((unsigned)last / (unsigned)chunk);
  }
  p.begins = first == (long long)p.w0 * chunk;
  return p;
}

}  // namespace amph
