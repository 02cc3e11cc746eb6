// Sequences (or requests) packed one after the other: sequence s owns rows offsets[s] .. offsets[s + 1] - 1.  Offsets stay on
// the device; kernels clamp them to the rows that there are, so that no offset leads out of bounds.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nugpr {

__device__ inline int64_t clamped(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }

// Sequence s has the piece numbers from (offsets[s] >> piece_log2) + s on: with ceil(rows / piece) pieces it ends before the next
// one's, so no table of them is needed.  The sequence of a piece is the last one that begins at or before it (seq < 0: none; where offsets do
// not ascend the search may end at one that begins later, which has no such piece); lo, hi: its rows.
struct PieceOf {
  int seq;
  int64_t lo, hi;
};
__device__ inline int64_t of_lane(int64_t x, int lane) {
  const uint32_t l = __builtin_amdgcn_readlane((int)(uint32_t)x, lane), h = __builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane);
  return (int64_t)((uint64_t)h << 32 | l);
}
__device__ inline PieceOf piece_of(const int64_t* off, int n_seqs, int64_t n_rows, int piece_log2, int item) {
  const int lane = threadIdx.x & 63;
  int from = 0, to = n_seqs;                  // the sequence lies in [from, to)
  while (to - from > 64) {                    // 64 probes a round
    const int step = (to - from + 63) / 64;
    const int at = from + lane * step;
    const bool before = at < to && (clamped(off[at], 0, n_rows) >> piece_log2) + at <= item;
    const int n = __popcll(__ballot(before));
    if (n == 0) return PieceOf{-1, 0, 0};
    from += (n - 1) * step;
    to = min(to, from + step);
  }
  const int at = from + lane;
  int64_t lo = 0, hi = 0;
  if (at < to) {
    lo = clamped(off[at], 0, n_rows);
    hi = clamped(off[at + 1], lo, n_rows);
  }
  const int n = __popcll(__ballot(at < to && (lo >> piece_log2) + at <= item)) - 1;
  if (n < 0) return PieceOf{-1, 0, 0};
  const PieceOf p{from + n, of_lane(lo, n), of_lane(hi, n)};
  return (p.lo >> piece_log2) + p.seq <= item ? p : PieceOf{-1, 0, 0};
}

// The sequence that owns a row: the last one that begins at or before it, if it reaches that far; else -1.  (All lanes of a wave
// with the same row.)
__device__ inline int owner_of(const int64_t* off, int n_seqs, int64_t row) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n_seqs;
  while (hi - lo > 64) {
    const int step = (hi - lo + 63) / 64;
    const int at = lo + lane * step;
    const int n = __popcll(__ballot(at < hi && off[at] <= row));
    if (n == 0) return -1;
    const int from = lo + (n - 1) * step;
    hi = min(hi, from + step);
    lo = from;
  }
  const int at = lo + lane;
  const int s = lo + __popcll(__ballot(at < hi && off[at] <= row)) - 1;
  return s >= 0 && row < off[s + 1] ? s : -1;
}

}  // namespace nugpr
