// What the files of the selective scan share: its arguments, where a workgroup stands, and clearing rows.  selective_scan.hip says what the kernels do.
#pragma once

#include <type_traits>
#include <utility>

#include "nugpr_internal.h"
#include "packed_rows.h"
#include "row_values.h"

namespace nugpr {

constexpr int TILE_ROWS = 16;
constexpr int ZERO_GROUPS = 128;     // workgroups that clear the rows without a sequence

// Up to that many sequences, spans are numbered one after the other, and a workgroup finds its own by counting; beyond, by piece_of, whose
// numbers have gaps.  (Gaps cost more than their workgroups' time: workgroups go to the compute units in turn, the empty ones too, and some units get more of
// the others than the rest.  16 x 1024 rows, 2048 channels, every second number a gap: 285 us instead of 185; 256 x 64 rows, 1024 channels counted 151 us,
// 257 of 63 with gaps 186.  Counting goes with the number of sequences: 1000 x 65 rows took 508 us counted, 469 with gaps.)
constexpr int COUNTED = 256;

struct ScanArgs {
  const void *x, *dt, *z, *B, *C, *dy;
  void *y, *dx, *ddt, *dz;
  int64_t x_row, dt_row, z_row, y_row, dy_row, dx_row, ddt_row, dz_row;
  int64_t B_row, B_head, C_row, C_head;
  const float *A, *D, *bias;
  const float *s_in, *ds_end;        // states at the sequences' begin; gradients of those at their end
  float *s_out, *ds_in;
  const int64_t* off;
  int64_t n_rows;
  int n_seqs, dim, groups, each, states, softplus, bf16;       // each: channels of a group
  int width, blocks;                 // channels of a workgroup; workgroups that have all
  int share;                         // states of a wave (of each chunk): as even as they can be shared out
  int threads, per_thread;           // the gradients': of a workgroup; states of a thread
  int span_log2, items;
  int64_t whole;                     // sequences are not cut into spans where none has more rows
  float* adds;                       // items x dim x states: what a span adds to the state, then its start state
  float* steps;                      // items x dim: sum of a span's d
  float* back;                       // the same as adds, of the gradients
  float* tiles;                      // tiles x blocks x threads x 4: states at the tiles' begin (from zero, but in a sequence's first span)
  float* tile_steps;                 // tiles x dim: sum of the span's d before the tile
  float *dB, *dC;                    // blocks of a group x n_rows x groups x states
  float *dA, *dD, *dbias;            // items x dim (x states)
  void *dB_out, *dC_out;             // the gradients themselves, from these parts
  int64_t dB_row, dB_head, dC_row, dC_head;
  float *dA_out, *dD_out, *dbias_out;
};

// A as the exponents of two take it: a factor is 2^(d rate).  (-infinity as a number, so that rows with d = 0 keep the state; NaN stays.)
__device__ __forceinline__ float rate_of(float A) {
  const float r = A * LOG2_E;
  return r < -3e38f ? -3e38f : r;
}

// f h + add with the factor of many steps, which may be zero where none of a single step is: an infinite h stays so.
__device__ __forceinline__ float over_steps(float f, float h, float add) {
  return h == 0.f || (f == 0.f && __builtin_isinf(h)) ? h + add : fmaf(f, h, add);
}

// Sum over the lanes up to this one.
__device__ __forceinline__ int sum_to_lane(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);       // of the lane before, two, four, eight before among 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // the last of 16 to the next 16, of 32 to the next 32
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

__device__ __forceinline__ int spans_of(const ScanArgs& a, int64_t lo, int64_t hi) {
  return hi == lo ? 1 : (int)((hi - lo + ((int64_t)1 << a.span_log2) - 1) >> a.span_log2);
}

// The spans of COUNTED sequences at most, a lane every 64th sequence.  (Whole waves.)
struct Counted {
  static constexpr int K = COUNTED / 64;
  int64_t lo[K], hi[K];
  int spans[K], to[K];               // how many the sequence has; the sum up to it, among 64
  // Whether a sequence is longer than those that are walked through whole.  Then all are cut, as what is short and walked through whole would still
  // be under way when the pieces of the long ones have ended.
  bool cut;
  __device__ __forceinline__ Counted(const ScanArgs& a) {
    const int lane = threadIdx.x & 63;
    uint64_t longer = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int at = k * 64 + lane;
      lo[k] = at < a.n_seqs ? a.off[at] : 0;
      hi[k] = at < a.n_seqs ? a.off[at + 1] : 0;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      lo[k] = clamped(lo[k], 0, a.n_rows);
      hi[k] = clamped(hi[k], lo[k], a.n_rows);
      longer |= __ballot(hi[k] - lo[k] > a.whole);
    }
    cut = longer != 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      spans[k] = k * 64 + lane >= a.n_seqs ? 0 : cut ? spans_of(a, lo[k], hi[k]) : 1;
      to[k] = sum_to_lane(spans[k]);
    }
  }
  // the number of a sequence's first span
  __device__ __forceinline__ int first(int seq) const {
    int before = 0;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (seq >= k * 64) before += __builtin_amdgcn_readlane(seq < k * 64 + 64 ? to[k] - spans[k] : to[k], seq < k * 64 + 64 ? seq - k * 64 : 63);
    return before;
  }
};

// Where a workgroup stands.
struct Place {
  int group, channel, valid;         // its first channel, and how many it has
  PieceOf piece;
  int64_t from, to;                  // its rows
  int span;                          // of the sequence
  bool last;                         // the sequence ends with it
};

__device__ __forceinline__ bool find(const ScanArgs& a, int item, int block, Place& p) {
  const int of_group = a.blocks / a.groups, b = block % of_group;
  p.group = block / of_group;
  p.channel = p.group * a.each + b * a.width;
  p.valid = min(a.width, a.each - b * a.width);
  bool cut = true;
  if (a.n_seqs > COUNTED) {
    p.piece = piece_of(a.off, a.n_seqs, a.n_rows, a.span_log2, item);
    if (p.piece.seq < 0) return false;
    p.span = item - (int)((p.piece.lo >> a.span_log2) + p.piece.seq);
    if (p.span >= spans_of(a, p.piece.lo, p.piece.hi)) return false;
  } else {
    const Counted c(a);
    cut = c.cut;
    int left = item;                 // spans of later sequences than those looked at
    p.piece.seq = -1;
#pragma unroll
    for (int k = 0; k < Counted::K; ++k) {
      const int all = __builtin_amdgcn_readlane(c.to[k], 63);
      if (p.piece.seq < 0 && left < all) {
        const int n = __popcll(__ballot(c.to[k] <= left));
        p.piece = PieceOf{k * 64 + n, of_lane(c.lo[k], n), of_lane(c.hi[k], n)};
        p.span = left - __builtin_amdgcn_readlane(c.to[k] - c.spans[k], n);
      }
      left -= all;
    }
    if (p.piece.seq < 0) return false;
  }
  p.from = p.piece.lo + ((int64_t)p.span << a.span_log2);
  p.to = !cut ? p.piece.hi : min(p.piece.hi, p.from + ((int64_t)1 << a.span_log2));
  p.last = p.to == p.piece.hi;
  return true;
}

// f(0), f(1), ..: with the number as a constant
template <class F, int... I>
__device__ __forceinline__ void repeat_all(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void repeat(F f) { repeat_all(f, std::make_integer_sequence<int, N>{}); }

// Rows before the first sequence and behind the last are cleared by workgroups of their own.
template <class TR>
__device__ void clear_rows(const ScanArgs& a, int who, void* to, int64_t stride) {
  if (!to) return;
  const int64_t first = clamped(a.off[0], 0, a.n_rows), last = clamped(a.off[a.n_seqs], first, a.n_rows);
  Values<TR, 4> zero;
  zero.clear();
  for (int64_t row = who; row < a.n_rows - (last - first); row += ZERO_GROUPS) {
    typename TR::T* p = static_cast<typename TR::T*>(to) + (row < first ? row : row + (last - first)) * stride;
    for (int col = threadIdx.x * 4; col < a.dim; col += blockDim.x * 4) zero.store(p + col, a.dim - col);
  }
}

// The gradients' kernels (selective_scan_backward.hip): their workgroups' shape, and the launches.  join: the kernel that goes from what
// spans add to their start states.
int scan_backward_width(int states);       // channels of a workgroup
int scan_backward_threads(int states);     // its threads
int scan_backward_states(int states);      // states of a thread: side by side, neighbouring threads have a channel's next
int launch_scan_backward(int dtype, const ScanArgs& a, bool one_span, void (*join)(const ScanArgs&, bool, hipStream_t), hipStream_t s);

}  // namespace nugpr
