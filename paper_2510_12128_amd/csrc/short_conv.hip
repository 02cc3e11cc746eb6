// Causal convolution along packed sequences, every channel by itself, with bias and SiLU: forward, gradients, and one token at a time.
//
//   p_t = b + sum_{k < W} w[W-1-k] x_{t-k},   y = p or p sigmoid(p)
//   dp_t = dy_t, or dy_t s (1 + p (1 - s)) with s = sigmoid(p_t)
//   dx_t = sum_k w[W-1-k] dp_{t+k},   dw[W-1-k] = sum_t dp_t x_{t-k},   db = sum_t dp_t
//
// Memory traffic bounds it.  A wave takes a run of rows of 64 V channels, V side by side a lane, and keeps the rows that it
// still needs in registers, so that a row is read once, and W - 1 rows more a run.
#include <algorithm>

#include "call_checks.h"
#include "packed_rows.h"
#include "row_values.h"

namespace nugpr {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int MAX_WIDTH = 8;
constexpr int COMPUTE_UNITS = 256;
constexpr int AHEAD = 4;               // rows that are loaded at one time

struct ConvArgs {
  const void *x, *dy;
  void *y, *dx;
  int64_t x_row, y_row, dy_row, dx_row;
  const void *weight, *bias;
  const void *w_in, *dw_end;           // windows at the sequences' begin; gradients of those at their end
  void *w_out, *dw_in;                 // windows at their end; gradients of those at their begin
  float* sums;                         // of dw and db: runs of a workgroup x (W + 1) x dim
  const int64_t* off;
  int64_t n_rows;
  int64_t runs;                        // workgroups along the rows
  int n_seqs, dim, silu, col_blocks;
  int64_t run;                         // rows of a wave
};

template <class TR>
__device__ inline float gate(float p) {
  return p * sigmoid_of<TR>(p);
}

// A run of rows of one sequence (or of none), ending where that does.
struct Piece {
  int seq;             // < 0: no sequence owns the rows
  int64_t lo, hi;      // the sequence's rows; without one: as far as there is none
};
__device__ inline Piece piece_at(const ConvArgs& a, int64_t row, int64_t end) {
  const int s = owner_of(a.off, a.n_seqs, row);
  if (s >= 0) return Piece{s, clamped(a.off[s], 0, row), clamped(a.off[s + 1], row + 1, a.n_rows)};
  const int64_t first = a.n_seqs > 0 ? a.off[0] : 0;
  return Piece{-1, 0, row < first ? clamped(first, row + 1, end) : end};
}

// Row t - back of the sequence, which may lie in its window.
template <class TR, int W, int V>
__device__ inline void load_back(Values<TR, V>& v, const ConvArgs& a, const Piece& p, int64_t row, int col, int valid) {
  typedef typename TR::T T;
  if (row >= p.lo) v.load(static_cast<const T*>(a.x) + row * a.x_row + col, valid);
  else if (a.w_in) v.load(static_cast<const T*>(a.w_in) + ((int64_t)p.seq * (W - 1) + (W - 1) + (row - p.lo)) * a.dim + col, valid);
  else v.clear();
}

template <class TR, int W, int V>
__device__ inline void load_weights(float (&w)[W][V], float (&b)[V], const ConvArgs& a, int col, int valid) {
  typedef typename TR::T T;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    b[j] = a.bias && j < valid ? TR::get(static_cast<const T*>(a.bias)[col + j]) : 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) w[i][j] = j < valid ? TR::get(static_cast<const T*>(a.weight)[(int64_t)(col + j) * W + i]) : 0.f;
  }
}

// Rows come and go once: 16384 rows, 4096 channels, four taps, bfloat16: 54 us, 4.9 TB/s where a copy reaches 5.1.  A lane loads AHEAD rows and only then
// computes; the rows that taps reach back to are registers that move on.
template <class TR, int W, int V>
__global__ __launch_bounds__(THREADS) void k_short_conv(const ConvArgs a) {
  typedef typename TR::T T;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int block = blockIdx.x % a.col_blocks;
  const int64_t group = blockIdx.x / a.col_blocks;
  const int col = (block * 64 + lane) * V, valid = a.dim - col;
  if (group >= a.runs) {                        // the windows at the sequences' end
    const int64_t s = (group - a.runs) * WAVES + wave;
    if (s >= a.n_seqs || valid <= 0) return;
    const int64_t lo = clamped(a.off[s], 0, a.n_rows), len = clamped(a.off[s + 1], lo, a.n_rows) - lo;
    const Piece p{(int)s, lo, lo + len};
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
      Values<TR, V> v;
      load_back<TR, W, V>(v, a, p, lo + len - (W - 1) + i, col, valid);
      v.store(static_cast<T*>(a.w_out) + (s * (W - 1) + i) * a.dim + col, valid);
    }
    return;
  }
  int64_t t = (group * WAVES + wave) * a.run;
  const int64_t end = min(a.n_rows, t + a.run);
  if (t >= end) return;                         // (lanes beyond the channels stay: the search for a row's sequence needs all)
  float w[W][V], b[V];
  load_weights<TR, W, V>(w, b, a, col, valid);
  while (t < end) {
    const Piece p = piece_at(a, t, end);
    const int64_t stop = min(end, p.hi);
    if (p.seq < 0) {
      Values<TR, V> zero;
      zero.clear();
      for (; t < stop; ++t) zero.store(static_cast<T*>(a.y) + t * a.y_row + col, valid);
      continue;
    }
    float x[W - 1 + AHEAD][V];                  // rows t - (W - 1) on
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
      Values<TR, V> v;
      load_back<TR, W, V>(v, a, p, t - (W - 1) + i, col, valid);
#pragma unroll
      for (int j = 0; j < V; ++j) x[i][j] = v.get(j);
    }
    for (; t < stop; t += AHEAD) {
      Values<TR, V> v[AHEAD];
#pragma unroll
      for (int r = 0; r < AHEAD; ++r) {
        if (t + r < stop) v[r].load(static_cast<const T*>(a.x) + (t + r) * a.x_row + col, valid);
        else v[r].clear();
      }
#pragma unroll
      for (int r = 0; r < AHEAD; ++r) {
        float y[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          x[W - 1 + r][j] = v[r].get(j);
          float s = b[j];
#pragma unroll
          for (int i = 0; i < W; ++i) s = fmaf(w[i][j], x[r + i][j], s);
          y[j] = a.silu ? gate<TR>(s) : s;
        }
        if (t + r < stop) {
          Values<TR, V> o;
          o.put(y);
          o.store(static_cast<T*>(a.y) + (t + r) * a.y_row + col, valid);
        }
      }
#pragma unroll
      for (int i = 0; i < W - 1; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) x[i][j] = x[AHEAD + i][j];
    }
    t = stop;
  }
}

// dp from p and dy
template <class TR>
__device__ inline float gate_gradient(float p, float dy) {
  const float s = sigmoid_of<TR>(p);
  return dy * s * fmaf(p, 1.f - s, 1.f);
}

// Gradients.  A run's dx needs dp of W - 1 rows behind it too (as far as the sequence goes): they are computed once more there.
// p is computed anew from x: the forward pass keeps nothing.  dw and db stay in registers over the run, join over the workgroup's waves in LDS and go to
// memory once a workgroup.  16384 rows, 2048 channels, four taps, bfloat16: 47 us, 4.2 TB/s of x, dy and dx (behind it k_conv_sums, 5 us); runs of 32 rows,
// for enough workgroups, read a tenth more than their own.
// (The bound: up to four taps four waves a SIMD, for which the compiler would take a register too many by itself.)
template <class TR, int W, int V>
__global__ __launch_bounds__(THREADS, W <= 4 ? 4 : 2) void k_short_conv_backward(const ConvArgs a) {
  typedef typename TR::T T;
  constexpr int UP = 2;                         // rows at one time
  __shared__ float red[WAVES - 1][W + 1][64 * V];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int block = blockIdx.x % a.col_blocks;
  const int64_t group = blockIdx.x / a.col_blocks;
  const int col = (block * 64 + lane) * V, valid = a.dim - col;
  float w[W][V], b[V];
  load_weights<TR, W, V>(w, b, a, col, valid);
  if (group >= a.runs) {                        // gradients of the windows: row i meets the sequence's rows q <= i
    const int64_t s = (group - a.runs) * WAVES + wave;
    if (s >= a.n_seqs || valid <= 0) return;
    const int64_t lo = clamped(a.off[s], 0, a.n_rows), len = clamped(a.off[s + 1], lo, a.n_rows) - lo;
    const Piece p{(int)s, lo, lo + len};
    float dp[W][V], x[2 * W][V];
#pragma unroll
    for (int i = 0; i < 2 * (W - 1); ++i) {
      Values<TR, V> v;
      if (i - (W - 1) < len) load_back<TR, W, V>(v, a, p, lo - (W - 1) + i, col, valid);
      else v.clear();
#pragma unroll
      for (int j = 0; j < V; ++j) x[i][j] = v.get(j);
    }
#pragma unroll
    for (int q = 0; q < W - 1; ++q) {
      Values<TR, V> v;
      v.clear();
      if (q < len) v.load(static_cast<const T*>(a.dy) + (lo + q) * a.dy_row + col, valid);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float sum = b[j];
#pragma unroll
        for (int i = 0; i < W; ++i) sum = fmaf(w[i][j], x[q + i][j], sum);
        dp[q][j] = a.silu ? gate_gradient<TR>(sum, v.get(j)) : v.get(j);
      }
    }
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
      float d[V];
#pragma unroll
      for (int j = 0; j < V; ++j) d[j] = 0.f;
#pragma unroll
      for (int q = 0; q <= i; ++q)
        if (q < len) {
#pragma unroll
          for (int j = 0; j < V; ++j) d[j] = fmaf(w[i - q][j], dp[q][j], d[j]);
        }
      if (a.dw_end && i >= len) {               // a window's row that is still in the window at the end
        Values<TR, V> e;
        e.load(static_cast<const T*>(a.dw_end) + (s * (W - 1) + i - len) * a.dim + col, valid);
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] += e.get(j);
      }
      Values<TR, V> o;
      o.put(d);
      o.store(static_cast<T*>(a.dw_in) + (s * (W - 1) + i) * a.dim + col, valid);
    }
    return;
  }
  float dw[W][V], db[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    db[j] = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) dw[i][j] = 0.f;
  }
  int64_t t = (group * WAVES + wave) * a.run;
  const int64_t end = min(a.n_rows, t + a.run);
  while (t < end) {
    const Piece p = piece_at(a, t, end);
    const int64_t stop = min(end, p.hi);
    if (p.seq < 0) {
      Values<TR, V> zero;
      zero.clear();
      for (; t < stop; ++t) zero.store(static_cast<T*>(a.dx) + t * a.dx_row + col, valid);
      continue;
    }
    // x: rows u - (W - 1) on; dp: the same rows
    float x[W - 1 + UP][V], dp[W - 1 + UP][V];
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
      Values<TR, V> v;
      load_back<TR, W, V>(v, a, p, t - (W - 1) + i, col, valid);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        x[i][j] = v.get(j);
        dp[i][j] = 0.f;
      }
    }
    for (int64_t u = t; u < stop + W - 1; u += UP) {
      Values<TR, V> vx[UP], vy[UP];
#pragma unroll
      for (int r = 0; r < UP; ++r) {
        vx[r].clear();
        vy[r].clear();
        if (u + r < min(p.hi, stop + W - 1)) {
          vx[r].load(static_cast<const T*>(a.x) + (u + r) * a.x_row + col, valid);
          vy[r].load(static_cast<const T*>(a.dy) + (u + r) * a.dy_row + col, valid);
        }
      }
#pragma unroll
      for (int r = 0; r < UP; ++r) {
        const bool there = u + r < p.hi, mine = u + r < stop;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          x[W - 1 + r][j] = vx[r].get(j);
          float d = vy[r].get(j);
          if (a.silu) {
            float s = b[j];
#pragma unroll
            for (int i = 0; i < W; ++i) s = fmaf(w[i][j], x[r + i][j], s);
            d = gate_gradient<TR>(s, d);
          }
          dp[W - 1 + r][j] = there ? d : 0.f;
        }
        if (mine) {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            db[j] += dp[W - 1 + r][j];
#pragma unroll
            for (int i = 0; i < W; ++i) dw[i][j] = fmaf(dp[W - 1 + r][j], x[r + i][j], dw[i][j]);
          }
        }
        const int64_t row = u + r - (W - 1);    // dx of this one is complete
        if (row >= t && row < stop) {
          float d[V];
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < W; ++k) s = fmaf(w[W - 1 - k][j], dp[r + k][j], s);
            d[j] = s;
          }
          if (row + W > p.hi) {                 // (a tap without a row behind it adds nothing, whatever the tap is)
#pragma unroll
            for (int j = 0; j < V; ++j) d[j] = w[W - 1][j] * dp[r][j];
#pragma unroll
            for (int k = 1; k < W; ++k)
              if (row + k < p.hi) {
#pragma unroll
                for (int j = 0; j < V; ++j) d[j] = fmaf(w[W - 1 - k][j], dp[r + k][j], d[j]);
              }
            if (a.dw_end) {
              Values<TR, V> e;
              e.load(static_cast<const T*>(a.dw_end) + ((int64_t)p.seq * (W - 1) + row - (p.hi - (W - 1))) * a.dim + col, valid);
#pragma unroll
              for (int j = 0; j < V; ++j) d[j] += e.get(j);
            }
          }
          Values<TR, V> o;
          o.put(d);
          o.store(static_cast<T*>(a.dx) + row * a.dx_row + col, valid);
        }
      }
#pragma unroll
      for (int i = 0; i < W - 1; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          x[i][j] = x[UP + i][j];
          dp[i][j] = dp[UP + i][j];
        }
    }
    t = stop;
  }
  // the workgroup's waves in their order
  if (wave > 0) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
#pragma unroll
      for (int i = 0; i < W; ++i) red[wave - 1][i][lane * V + j] = dw[i][j];
      red[wave - 1][W][lane * V + j] = db[j];
    }
  }
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int i = 0; i <= W; ++i) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float s = i < W ? dw[i < W ? i : 0][j] : db[j];
        for (int k = 0; k < WAVES - 1; ++k) s += red[k][i][lane * V + j];
        if (j < valid) a.sums[(group * (W + 1) + i) * a.dim + col + j] = s;
      }
    }
  }
}

// dw and db from the workgroups' sums, in their order: 64 channels a workgroup, each wave a part of the sums of one tap.  (5 us for 130 workgroups' sums of
// 2048 channels: the start of a launch and one wait for memory.)
constexpr int SUM_WAVES = 8;
template <class TR>
__global__ __launch_bounds__(64 * SUM_WAVES) void k_conv_sums(const float* sums, int64_t n, int width, int dim, typename TR::T* dw, typename TR::T* db) {
  __shared__ float part[SUM_WAVES][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int c = blockIdx.x * 64 + lane, i = blockIdx.y;
  const int64_t each = (n + SUM_WAVES - 1) / SUM_WAVES, to = min(n, (wave + 1) * each);
  float s = 0.f;
  if (c < dim)
#pragma unroll 8
    for (int64_t k = wave * each; k < to; ++k) s += sums[(k * (width + 1) + i) * dim + c];
  part[wave][lane] = s;
  __syncthreads();
  if (wave || c >= dim) return;
  s = part[0][lane];
#pragma unroll
  for (int k = 1; k < SUM_WAVES; ++k) s += part[k][lane];
  if (i < width) dw[(int64_t)c * width + i] = TR::put(s);
  else if (db) db[c] = TR::put(s);
}

struct ConvStepArgs {
  const void* x;
  void *y, *window;
  int64_t x_row, y_row;
  const void *weight, *bias;
  const int32_t* slots;
  int n_windows, dim, silu, col_blocks;
};

// One launch, every value on its own lane.  (256 requests, 4096 channels, bfloat16: 13.3 us a call, one request 12.8: the call's host side.)
template <class TR, int W, int V>
__global__ __launch_bounds__(THREADS) void k_short_conv_step(const ConvStepArgs a) {
  typedef typename TR::T T;
  const int64_t row = blockIdx.x / a.col_blocks;
  const int col = ((int)(blockIdx.x % a.col_blocks) * THREADS + threadIdx.x) * V, valid = a.dim - col;
  if (valid <= 0) return;
  const int64_t slot = a.slots ? a.slots[row] : row;
  T* y = static_cast<T*>(a.y) + row * a.y_row + col;
  Values<TR, V> v[W], o;
  if (slot < 0 || slot >= a.n_windows) {
    o.clear();
    o.store(y, valid);
    return;
  }
  T* window = static_cast<T*>(a.window) + slot * (W - 1) * a.dim + col;
#pragma unroll
  for (int i = 0; i < W - 1; ++i) v[i].load(window + (int64_t)i * a.dim, valid);
  v[W - 1].load(static_cast<const T*>(a.x) + row * a.x_row + col, valid);
  float p[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    p[j] = a.bias && j < valid ? TR::get(static_cast<const T*>(a.bias)[col + j]) : 0.f;
    if (j < valid)
#pragma unroll
      for (int i = 0; i < W; ++i) p[j] = fmaf(TR::get(static_cast<const T*>(a.weight)[(int64_t)(col + j) * W + i]), v[i].get(j), p[j]);
    if (a.silu) p[j] = gate<TR>(p[j]);
  }
  o.put(p);
  o.store(y, valid);
#pragma unroll
  for (int i = 0; i < W - 1; ++i) v[i + 1].store(window + (int64_t)i * a.dim, valid);
}

// ---- host --------------------------------------------------------------------------------------------------------------
int check(const nugpr_short_conv* p) {
  if (!p) return invalid("problem is null");
  if (p->dtype != NUGPR_FLOAT32 && p->dtype != NUGPR_BFLOAT16) return invalid("dtype must be NUGPR_FLOAT32 or NUGPR_BFLOAT16");
  if (p->dim < 1 || p->dim > 65536) return invalid("dim must be 1..65536");
  if (p->width < 1 || p->width > MAX_WIDTH) return invalid("width must be 1..8");
  if (p->n_rows < 0 || p->n_rows > (int64_t)1 << 40) return invalid("n_rows must be 0..2^40");
  if (p->n_seqs < 0) return invalid("n_seqs must be >= 0");
  return NUGPR_OK;
}

size_t value_size(const nugpr_short_conv* p) { return p->dtype == NUGPR_BFLOAT16 ? 2 : 4; }

int check_pointer(const void* x, const char* name, size_t value, bool needed) {
  if (!x && needed) return invalid(std::string(name) + " is null");
  if (reinterpret_cast<uintptr_t>(x) % value) return invalid(std::string(name) + " misaligned");
  return NUGPR_OK;
}

// Channels of a lane: 16 bytes forward, four in the gradients, whose windows, weights and sums have to stay in registers.
int channels_of(const nugpr_short_conv* p, bool backward) { return backward || p->dtype == NUGPR_FLOAT32 ? 4 : 8; }
int64_t blocks_of(const nugpr_short_conv* p, bool backward) { return (p->dim + 64 * channels_of(p, backward) - 1) / (64 * channels_of(p, backward)); }

// Rows of a wave, eight or more, so many that the workgroups are two for each compute unit, four in the gradients, or somewhat fewer: a few more of
// them than there is room for take a turn of their own (22980 rows, 1408 channels, float32: 71 us in 540 workgroups, 61 in 510).  16384 rows, 4096 channels,
// bfloat16: 55, 58, 67 us with two, four, eight; gradients, 2048 channels: 68, 55, 66.
int64_t run_of(const nugpr_short_conv* p, bool backward) {
  const int64_t along = std::max<int64_t>(1, COMPUTE_UNITS * (backward ? 4 : 2) / blocks_of(p, backward));
  return std::max<int64_t>(8, (p->n_rows + along * WAVES - 1) / (along * WAVES));
}

int64_t groups_of(const nugpr_short_conv* p, bool backward) {
  const int64_t rows = WAVES * run_of(p, backward);
  return (p->n_rows + rows - 1) / rows;
}

size_t sums_bytes(const nugpr_short_conv* p) {
  return ((size_t)groups_of(p, true) * (p->width + 1) * p->dim * sizeof(float) + 255) / 256 * 256;
}

template <class TR, int V, class F>
void with_width(int width, F f) {
  switch (width) {
    case 1: f(std::integral_constant<int, 1>()); break;
    case 2: f(std::integral_constant<int, 2>()); break;
    case 3: f(std::integral_constant<int, 3>()); break;
    case 4: f(std::integral_constant<int, 4>()); break;
    case 5: f(std::integral_constant<int, 5>()); break;
    case 6: f(std::integral_constant<int, 6>()); break;
    case 7: f(std::integral_constant<int, 7>()); break;
    default: f(std::integral_constant<int, 8>()); break;
  }
}

// What both calls over sequences share; the grid's workgroups, behind those of the rows one for every four windows that are written.
int conv_args(const nugpr_short_conv* p, bool backward, bool windows, ConvArgs& a, int64_t& grid) {
  a.weight = p->weight; a.bias = p->bias; a.off = p->seq_offsets; a.n_rows = p->n_rows; a.n_seqs = p->n_seqs;
  a.dim = p->dim; a.silu = p->silu != 0; a.run = run_of(p, backward);
  a.col_blocks = (int)blocks_of(p, backward);
  a.runs = groups_of(p, backward);
  grid = (a.runs + (windows ? ((int64_t)p->n_seqs + WAVES - 1) / WAVES : 0)) * a.col_blocks;
  // (the threads of a launch are counted in 32 bits)
  if (grid > (int64_t)0xffffffff / THREADS) return invalid("too many rows, sequences and channels for one call");
  return NUGPR_OK;
}

}  // namespace

}  // namespace nugpr

using namespace nugpr;

extern "C" {

size_t nugpr_short_conv_workspace_bytes(const nugpr_short_conv* p) {
  if (check(p) != NUGPR_OK) return 0;
  return 256 + sums_bytes(p);
}

int nugpr_short_conv_forward(const nugpr_short_conv* p, const nugpr_rows* x, const void* initial_window, const nugpr_rows* y,
                             void* final_window, void* stream) {
  NUGPR_TRY(check(p));
  if (p->n_rows == 0 && p->n_seqs == 0) return NUGPR_OK;
  const size_t z = value_size(p);
  if (p->n_rows > 0) {
    NUGPR_TRY(check_rows(x, "x", z));
    NUGPR_TRY(check_rows(y, "y", z));
  }
  if (!p->seq_offsets) return invalid("seq_offsets is null");
  NUGPR_TRY(check_pointer(p->weight, "weight", z, true));
  NUGPR_TRY(check_pointer(p->bias, "bias", z, false));
  NUGPR_TRY(check_pointer(initial_window, "initial_window", z, false));
  NUGPR_TRY(check_pointer(final_window, "final_window", z, false));
  if (overlap(initial_window, final_window, (size_t)p->n_seqs * (p->width - 1) * p->dim * z)) return invalid("final_window overlaps initial_window");
  ConvArgs a{};
  int64_t grid;
  const bool windows = final_window && p->width > 1;
  NUGPR_TRY(conv_args(p, false, windows, a, grid));
  if (p->n_rows > 0) { a.x = x->data; a.x_row = x->row_stride; a.y = y->data; a.y_row = y->row_stride; }
  a.w_in = initial_window; a.w_out = final_window;
  if (grid == 0) return NUGPR_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const dim3 blocks((unsigned)grid), threads(THREADS);
  if (p->dtype == NUGPR_BFLOAT16)
    with_width<Bf16, 8>(p->width, [&](auto w) { hipLaunchKernelGGL((k_short_conv<Bf16, decltype(w)::value, 8>), blocks, threads, 0, s, a); });
  else
    with_width<F32, 4>(p->width, [&](auto w) { hipLaunchKernelGGL((k_short_conv<F32, decltype(w)::value, 4>), blocks, threads, 0, s, a); });
  NUGPR_HIP(hipGetLastError());
  return NUGPR_OK;
}

int nugpr_short_conv_backward(const nugpr_short_conv* p, const nugpr_rows* x, const void* initial_window, const nugpr_rows* d_y,
                              const void* d_final_window, const nugpr_rows* dx, void* dweight, void* dbias, void* d_initial_window,
                              void* stream) {
  NUGPR_TRY(check(p));
  const size_t z = value_size(p), windows = (size_t)p->n_seqs * (p->width - 1) * p->dim * z;
  if (p->n_rows > 0) {
    NUGPR_TRY(check_rows(x, "x", z));
    NUGPR_TRY(check_rows(d_y, "d_y", z));
    NUGPR_TRY(check_rows(dx, "dx", z));
  }
  if ((p->n_rows > 0 || p->n_seqs > 0) && !p->seq_offsets) return invalid("seq_offsets is null");
  NUGPR_TRY(check_pointer(p->weight, "weight", z, true));
  NUGPR_TRY(check_pointer(p->bias, "bias", z, false));
  NUGPR_TRY(check_pointer(dweight, "dweight", z, true));
  NUGPR_TRY(check_pointer(dbias, "dbias", z, p->bias != nullptr));
  NUGPR_TRY(check_pointer(initial_window, "initial_window", z, false));
  NUGPR_TRY(check_pointer(d_final_window, "d_final_window", z, false));
  NUGPR_TRY(check_pointer(d_initial_window, "d_initial_window", z, false));
  if (overlap(d_final_window, d_initial_window, windows)) return invalid("d_initial_window overlaps d_final_window");
  const size_t need = sums_bytes(p);
  if (need && (!p->workspace || (reinterpret_cast<uintptr_t>(p->workspace) & 255u))) { set_error("workspace is null or not 256-byte aligned"); return NUGPR_ERR_WORKSPACE; }
  if (p->workspace_bytes < need) { set_error("workspace smaller than nugpr_short_conv_workspace_bytes()"); return NUGPR_ERR_WORKSPACE; }
  ConvArgs a{};
  int64_t grid;
  NUGPR_TRY(conv_args(p, true, d_initial_window && p->width > 1, a, grid));
  if (p->n_rows > 0) {
    a.x = x->data; a.x_row = x->row_stride; a.dy = d_y->data; a.dy_row = d_y->row_stride; a.dx = dx->data; a.dx_row = dx->row_stride;
  }
  a.w_in = initial_window; a.dw_end = d_final_window; a.dw_in = d_initial_window;
  a.sums = static_cast<float*>(p->workspace);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const dim3 blocks((unsigned)grid), threads(THREADS), sum_grid((unsigned)(p->dim + 63) / 64, p->width + 1), sum_threads(64 * SUM_WAVES);
  if (p->dtype == NUGPR_BFLOAT16) {
    if (grid) with_width<Bf16, 4>(p->width, [&](auto w) { hipLaunchKernelGGL((k_short_conv_backward<Bf16, decltype(w)::value, 4>), blocks, threads, 0, s, a); });
    hipLaunchKernelGGL(k_conv_sums<Bf16>, sum_grid, sum_threads, 0, s, a.sums, a.runs, p->width, p->dim, static_cast<uint16_t*>(dweight), static_cast<uint16_t*>(dbias));
  } else {
    if (grid) with_width<F32, 4>(p->width, [&](auto w) { hipLaunchKernelGGL((k_short_conv_backward<F32, decltype(w)::value, 4>), blocks, threads, 0, s, a); });
    hipLaunchKernelGGL(k_conv_sums<F32>, sum_grid, sum_threads, 0, s, a.sums, a.runs, p->width, p->dim, static_cast<float*>(dweight), static_cast<float*>(dbias));
  }
  NUGPR_HIP(hipGetLastError());
  return NUGPR_OK;
}

int nugpr_short_conv_step(const nugpr_short_conv* p, const nugpr_rows* x, void* window, const int32_t* slots, const nugpr_rows* y,
                          void* stream) {
  NUGPR_TRY(check(p));
  if (p->n_rows == 0) return NUGPR_OK;
  const size_t z = value_size(p);
  NUGPR_TRY(check_rows(x, "x", z));
  NUGPR_TRY(check_rows(y, "y", z));
  NUGPR_TRY(check_pointer(p->weight, "weight", z, true));
  NUGPR_TRY(check_pointer(p->bias, "bias", z, false));
  NUGPR_TRY(check_pointer(window, "window", z, p->n_seqs > 0 && p->width > 1));
  if (!slots && p->n_rows > p->n_seqs) return invalid("more requests than windows");
  ConvStepArgs a{};
  a.x = x->data; a.x_row = x->row_stride; a.y = y->data; a.y_row = y->row_stride; a.window = window;
  a.weight = p->weight; a.bias = p->bias; a.slots = slots; a.n_windows = p->n_seqs; a.dim = p->dim; a.silu = p->silu != 0;
  constexpr int V = 2;                          // (few values a lane: a single request is spread over more of the card)
  a.col_blocks = (p->dim + V * THREADS - 1) / (V * THREADS);
  const int64_t grid = p->n_rows * a.col_blocks;
  if (grid > (int64_t)0xffffffff / THREADS) return invalid("too many requests and channels for one call");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const dim3 blocks((unsigned)grid), threads(THREADS);
  if (p->dtype == NUGPR_BFLOAT16)
    with_width<Bf16, V>(p->width, [&](auto w) { hipLaunchKernelGGL((k_short_conv_step<Bf16, decltype(w)::value, V>), blocks, threads, 0, s, a); });
  else
    with_width<F32, V>(p->width, [&](auto w) { hipLaunchKernelGGL((k_short_conv_step<F32, decltype(w)::value, V>), blocks, threads, 0, s, a); });
  NUGPR_HIP(hipGetLastError());
  return NUGPR_OK;
}

}  // extern "C"
