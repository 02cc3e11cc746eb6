// Linear attention with a decay for each head, over packed sequences: forward, gradients, and one token at a time.
//
//   S_t = lam S_{t-1} + k_t v_t^T,   o_t = scale q_t S_t
//
// In blocks of C rows with start state S the same is
//   o_t = lam^{t+1} q_t S + sum_{s <= t} lam^{t-s} (q_t . k_s) v_s,     S' = lam^C S + sum_s lam^{C-1-s} k_s v_s^T,
// all matrix products.  The gradients are scans of the same kind, with the roles exchanged (U_t: gradient by S_t)
//   dq_t = scale S_t do_t                      scan over (q, k, v) := (do, v, k)
//   dk_t = U_t v_t                             backwards in time over (v, do, q)
//   dv_t = U_t^T k_t                           backwards in time over (k, q, do)
//   U_t = lam U_{t+1} + scale q_t do_t^T,  dS_0 = lam U_1
// so that one kernel serves all four: backwards, rows are read from the end and the state takes its decay before it is
// read instead of after (exponents one less in o, one more in S').
#include <cmath>

#include "matrix_core.h"
#include "nugpr_internal.h"
#include "packed_rows.h"

namespace nugpr {

namespace {

constexpr int THREADS = 256;
constexpr float LOWEST_LOG = -1e4f;   // lam^0 = 1, any other power zero: log_decay = -infinity

// One scan: what plays the parts of q, k, v and o (values per row and head), and its states.
struct ScanRole {
  const void *q, *k, *v;
  void* o;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
  const float* s_in;      // start states of the sequences, or null
  float* s_out;           // end states, or null
  float* spans;           // start state of every span of a sequence that has several (between: what the span adds)
  float wscale, oscale;   // of k_s v_s^T, of o
  int gq, gk;             // heads of q and o, of k and v, that share one state (one of the two is 1)
  int dk, dv;
  int back;               // against time
  int s_trans;            // states are stored dv x dk
};

struct ScanArgs {
  ScanRole role[3];       // (first, see k_decay_scan)
  const int64_t* off;
  const float* log_decay;
  int64_t n_rows;
  int n_seqs, kv;
  int span_log2;          // rows of a span
  int items;              // spans that there may be
};

__device__ float log_of(const float* log_decay, int h) {
  const float g = log_decay[h];
  return g < LOWEST_LOG ? LOWEST_LOG : g;     // NaN stays
}

// lam^n as the sum of two float32: the powers of a block multiply up over a long sequence
__device__ void power(float g, double n, float& hi, float& lo) {
  const double p = exp((double)g * n);
  hi = (float)p;
  lo = (float)(p - (double)hi);
}

// x lam + add, lam as the sum of two float32 (an infinite x keeps its sign beside the smaller one)
__device__ inline float decayed(float x, float hi, float lo, float add) { return fmaf(x, hi, fmaf(__builtin_isinf(x) ? 0.f : x, lo, add)); }

// (a value that all lanes have, in a scalar register)
__device__ inline double same_in_all(double x) {
  const u32x2 v = __builtin_bit_cast(u32x2, x);
  return __builtin_bit_cast(double, (u32x2{(uint32_t)__builtin_amdgcn_readfirstlane((int)v[0]), (uint32_t)__builtin_amdgcn_readfirstlane((int)v[1])}));
}

// Blocks of C rows, widths up to D.
template <class TR, int D, int C>
struct Tile {
  static constexpr int NT = 1;                              // a wave's tiles of 16 of the state's columns
  static constexpr int WAVES = D / 16 / NT;
  static constexpr int A_ROW = D / TR::E;                   // threads a row
  static constexpr int PASS = 64 * WAVES / A_ROW;           // rows that one load of all threads covers
  static constexpr int N = C / PASS;
};

// A block's rows in an array, cnt of them, as a buffer that begins at their lowest address and ends behind the last one: what lies
// beyond reads as zero and is not stored.  `at`: the thread's byte offset from row 0 of the block (place_in); `pass`, in
// bytes, is added for every further pass.  Only where AL; else everything by 64-bit pointers, value by value.
template <class TR, int D, int C>
struct Window {
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t from, pass;
  __device__ Window(const typename TR::T* base, int64_t stride, int dir, int cnt, int width) {
    constexpr int S = sizeof(typename TR::T);
    const int64_t below = dir > 0 ? 0 : (cnt - 1) * stride;
    rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<typename TR::T*>(base - below), 0, (int)(((cnt - 1) * stride + width) * S), 0x00027000);
    from = (uint32_t)below * S;
    pass = (uint32_t)(dir * Tile<TR, D, C>::PASS) * (uint32_t)stride * S;
  }
  __device__ u32x4 load(uint32_t at, int p) const {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at + (from + p * pass), 0, 0));
  }
  __device__ void store(uint32_t at, int p, u32x4 v) const { __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, at + (from + p * pass), 0, 0); }
};

template <class TR, int D, int C>
__device__ inline uint32_t place_in(int tid, int64_t stride, int dir, int width) {
  using L = Tile<TR, D, C>;
  const int col = tid % L::A_ROW * TR::E;
  // (columns beyond the width: beyond any buffer)
  return col < width ? (uint32_t)(dir * (tid / L::A_ROW)) * (uint32_t)stride * (uint32_t)sizeof(typename TR::T) + col * (uint32_t)sizeof(typename TR::T)
                     : 0x80000000u;
}

// Rows of a block, 16 bytes a thread and pass; zero from row cnt and column `width` on.
template <class TR, int D, int C, bool AL>
__device__ inline void fetch(u32x4* r, int tid, const typename TR::T* base, int64_t stride, int dir, uint32_t at, int cnt, int width) {
  using L = Tile<TR, D, C>;
  if constexpr (AL) {
    const Window<TR, D, C> w(base, stride, dir, cnt, width);
#pragma unroll
    for (int p = 0; p < L::N; ++p) r[p] = w.load(at, p);
  } else {
    const int col = (tid % L::A_ROW) * TR::E, row0 = tid / L::A_ROW;
    const typename TR::T* x = base + (int64_t)dir * row0 * stride + col;
#pragma unroll
    for (int p = 0; p < L::N; ++p, x += dir * L::PASS * stride) {
      u32x4 v = {0, 0, 0, 0};
      if (row0 + p * L::PASS < cnt && col + TR::E <= width) {
        v = load16(x);
      } else if (row0 + p * L::PASS < cnt) {
#pragma unroll
        for (int j = 0; j < TR::E; ++j)
          if (col + j < width) {
            if constexpr (TR::E == 8) v[j >> 1] |= (uint32_t)x[j] << (16 * (j & 1));
            else v[j] = __builtin_bit_cast(uint32_t, x[j]);
          }
      }
      r[p] = v;
    }
  }
}

// the block into a tile in LDS; `at`: the thread's byte offset in it for the first pass
template <class TR, int D, int C>
__device__ inline void put(typename TR::T* tile, int at, const u32x4* r) {
  using L = Tile<TR, D, C>;
  static_assert(L::PASS % 16 == 0, "rows of one thread are permuted alike");
#pragma unroll
  for (int p = 0; p < L::N; ++p)
    *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(tile) + at + p * L::PASS * D * (int)sizeof(typename TR::T)) = r[p];
}

// (ScanArgs is k_decay_scan's only argument, its roles come first)
typedef const __attribute__((address_space(4))) ScanRole* RolePtr;

// A workgroup's span.
struct Span {
  int seq;                  // < 0: there is none
  int64_t lo, len, from;    // rows of the sequence; the span's first one, counted along the scan
};
__device__ inline Span span_of(const ScanArgs& a, int item) {
  const PieceOf piece = piece_of(a.off, a.n_seqs, a.n_rows, a.span_log2, item);
  return Span{piece.seq, piece.lo, piece.hi - piece.lo, (int64_t)(item - ((piece.lo >> a.span_log2) + piece.seq)) << a.span_log2};
}

// Where the state of a span comes from and goes to, or null.
template <bool WALK>
__device__ inline const float* start_of(const ScanArgs& a, RolePtr ro, const Span& sp, int item, int h) {
  if (!WALK) return nullptr;
  const int64_t size = (int64_t)ro->dk * ro->dv;
  if (sp.len > (int64_t)1 << a.span_log2) return ro->spans + ((int64_t)item * a.kv + h) * size;
  return ro->s_in ? ro->s_in + ((int64_t)sp.seq * a.kv + h) * size : nullptr;
}
template <bool WALK>
__device__ inline float* end_of(const ScanArgs& a, RolePtr ro, const Span& sp, int item, int h) {
  const int64_t size = (int64_t)ro->dk * ro->dv;
  if (!WALK) return ro->spans + ((int64_t)item * a.kv + h) * size;
  return sp.from + ((int64_t)1 << a.span_log2) >= sp.len && ro->s_out ? ro->s_out + ((int64_t)sp.seq * a.kv + h) * size : nullptr;
}

// N values of a row that has `left` more; zero past its end.
template <class TR, int N>
__device__ inline void row_part(const typename TR::T* row, int left, float (&v)[N]) {
  constexpr int E = TR::E;
  static_assert(N % E == 0, "");
#pragma unroll
  for (int c = 0; c < N / E; ++c) {
    typename TR::T part[E] = {};
    if (c * E + E <= left) {
      const u32x4 x = load16(row + c * E);
      __builtin_memcpy(part, &x, 16);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (c * E + j < left) part[j] = row[c * E + j];
    }
#pragma unroll
    for (int j = 0; j < E; ++j) v[c * E + j] = TR::get(part[j]);
  }
}

// A workgroup's span for the rare ways that find it anew.
template <class TR, bool WALK, bool SUM>
struct SpanRows {
  using T = typename TR::T;
  RolePtr ro;
  Span sp;
  int h, item, n_tok, dir, gq, gk;
  int64_t first;
  __device__ SpanRows(const ScanArgs& a, RolePtr ro, int block) : ro(ro), sp(span_of(a, block / a.kv)), h(block % a.kv), item(block / a.kv) {
    n_tok = (int)min((int64_t)1 << a.span_log2, sp.len - sp.from);
    dir = ro->back ? -1 : 1;
    gq = WALK ? ro->gq : 0;
    gk = SUM ? ro->gk : 1;
    first = ro->back ? sp.lo + sp.len - 1 - sp.from : sp.lo + sp.from;
  }
  __device__ const T* q(int t, int m) const { return static_cast<const T*>(ro->q) + (first + (int64_t)dir * t) * ro->q_row + ((int64_t)h * ro->gq + m) * ro->q_head; }
  __device__ const T* k(int t, int m) const { return static_cast<const T*>(ro->k) + (first + (int64_t)dir * t) * ro->k_row + ((int64_t)h * ro->gk + m) * ro->k_head; }
  __device__ const T* v(int t, int m) const { return static_cast<const T*>(ro->v) + (first + (int64_t)dir * t) * ro->v_row + ((int64_t)h * ro->gk + m) * ro->v_head; }
  __device__ T* o(int t, int m) const { return static_cast<T*>(ro->o) + (first + (int64_t)dir * t) * ro->o_row + ((int64_t)h * ro->gq + m) * ro->o_head; }
};

// What makes a span's results not finite.  MUST: something that they may be wrong for: an infinity among the rows or in the start state, or, where o
// is written, a NaN in a column of v whose state was none before.  HAS_NAN: any other NaN, which goes where it belongs.  A thread's share; the span has what one
// thread has.
constexpr int MUST = 2, HAS_NAN = 1;
template <class TR, int D, bool WALK, bool SUM>
__device__ inline int needs_tokens(const ScanArgs& a, RolePtr ro, int tid, int block) {
  const SpanRows<TR, WALK, SUM> rows(a, ro, block);
  constexpr int E = TR::E, A_ROW = D / E;
  const int col = tid % A_ROW * E, s_c = ro->s_trans ? ro->dk : 1;
  const float* from = start_of<WALK>(a, ro, rows.sp, rows.item, rows.h);
  int found = 0;
  bool was[E];                         // (v makes a column of the state NaN, or none of it)
#pragma unroll
  for (int j = 0; j < E; ++j) was[j] = !WALK || (from && col + j < ro->dv && __builtin_isnan(from[(col + j) * s_c]));
#pragma unroll 1
  for (int t = tid / A_ROW; t < rows.n_tok; t += blockDim.x / A_ROW) {
    float x[E];
#pragma unroll 1
    for (int m = 0; m < rows.gk; ++m) {
      row_part<TR>(rows.k(t, m) + col, ro->dk - col, x);
#pragma unroll
      for (int j = 0; j < E; ++j) found |= __builtin_isinf(x[j]) ? MUST : __builtin_isnan(x[j]) ? HAS_NAN : 0;
      row_part<TR>(rows.v(t, m) + col, ro->dv - col, x);
#pragma unroll
      for (int j = 0; j < E; ++j) found |= __builtin_isinf(x[j]) || (__builtin_isnan(x[j]) && !was[j]) ? MUST : __builtin_isnan(x[j]) ? HAS_NAN : 0;
    }
#pragma unroll 1
    for (int m = 0; m < rows.gq; ++m) {
      row_part<TR>(rows.q(t, m) + col, ro->dk - col, x);
#pragma unroll
      for (int j = 0; j < E; ++j) found |= __builtin_isinf(x[j]) ? MUST : __builtin_isnan(x[j]) ? HAS_NAN : 0;
    }
  }
  if (from)
    for (int e = tid; e < ro->dk * ro->dv; e += blockDim.x) found |= __builtin_isinf(from[e]) ? MUST : __builtin_isnan(from[e]) ? HAS_NAN : 0;
  return found;
}

// A span by the recurrence itself, token by token in float32, without LDS or barriers: a wave has 16 columns of the state, a lane D / 4 rows
// of one of them.  The wait for a row's loads bounds it, about a microsecond each: 65536 rows, 16 / 4 heads of 128, bfloat16, with one infinity:
// 2.7 ms instead of 0.25.
template <class TR, int D, bool WALK, bool SUM>
__device__ inline void walk_tokens(const ScanArgs& a, RolePtr ro, int tid, int block) {
  constexpr int EACH = D / 4;
  const SpanRows<TR, WALK, SUM> span(a, ro, block);
  const float g = log_of(a.log_decay, span.h);
  const int col = tid / 64 * 16 + (tid & 15), e = ro->back, dk = ro->dk, n_tok = span.n_tok, gq = span.gq, gk = span.gk;
  const bool live = col < ro->dv;
  const int s_r = ro->s_trans ? 1 : ro->dv, s_c = ro->s_trans ? dk : 1;
  const float* from = start_of<WALK>(a, ro, span.sp, span.item, span.h);
  float* to = end_of<WALK>(a, ro, span.sp, span.item, span.h);
  const int row0 = (tid >> 4 & 3) * EACH;
  int rows = dk - row0;
  float S[EACH], lam_hi, lam_lo;
  power(g, 1.0, lam_hi, lam_lo);
#pragma unroll
  for (int x = 0; x < EACH; ++x) S[x] = from && live && x < rows ? from[(row0 + x) * s_r + col * s_c] : 0.f;
#pragma unroll 1
  for (int t = 0; t < n_tok; ++t) {
    asm volatile("" : "+v"(rows));                         // (which rows there are is not kept ready, lane by lane)
    if (!e)
#pragma unroll
      for (int x = 0; x < EACH; ++x) S[x] = decayed(S[x], lam_hi, lam_lo, 0.f);
#pragma unroll 1
    for (int m = 0; m < gk; ++m) {
      float k[EACH];
      row_part<TR>(span.k(t, m) + row0, rows, k);
      const float v = live ? ro->wscale * TR::get(span.v(t, m)[col]) : 0.f;
#pragma unroll
      for (int x = 0; x < EACH; ++x) S[x] = fmaf(k[x], v, S[x]);
    }
#pragma unroll 1
    for (int m = 0; m < gq; ++m) {
      float q[EACH], o = 0.f;
      row_part<TR>(span.q(t, m) + row0, rows, q);
#pragma unroll
      for (int x = 0; x < EACH; ++x) o = x < rows ? fmaf(q[x], S[x], o) : o;      // (rows beyond the width may hold zero times an infinity)
      o += __shfl_xor(o, 16);
      o += __shfl_xor(o, 32);
      if (live && row0 == 0) span.o(t, m)[col] = TR::put(ro->oscale * o);
    }
    if (e)
#pragma unroll
      for (int x = 0; x < EACH; ++x) S[x] = decayed(S[x], lam_hi, lam_lo, 0.f);
  }
  if (to && live)
#pragma unroll
    for (int x = 0; x < EACH; ++x)
      if (x < rows) to[(row0 + x) * s_r + col * s_c] = S[x];
}

// One workgroup walks one span of one sequence and key / value head in blocks of C rows; the state stays in accumulator
// registers, 16 of its columns a wave.  WALK: writes o from given start states; else: what the span adds to
// the state, for k_span_join.  SUM: some role's o is a sum over heads of k and v (gk > 1).
// Per block and head: P^T = K Q^T (each wave tiles of 16 rows of Q), masked and decayed, goes through LDS; o^T = S^T Q^T and V^T P^T with
// the wave's columns of S and V; S += K^T (w V).  S is read as an operand where it lies (matrix_core.h).  In bfloat16 P and
// S are each read as two bfloat16, 17 bits of them: no more than the float32 sums' own error, so that o is rounded once.  (With one bfloat16 of
// each o had 1.4 times the error of its last rounding; it took 217 us instead of 250 for 65536 rows, 16 / 4 heads of 128, 197 instead of 220 for the
// gradients of 16 x 1024 rows, 16 heads.)  w V, which is summed into the float32 state, keeps all 24 bits.
// Values that are not finite: rows s > t must not touch o_t, but 0 x NaN in the masked part of P would, nor may an infinity meet the
// zeros beside a width or the difference of two infinities between the parts of a factor, as where a product leaves float32's range.  So a span
// whose results are not all finite is looked through for what made them so (needs_tokens) and, if need be, walked once more (walk_tokens).
// What bounds it: in bfloat16 the way of the rows together with the work between (of 65536 rows, 16 / 4 heads of 128: vector pipe 45 % of the
// time, LDS 40 %, matrix cores 27 %); in float32 the waits of a block's steps, which few waves hide (matrix cores busy a third of the time, LDS 13 %,
// waves waiting 36 % of it); the length of the chain where there are few rows.
// Measured under the profiler, median and least: those 65536 rows: 247 and 202 us to walk (671 MB, 2.7 and 3.3 TB/s) after 47 and 40 to add
// up; 16 x 1024 rows, 16 heads, gradients: 230 and 211 (three roles, 805 MB, 3.5 and 3.8 TB/s); 20011 rows, 8 heads of 64, float32: 62 after 26.
// 128 registers a lane do not hold it all for widths beyond 64: in float32 the walks spill 17 to 50 of them, in bfloat16 none to 11.
template <class TR, int D, int C, bool AL, bool WALK, bool SUM>
__global__ __launch_bounds__((64 * Tile<TR, D, C>::WAVES), 4) void k_decay_scan(const ScanArgs a) {
  using T = typename TR::T;
  using Frag = typename TR::Frag;
  using L = Tile<TR, D, C>;
  constexpr int KS = TR::KS, KT = KS / 16;       // accumulator tiles of a contraction step
  constexpr bool LOOK = TR::E == 4;              // steps of the contraction beyond the width, and waves beyond the columns, are left out (in
                                                 // bfloat16 the products are not what bounds the time, and the looks cost registers)
  constexpr int NT = L::NT, THREADS = 64 * L::WAVES;
  constexpr int SHARE = L::WAVES / (C / 16);      // waves that share 16 rows of Q in K Q^T
  constexpr int EACH = SHARE < C / 16 ? C / 16 / SHARE : 1;     // tiles of rows of K for each of them
  constexpr int PLD = C + (TR::E == 8 ? 8 : 4);
  __shared__ __align__(16) T sK[C * D];
  __shared__ __align__(16) T sV[C * D];
  __shared__ __align__(16) T sQ[WALK ? C * D : 8];
  __shared__ __align__(16) T sP[WALK ? TR::SPLIT * C * PLD : 8];
  __shared__ __align__(16) float sLam[2 * C + 4];    // lam^n at C + n; zero before C
  __shared__ __align__(16) float sPw[WALK ? 2 * C + 4 : 4];    // the same, as P is multiplied by it
  __shared__ __align__(16) float sW[C];          // weights of the block's rows in the state

  // The role's numbers are read from the arguments where they are needed: kept over the loop they would not fit the scalar registers.
  RolePtr ro = (RolePtr)((const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr() + blockIdx.y * sizeof(ScanRole));
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int i = tid & 15, kg = (tid >> 4) & 3;
  const int h = blockIdx.x % a.kv, item = blockIdx.x / a.kv;

  if (WALK && item == a.items) {                 // rows that no sequence owns (one workgroup a head: for few of them; half of 65536 rows, 16 heads of 128: 9 ms)
    const int64_t lo = clamped(a.off[0], 0, a.n_rows), hi = clamped(a.off[a.n_seqs], lo, a.n_rows);
    const int64_t none = lo + a.n_rows - hi, per = (int64_t)ro->gq * ro->dv;
    for (int64_t e = tid; e < none * per; e += THREADS) {
      const int64_t r = e / per;
      const int c = (int)(e - r * per);
      static_cast<T*>(ro->o)[(r < lo ? r : r - lo + hi) * ro->o_row + (int64_t)(h * ro->gq + c / ro->dv) * ro->o_head + c % ro->dv] = TR::put(0.f);
    }
    return;
  }
  const float g = log_of(a.log_decay, h);
  const Span sp = span_of(a, item);
  if (sp.seq < 0) return;
  const int64_t len = sp.len, span = (int64_t)1 << a.span_log2, c0 = sp.from;
  const bool last = c0 + span >= len;
  if (c0 > 0 && c0 >= len) return;
  if (!WALK && last) return;
  const int n_tok = (int)min(span, len - c0);
  const int e = ro->back;

  // the first loads are on their way while the rest is made ready
  const int gq = WALK ? ro->gq : 1, gk = SUM ? ro->gk : 1, heads = max(gq, gk);
  const int blocks = (n_tok + C - 1) / C;
  const int64_t first = e ? sp.lo + len - 1 - c0 : sp.lo + c0;
  const int dir = e ? -1 : 1;
  // row 0 of the block to load next in the arrays, and a thread's places
  const int row0 = tid / L::A_ROW, col_in = tid % L::A_ROW * TR::E;
  const T* q_at = static_cast<const T*>(ro->q) + (int64_t)h * ro->gq * ro->q_head + first * ro->q_row;
  const T* k_at = static_cast<const T*>(ro->k) + (int64_t)h * ro->gk * ro->k_head + first * ro->k_row;
  const T* v_at = static_cast<const T*>(ro->v) + (int64_t)h * ro->gk * ro->v_head + first * ro->v_row;
  T* o_at = WALK ? static_cast<T*>(ro->o) + (int64_t)h * ro->gq * ro->o_head + first * ro->o_row : nullptr;
  const uint32_t q_off = place_in<TR, D, C>(tid, ro->q_row, dir, ro->dk), k_off = place_in<TR, D, C>(tid, ro->k_row, dir, ro->dk),
                 v_off = place_in<TR, D, C>(tid, ro->v_row, dir, ro->dv), o_off = place_in<TR, D, C>(tid, ro->o_row, dir, ro->dv);
  u32x4 rq[WALK ? L::N : 1], rk[L::N], rv[L::N];
  auto fetch_block = [&](int b, int m) {
    const int cnt = min(C, n_tok - b * C);
    if (gk > 1 || m == 0) {
      fetch<TR, D, C, AL>(rk, tid, k_at + m * ro->k_head, ro->k_row, dir, k_off, cnt, ro->dk);
      fetch<TR, D, C, AL>(rv, tid, v_at + m * ro->v_head, ro->v_row, dir, v_off, cnt, ro->dv);
    }
    if constexpr (WALK)
      if (gq > 1 || m == 0) fetch<TR, D, C, AL>(rq, tid, q_at + m * ro->q_head, ro->q_row, dir, q_off, cnt, ro->dk);
    if (m + 1 == heads) {
      k_at += dir * C * ro->k_row;
      v_at += dir * C * ro->v_row;
      if constexpr (WALK) q_at += dir * C * ro->q_row;
    }
  };
  if (blocks > 0) fetch_block(0, 0);

  for (int n = tid; n <= 2 * C; n += THREADS) {
    sLam[n] = n < C ? 0.f : (float)exp((double)g * (n - C));
    if (WALK) sPw[n] = ro->wscale * ro->oscale * sLam[n];
  }
  // lam^C in every block is rounded so that the product of them all stays within a rounding of its exact value: a block's
  // rounding error would otherwise add up over the hundreds of blocks that a slowly decaying state remembers
  const double lam_block = same_in_all(exp((double)g * C)), lam_inv = same_in_all(lam_block > 1e-30 ? 1.0 / lam_block : 0.0);
  double drift = 1.0;

  // the state: rows acc_row(m, kg) .., columns col0 + 16 n + i
  f32x4 S[D / 16][NT];
  const int col0 = wave * 16 * NT;
  const bool mine = !LOOK || col0 < ro->dv;
  const int s_r = ro->s_trans ? 1 : ro->dv, s_c = ro->s_trans ? ro->dk : 1;
  const float* from = start_of<WALK>(a, ro, sp, item, h);
  bool have = from != nullptr;
#pragma unroll
  for (int m = 0; m < D / 16; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = TR::acc_row(m, kg) + r, col = col0 + 16 * n + i;
        S[m][n][r] = have && row < ro->dk && col < ro->dv ? from[row * s_r + col * s_c] : 0.f;
      }

  float odd = 0.f;      // NaN: a result was not finite

  // and in LDS
  int put_at = TR::template unit<D>(row0, col_in), along_at = TR::template along_at<D>(i, kg);
  int v_cols[TR::ACROSS], k_cols[TR::ACROSS];
  TR::template columns_at<D>(v_cols, col0, i, kg);
  TR::template acc_columns_at<D>(k_cols, i, kg);
  f32x4 o[NT][C / 16];
  // A block's o goes into Q's tile, which nobody reads any more by then, and on to memory at the beginning of the next step, by the
  // threads that write the next rows of Q to the same places: whole lines, and ahead of that step's loads (who waits for loads
  // waits for what was stored before them, too, and would wait for the stores' way to memory right behind them).
  T* out_at = nullptr;
  int out_cnt = 0;
  auto flush = [&]() {
    const char* tile = reinterpret_cast<const char*>(sQ) + put_at;
    if constexpr (AL) {
      const Window<TR, D, C> w(out_at, ro->o_row, dir, out_cnt, ro->dv);
#pragma unroll
      for (int p = 0; p < L::N; ++p) w.store(o_off, p, *reinterpret_cast<const u32x4*>(tile + p * L::PASS * D * (int)sizeof(T)));
    } else {
      T* x = out_at + (int64_t)dir * row0 * ro->o_row + col_in;
#pragma unroll
      for (int p = 0; p < L::N; ++p, x += dir * L::PASS * ro->o_row)
        if (row0 + p * L::PASS < out_cnt && col_in + TR::E <= ro->dv) store_any(x, *reinterpret_cast<const u32x4*>(tile + p * L::PASS * D * (int)sizeof(T)));
        else if (row0 + p * L::PASS < out_cnt)
#pragma unroll
          for (int j = 0; j < TR::E; ++j)
            if (col_in + j < ro->dv) x[j] = reinterpret_cast<const T*>(tile + p * L::PASS * D * (int)sizeof(T))[j];
    }
    out_cnt = 0;
  };
  for (int b = 0; b < blocks; ++b) {
    const int cnt = min(C, n_tok - b * C);
    for (int m = 0; m < heads; ++m) {
      // (what follows from these is cheaper made anew than kept in registers from step to step)
      asm volatile("" : "+v"(i), "+v"(kg), "+v"(put_at), "+v"(along_at), "+s"(ro));
#pragma unroll
      for (int x = 0; x < TR::ACROSS; ++x) asm volatile("" : "+v"(v_cols[x]), "+v"(k_cols[x]));
      const bool kv_new = gk > 1 || m == 0, q_new = WALK && (gq > 1 || m == 0);
      __syncthreads();
      if constexpr (WALK)
        if (out_cnt > 0) flush();
      if (kv_new) {
        put<TR, D, C>(sK, put_at, rk);
        put<TR, D, C>(sV, put_at, rv);
        if (tid < C) sW[tid] = tid < cnt ? ro->wscale * sLam[C + cnt - 1 - tid + e] : 0.f;
      }
      if constexpr (WALK)
        if (q_new) put<TR, D, C>(sQ, put_at, rq);
      __syncthreads();
      if (m + 1 < heads) fetch_block(b, m + 1);
      else if (b + 1 < blocks) fetch_block(b + 1, 0);

      const bool end = gq == 1 || m + 1 == heads;          // the state moves on
      const bool keep = !WALK || b + 1 < blocks || (last && ro->s_out);
      if constexpr (WALK) {
        // P^T, rows of K x 16 rows of Q
        const int qt = wave / SHARE, t = 16 * qt + i;
        Frag qf[D / KS];
#pragma unroll
        for (int k = 0; k < D / KS; ++k) {
          if (LOOK && k * KS >= ro->dk) break;
          qf[k] = TR::template along<D>(sQ, along_at, 16 * qt, k * KS);
        }
#pragma unroll
        for (int x = 0; x < EACH; ++x) {
          const int st = wave % SHARE * EACH + x;
          if (st > (KT == 2 ? qt | 1 : qt)) break;         // (a product of 32 rows reads the masked tile too)
          f32x4 p = {0.f, 0.f, 0.f, 0.f};
          if (st <= qt) {
#pragma unroll
            for (int k = 0; k < D / KS; ++k) {
              if (LOOK && k * KS >= ro->dk) break;
              p = TR::mfma(TR::template along<D>(sK, along_at, 16 * st, k * KS), qf[k], p);
            }
            const int d = t - 16 * st - 4 * kg;            // rows apart, of the first of four
            if (st == qt) {
#pragma unroll
              for (int r = 0; r < 4; ++r) p[r] = d >= r ? p[r] * sPw[C + d - r] : 0.f;
            } else {
#pragma unroll
              for (int r = 0; r < 4; ++r) p[r] *= sPw[C + d - r];
            }
          }
          T* to = sP + t * PLD + 16 * st + 4 * kg;
          if constexpr (KT == 2) {
            const u32x2 near = {two_bf16(p[0], p[1]), two_bf16(p[2], p[3])};
            float rest[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              rest[r] = p[r] - from_two(near[r >> 1], r & 1);
              rest[r] = rest[r] == rest[r] ? rest[r] : 0.f;      // (an infinity has none)
            }
            *reinterpret_cast<u32x2*>(to) = near;
            *reinterpret_cast<u32x2*>(to + C * PLD) = u32x2{two_bf16(rest[0], rest[1]), two_bf16(rest[2], rest[3])};
          } else {
            *reinterpret_cast<f32x4*>(to) = p;
          }
        }
        // o^T = S^T Q^T, rows of the state's columns
        if (gk == 1 || m == 0) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int tt = 0; tt < C / 16; ++tt) o[n][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (have && mine) {
#pragma unroll
            for (int k = 0; k < D / KS; ++k) {
              if (LOOK && k * KS >= ro->dk) break;
              __builtin_amdgcn_sched_barrier(0);
              Frag sf[NT][TR::SPLIT];
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                f32x4 part[KT];
#pragma unroll
                for (int x = 0; x < KT; ++x) part[x] = S[k * KT + x][n];
                acc_frags(part, sf[n], TR{});
              }
#pragma unroll
              for (int tt = 0; tt < C / 16; ++tt) {
                const Frag q = TR::template along<D>(sQ, along_at, 16 * tt, k * KS);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                  for (int x = 0; x < TR::SPLIT; ++x) o[n][tt] = TR::mfma(sf[n][x], q, o[n][tt]);
              }
            }
#pragma unroll
            for (int tt = 0; tt < C / 16; ++tt) {
              const float w = ro->oscale * sLam[C + 16 * tt + i + 1 - e];
#pragma unroll
              for (int n = 0; n < NT; ++n) o[n][tt] *= w;
            }
          }
        }
      }
      // S moves on: its decay, then K^T (w V)
      if (end && keep && mine) {
        if ((have || !WALK) && (gk == 1 || m == 0)) {
          float lam = sLam[C + cnt];
          if (cnt == C) {
            const double want = lam_block * drift;
            lam = (float)want;
            drift = same_in_all(fma(want - (double)lam, lam_inv, 1.0));
          }
#pragma unroll
          for (int mm = 0; mm < D / 16; ++mm)
#pragma unroll
            for (int n = 0; n < NT; ++n) S[mm][n] *= lam;
        }
#pragma unroll
        for (int k = 0; k < C / KS; ++k) {
          __builtin_amdgcn_sched_barrier(0);
          float w[TR::E];
#pragma unroll
          for (int j = 0; j < TR::E; ++j) w[j] = sW[k * KS + TR::col_k(j, kg)];
          Frag vw[NT][TR::PARTS];
#pragma unroll
          for (int n = 0; n < NT; ++n) weighted_frags(TR::template columns<D>(sV, v_cols, k * KS, n), w, vw[n], TR{});
#pragma unroll
          for (int mm = 0; mm < D / 16; ++mm) {
            if (LOOK && 16 * mm >= ro->dk) break;
            if (mm % 4 == 0) __builtin_amdgcn_sched_barrier(0);     // (operands read further ahead would not fit the registers)
            const Frag kf = TR::template acc_columns<D>(sK, k_cols, k * KS, mm);
#pragma unroll
            for (int x = 0; x < TR::PARTS; ++x)
#pragma unroll
              for (int n = 0; n < NT; ++n) S[mm][n] = TR::mfma(kf, vw[n][x], S[mm][n]);
          }
        }
      }
      if constexpr (WALK) {
        __syncthreads();
        // o^T += V^T P^T (P lies in its natural order, as the transposing reads give V)
        if (mine) {
#pragma unroll
          for (int k = 0; k < C / KS; ++k) {
            __builtin_amdgcn_sched_barrier(0);
            Frag vf[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) vf[n] = TR::template columns<D>(sV, v_cols, k * KS, n);
#pragma unroll
            for (int tt = 0; tt < C / 16; ++tt)
              if (16 * tt + 15 >= k * KS) {
#pragma unroll
                for (int x = 0; x < TR::SPLIT; ++x) {
                  const Frag pf = TR::row_frag(sP + (x * C + 16 * tt + i) * PLD, k * KS, kg);
#pragma unroll
                  for (int n = 0; n < NT; ++n) o[n][tt] = TR::mfma(vf[n], pf, o[n][tt]);
                }
              }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (gk == 1 || m + 1 == heads) {
#pragma unroll
          for (int tt = 0; tt < C / 16; ++tt)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int r = 0; r < 4; ++r) odd = fmaf(o[n][tt][r], 0.f, odd);
          asm volatile("" : "+v"(odd));
          out_at = o_at + (gq > 1 ? m * ro->o_head : 0);
          out_cnt = cnt;
#pragma unroll
          for (int tt = 0; tt < C / 16; ++tt)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              char* x = reinterpret_cast<char*>(sQ) + TR::template unit<D>(i, col0 + 16 * n + 4 * kg) + 16 * tt * D * (int)sizeof(T);
              if constexpr (KT == 2) *reinterpret_cast<u32x2*>(x) = u32x2{two_bf16(o[n][tt][0], o[n][tt][1]), two_bf16(o[n][tt][2], o[n][tt][3])};
              else *reinterpret_cast<f32x4*>(x) = o[n][tt];
            }
          if (m + 1 == heads) o_at += dir * C * ro->o_row;
        }
      }
      if (end && (gk == 1 || m + 1 == heads)) have = true;
    }
  }
  if constexpr (WALK) {
    __syncthreads();
    if (out_cnt > 0) flush();
  }
#pragma unroll
  for (int m = 0; m < D / 16; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) odd = fmaf(S[m][n][r], 0.f, odd);
  bool anew = __syncthreads_or(odd != 0.f);
  if (anew) {
    int block = blockIdx.x;
    asm volatile("" : "+s"(block));              // (it finds its span anew: kept so far, that would not fit the registers)
    const int what = needs_tokens<TR, D, WALK, SUM>(a, ro, tid, block);          // (by all lanes: they search for the span together)
    const bool must = __syncthreads_or(what & MUST), nan = __syncthreads_or(what & HAS_NAN);
    anew = must || !nan;                         // (finite throughout: something has left float32's range, where the parts of a factor may cancel)
    if (anew) {
      __threadfence();                           // (rows of o that are written once more)
      __syncthreads();
      walk_tokens<TR, D, WALK, SUM>(a, ro, tid, block);
    }
  }
  float* to = anew ? nullptr : end_of<WALK>(a, ro, sp, item, h);
  if (to) {
#pragma unroll
    for (int m = 0; m < D / 16; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = TR::acc_row(m, kg) + r, col = col0 + 16 * n + i;
          if (row < ro->dk && col < ro->dv) to[row * s_r + col * s_c] = S[m][n][r];
        }
  }
}

// Sequences of several spans: what each span adds to the state becomes each span's start state.  A wave takes 64 values of the
// states and a quarter of 128 spans, which it has in registers at once; the quarters' sums meet in LDS.  The wait for these loads bounds it:
// 13 to 15 us for 128 spans x 4 heads of 128 x 128 (67 MB), 7 to 8 for 32 spans x 8 heads of 64 x 64.
struct JoinArgs {
  float* spans[2];
  const float* s_in[2];
  const int64_t* off;
  const float* log_decay;
  int64_t n_rows;
  int kv, span_log2, size;
};

constexpr int JOIN_EACH = 32;
__global__ __launch_bounds__(THREADS) void k_span_join(const JoinArgs a) {
  constexpr int PARTS = THREADS / 64;
  __shared__ float sum[PARTS][64];
  const int h = blockIdx.x % a.kv, seq = blockIdx.x / a.kv;
  const int64_t lo = clamped(a.off[seq], 0, a.n_rows), hi = clamped(a.off[seq + 1], lo, a.n_rows);
  const int spans = (int)((hi - lo + ((int64_t)1 << a.span_log2) - 1) >> a.span_log2);
  if (spans < 2) return;
  const int lane = threadIdx.x & 63, part = threadIdx.x >> 6;
  const float g = log_of(a.log_decay, h);
  float lam_hi, lam_lo;
  power(g, (double)((int64_t)1 << a.span_log2), lam_hi, lam_lo);
  const int64_t stride = (int64_t)a.kv * a.size;
  const float* s_in = a.s_in[blockIdx.z];
  s_in = s_in ? s_in + ((int64_t)seq * a.kv + h) * a.size : nullptr;
  float* first = a.spans[blockIdx.z] + (((lo >> a.span_log2) + seq) * a.kv + h) * a.size;
  if (spans <= JOIN_EACH) {                                // few: every thread its own value, all of its spans
    for (int e = blockIdx.y * THREADS + threadIdx.x; e < a.size; e += gridDim.y * THREADS) {
      float cur = s_in ? s_in[e] : 0.f;
      for (int j0 = 0; j0 < spans; j0 += 8) {
        float add[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) add[x] = j0 + x + 1 < spans ? first[(j0 + x) * stride + e] : 0.f;
#pragma unroll
        for (int x = 0; x < 8; ++x)
          if (j0 + x < spans) {
            first[(j0 + x) * stride + e] = cur;
            cur = decayed(cur, lam_hi, lam_lo, add[x]);
          }
      }
    }
    return;
  }
  float far_hi, far_lo;
  power(g, (double)((int64_t)JOIN_EACH << a.span_log2), far_hi, far_lo);
  for (int e0 = blockIdx.y * 64; e0 < a.size; e0 += gridDim.y * 64) {
    const int e = min(e0 + lane, a.size - 1);              // (lanes past the end repeat the last value and store nothing)
    const bool live = e0 + lane < a.size;
    float* p = first + e;
    float start = s_in ? s_in[e] : 0.f;
    for (int j0 = 0; j0 < spans; j0 += PARTS * JOIN_EACH) {
      const int j1 = j0 + part * JOIN_EACH, n = min(JOIN_EACH, spans - j1);
      float add[JOIN_EACH], all = 0.f;
#pragma unroll
      for (int x = 0; x < JOIN_EACH; ++x) add[x] = j1 + x + 1 < spans ? p[(j1 + x) * stride] : 0.f;
#pragma unroll
      for (int x = 0; x < JOIN_EACH; ++x) all = decayed(all, lam_hi, lam_lo, add[x]);
      __syncthreads();
      sum[part][lane] = all;
      __syncthreads();
      float cur = start;
      for (int k = 0; k < PARTS; ++k) {
        if (k == part) {
          float c = cur;
#pragma unroll
          for (int x = 0; x < JOIN_EACH; ++x) {
            if (x < n && live) p[(j1 + x) * stride] = c;
            c = decayed(c, lam_hi, lam_lo, add[x]);
          }
        }
        cur = decayed(cur, far_hi, far_lo, sum[k][lane]);
      }
      start = cur;                                         // (used where all parts were full)
    }
  }
}

// One token a request: the state is read and written once, which bounds it.  A workgroup takes 32 columns of one state (V of
// them a thread and row), all of them in registers: each load is on its way before the first is waited for.  256 requests, 16 heads of
// 128 x 128: 537 MB in 97 to 118 us (5.5 to 4.6 TB/s); one request, 8 heads of 64: 4 us.
struct StepArgs {
  const void *q, *k, *v;
  void* o;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
  float* state;
  const int32_t* slots;
  const float* log_decay;
  float scale;
  int n_states, kv, g, dk, dv, slices;
};

template <class TR, int V>
__global__ __launch_bounds__(THREADS) void k_decay_step(const StepArgs a) {
  using T = typename TR::T;
  constexpr int COLS = 32, ACROSS = COLS / V, ROWS = THREADS / ACROSS, STEPS = 128 / ROWS;
  __shared__ float red[THREADS / 64][COLS];
  const int tid = threadIdx.x;
  const int slice = blockIdx.x % a.slices, bh = blockIdx.x / a.slices, h = bh % a.kv, b = bh / a.kv;
  const int col = slice * COLS + (tid % ACROSS) * V, row0 = tid / ACROSS;
  const int slot = a.slots ? a.slots[b] : b;
  T* ob = static_cast<T*>(a.o) + b * a.o_row + (int64_t)h * a.g * a.o_head;
  if (slot < 0 || slot >= a.n_states) {
    for (int x = tid; x < a.g * COLS; x += THREADS)
      if (slice * COLS + x % COLS < a.dv) ob[(x / COLS) * a.o_head + slice * COLS + x % COLS] = TR::put(0.f);
    return;
  }
  // (the rounding of one float32 would be the same at every token, and add up over all that the state remembers)
  float lam_hi, lam_lo;
  power(log_of(a.log_decay, h), 1.0, lam_hi, lam_lo);
  const T* qb = static_cast<const T*>(a.q) + b * a.q_row + (int64_t)h * a.g * a.q_head;
  const T* kb = static_cast<const T*>(a.k) + b * a.k_row + h * a.k_head;
  const T* vb = static_cast<const T*>(a.v) + b * a.v_row + h * a.v_head;
  float* sb = a.state + ((int64_t)slot * a.kv + h) * a.dk * a.dv;
  const bool live = col < a.dv;             // (V = 4: dv is a multiple of 4)
  float S[STEPS][V], v[V];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int row = row0 + s * ROWS;
    if (live && row < a.dk) {
      if constexpr (V == 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(sb + row * a.dv + col);
#pragma unroll
        for (int j = 0; j < V; ++j) S[s][j] = x[j];
      } else {
        S[s][0] = sb[row * a.dv + col];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = live ? TR::get(vb[col + j]) : 0.f;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int row = row0 + s * ROWS;
    if (live && row < a.dk) {
      const float k = TR::get(kb[row]);
#pragma unroll
      for (int j = 0; j < V; ++j) S[s][j] = decayed(S[s][j], lam_hi, lam_lo, k * v[j]);
      if constexpr (V == 4) *reinterpret_cast<f32x4*>(sb + row * a.dv + col) = f32x4{S[s][0], S[s][1], S[s][2], S[s][3]};
      else sb[row * a.dv + col] = S[s][0];
    }
  }
  for (int m = 0; m < a.g; ++m) {
    float o[V];
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = 0.f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int row = row0 + s * ROWS;
      if (live && row < a.dk) {
        const float q = TR::get(qb[m * a.q_head + row]);
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = fmaf(q, S[s][j], o[j]);
      }
    }
#pragma unroll
    for (int d = ACROSS; d < 64; d *= 2)
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] += __shfl_xor(o[j], d);
    if ((tid & 63) < ACROSS)
#pragma unroll
      for (int j = 0; j < V; ++j) red[tid >> 6][(tid & 63) * V + j] = o[j];
    __syncthreads();
    if (tid < COLS && slice * COLS + tid < a.dv)
      ob[m * a.o_head + slice * COLS + tid] = TR::put(a.scale * (red[0][tid] + red[1][tid] + red[2][tid] + red[3][tid]));
    __syncthreads();
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------
int check(const nugpr_decay_attention* p) {
  if (!p) { set_error("problem is null"); return NUGPR_ERR_INVALID; }
  if (p->dtype != NUGPR_FLOAT32 && p->dtype != NUGPR_BFLOAT16) { set_error("dtype must be NUGPR_FLOAT32 or NUGPR_BFLOAT16"); return NUGPR_ERR_INVALID; }
  if (p->kv_heads < 1 || p->heads < p->kv_heads || p->heads % p->kv_heads || p->heads > 4096) {
    set_error("heads must be 1..4096 and a multiple of kv_heads");
    return NUGPR_ERR_INVALID;
  }
  if (p->dim_k < 1 || p->dim_k > 128 || p->dim_v < 1 || p->dim_v > 128) { set_error("dim_k and dim_v must be 1..128"); return NUGPR_ERR_INVALID; }
  if (p->n_rows < 0 || p->n_rows > (int64_t)1 << 40) { set_error("n_rows must be 0..2^40"); return NUGPR_ERR_INVALID; }
  if (p->n_seqs < 0) { set_error("n_seqs must be >= 0"); return NUGPR_ERR_INVALID; }
  return NUGPR_OK;
}

int check_heads(const nugpr_heads* x, const char* name, size_t value) {
  if (!x || !x->data) { set_error(std::string(name) + " is null"); return NUGPR_ERR_INVALID; }
  if (x->row_stride < 0 || x->head_stride < 0) { set_error(std::string(name) + ": negative stride"); return NUGPR_ERR_INVALID; }
  if (reinterpret_cast<uintptr_t>(x->data) % value) { set_error(std::string(name) + " misaligned"); return NUGPR_ERR_INVALID; }
  return NUGPR_OK;
}

size_t value_size(const nugpr_decay_attention* p) { return p->dtype == NUGPR_BFLOAT16 ? 2 : 4; }

bool wide(const nugpr_heads* x, int width, size_t value) {
  const int64_t e = 16 / (int64_t)value;
  return !(reinterpret_cast<uintptr_t>(x->data) & 15u) && x->row_stride % e == 0 && x->head_stride % e == 0 && width % e == 0 &&
         x->row_stride >= width && x->row_stride < (int64_t)1 << 22;      // (rows one behind the other, a block of them within 31-bit offsets)
}

// Whether the instantiation for widths up to 64 serves a problem.
bool narrow(const nugpr_decay_attention* p) { return p->dim_k <= 64 && p->dim_v <= 64; }

// Rows of a span: a power of two, no less than a block, so large that the scans of the call give about 512 workgroups, or more (2048 at
// most) the smaller their states, whose way through memory is what a span costs.  65536 rows, 16 / 4 heads of 128: 310, 250, 274,
// 313 us with 256, 512, 1024, 2048 workgroups; 20011 rows in 40 uneven sequences, 8 heads of 64, float32: 145, 112, 108, 132 with
// 512, 1024, 2048, 4096.
int span_log2(const nugpr_decay_attention* p, int scans) {
  const int64_t groups = min((int64_t)2048, (int64_t)512 * 128 * 128 / (p->dim_k * p->dim_v));
  int k = p->dtype == NUGPR_BFLOAT16 ? 6 : 5;
  while (k < 30 && ((p->n_rows * p->kv_heads * scans) >> k) > groups) ++k;
  return k;
}
int64_t span_count(const nugpr_decay_attention* p, int scans) { return (p->n_rows >> span_log2(p, scans)) + p->n_seqs; }
size_t span_bytes(const nugpr_decay_attention* p, int scans) {
  const size_t b = (size_t)span_count(p, scans) * p->kv_heads * p->dim_k * p->dim_v * sizeof(float);
  return (b + 255) / 256 * 256;
}

constexpr int FORWARD_SCANS = 1, BACKWARD_SCANS = 3;

template <class TR, int D, int C>
void launch_adds(const ScanArgs& adds, int n_adds, bool al, hipStream_t s) {
  const dim3 grid((unsigned)adds.items * adds.kv, n_adds), threads(64 * Tile<TR, D, C>::WAVES);
  if (al) hipLaunchKernelGGL((k_decay_scan<TR, D, C, true, false, true>), grid, threads, 0, s, adds);
  else hipLaunchKernelGGL((k_decay_scan<TR, D, C, false, false, true>), grid, threads, 0, s, adds);
}

template <class TR, int D, int C, bool SUM>
void launch_walk(const ScanArgs& walk, int n_walk, bool al, hipStream_t s) {
  const dim3 grid((unsigned)walk.items * walk.kv + walk.kv, n_walk), threads(64 * Tile<TR, D, C>::WAVES);
  if (al) hipLaunchKernelGGL((k_decay_scan<TR, D, C, true, true, SUM>), grid, threads, 0, s, walk);
  else hipLaunchKernelGGL((k_decay_scan<TR, D, C, false, true, SUM>), grid, threads, 0, s, walk);
}

// Rows of a block: 64 in bfloat16 for widths beyond 64, else 32.  In float32, tiles and operands of 64 leave room for one workgroup of the wide
// kernels on a compute unit instead of two (16384 rows, 8 heads of 128: 223 against 189 us), and for fewer of the narrow ones (20011 rows, 8
// heads of 64: 125 against 108), as they do in narrow bfloat16 (30000 rows, 16 / 4 heads of 64: 94 against 83; 2048 rows, 8 heads: 22.5 and 23).
// Wide bfloat16 has the state's operand to make once a block (65536 rows, 16 / 4 heads of 128: 282 with 32, 258 with 64; gradients of 16 x 1024
// rows, 16 heads: 236 and 223).
template <class TR, int D>
int launch_scans(const ScanArgs& adds, int n_adds, const JoinArgs& join, const ScanArgs& walk, int n_walk, bool al, hipStream_t s) {
  constexpr int C = TR::E == 8 && D > 64 ? 64 : 32;
  // (a span that holds all rows: no sequence has several)
  if (((int64_t)1 << walk.span_log2) < walk.n_rows) {
    launch_adds<TR, D, C>(adds, n_adds, al, s);
    // (workgroups to fill the card with few sequences, not so many with many, most of which have one span: four times as many make 218 us of
    // gradients 221, 16 x 1024 rows, 16 heads of 128, and 108.6 us 107.5, 20011 rows in 40 uneven sequences, 8 heads of 64, float32)
    const int64_t pairs = (int64_t)walk.n_seqs * walk.kv, blocks = (join.size + 63) / 64;
    const int64_t y = min(blocks, (2047 + pairs) / pairs);
    hipLaunchKernelGGL(k_span_join, dim3((unsigned)pairs, (unsigned)y, n_adds), dim3(THREADS), 0, s, join);
  }
  if (n_walk == 1) launch_walk<TR, D, C, false>(walk, n_walk, al, s);
  else if (walk.role[1].gk > 1) launch_walk<TR, D, C, true>(walk, n_walk, al, s);
  else launch_walk<TR, D, C, false>(walk, n_walk, al, s);
  NUGPR_HIP(hipGetLastError());
  return NUGPR_OK;
}

int launch_scans(const nugpr_decay_attention* p, const ScanArgs& adds, int n_adds, const JoinArgs& join, const ScanArgs& walk, int n_walk,
                 bool al, hipStream_t s) {
  if (p->dtype == NUGPR_BFLOAT16)
    return narrow(p) ? launch_scans<Bf16, 64>(adds, n_adds, join, walk, n_walk, al, s) : launch_scans<Bf16, 128>(adds, n_adds, join, walk, n_walk, al, s);
  return narrow(p) ? launch_scans<F32, 64>(adds, n_adds, join, walk, n_walk, al, s) : launch_scans<F32, 128>(adds, n_adds, join, walk, n_walk, al, s);
}

ScanRole role(const nugpr_heads* q, const nugpr_heads* k, const nugpr_heads* v, const nugpr_heads* o, int gq, int gk, int dk, int dv,
              float wscale, float oscale, int back, int s_trans, const float* s_in, float* s_out, float* spans) {
  ScanRole r{};
  r.q = q->data; r.q_row = q->row_stride; r.q_head = q->head_stride;
  r.k = k->data; r.k_row = k->row_stride; r.k_head = k->head_stride;
  r.v = v->data; r.v_row = v->row_stride; r.v_head = v->head_stride;
  r.o = o->data; r.o_row = o->row_stride; r.o_head = o->head_stride;
  r.gq = gq; r.gk = gk; r.dk = dk; r.dv = dv;
  r.wscale = wscale; r.oscale = oscale; r.back = back; r.s_trans = s_trans;
  r.s_in = s_in; r.s_out = s_out; r.spans = spans;
  return r;
}

// what both scanning calls check; *done: nothing is left to do
int check_scan(const nugpr_decay_attention* p, int scans, size_t need, bool* done) {
  *done = false;
  if (!std::isfinite((float)p->scale)) { set_error("scale must be finite in float32"); return NUGPR_ERR_INVALID; }
  if (p->n_rows == 0 && p->n_seqs == 0) { *done = true; return NUGPR_OK; }
  if (p->n_seqs < 1 || !p->seq_offsets || !p->log_decay) { set_error("seq_offsets or log_decay is null, or there is no sequence"); return NUGPR_ERR_INVALID; }
  // (the threads of a launch are counted in 32 bits)
  if ((span_count(p, scans) + 1) * p->kv_heads > (int64_t)0xffffffff / (narrow(p) ? 256 : 512)) { set_error("too many rows, sequences and heads for one call"); return NUGPR_ERR_INVALID; }
  if (need && (!p->workspace || (reinterpret_cast<uintptr_t>(p->workspace) & 255u))) { set_error("workspace is null or not 256-byte aligned"); return NUGPR_ERR_WORKSPACE; }
  if (p->workspace_bytes < need) { set_error("workspace smaller than nugpr_decay_attention_workspace_bytes()"); return NUGPR_ERR_WORKSPACE; }
  return NUGPR_OK;
}

ScanArgs scan_args(const nugpr_decay_attention* p, int scans) {
  ScanArgs a{};
  a.off = p->seq_offsets; a.log_decay = p->log_decay; a.n_rows = p->n_rows; a.n_seqs = p->n_seqs; a.kv = p->kv_heads;
  a.span_log2 = span_log2(p, scans);
  a.items = (int)span_count(p, scans);
  return a;
}

JoinArgs join_args(const nugpr_decay_attention* p, int scans) {
  JoinArgs j{};
  j.off = p->seq_offsets; j.log_decay = p->log_decay; j.n_rows = p->n_rows; j.kv = p->kv_heads;
  j.span_log2 = span_log2(p, scans);
  j.size = p->dim_k * p->dim_v;
  return j;
}

}  // namespace

}  // namespace nugpr

using namespace nugpr;

#define NUGPR_TRY(call)                 \
  do {                                  \
    const int c__ = (call);             \
    if (c__ != NUGPR_OK) return c__;    \
  } while (0)

extern "C" {

size_t nugpr_decay_attention_workspace_bytes(const nugpr_decay_attention* p, int32_t backward) {
  if (check(p) != NUGPR_OK) return 0;
  return 256 + (backward ? 2 * span_bytes(p, BACKWARD_SCANS) : span_bytes(p, FORWARD_SCANS));
}

int nugpr_decay_attention_forward(const nugpr_decay_attention* p, const nugpr_heads* q, const nugpr_heads* k, const nugpr_heads* v,
                                  const float* initial_state, const nugpr_heads* o, float* final_state, void* stream) {
  NUGPR_TRY(check(p));
  bool done;
  NUGPR_TRY(check_scan(p, FORWARD_SCANS, span_bytes(p, FORWARD_SCANS), &done));
  if (done) return NUGPR_OK;
  const size_t z = value_size(p);
  if (p->n_rows > 0) {
    NUGPR_TRY(check_heads(q, "q", z));
    NUGPR_TRY(check_heads(k, "k", z));
    NUGPR_TRY(check_heads(v, "v", z));
    NUGPR_TRY(check_heads(o, "o", z));
  } else if (!q || !k || !v || !o) {
    set_error("q, k, v or o is null");
    return NUGPR_ERR_INVALID;
  }
  const int g = p->heads / p->kv_heads, dk = p->dim_k, dv = p->dim_v;
  const bool al = wide(q, dk, z) && wide(k, dk, z) && wide(v, dv, z) && wide(o, dv, z);
  ScanArgs walk = scan_args(p, FORWARD_SCANS);
  walk.role[0] = role(q, k, v, o, g, 1, dk, dv, 1.f, (float)p->scale, 0, 0, initial_state, final_state, static_cast<float*>(p->workspace));
  JoinArgs join = join_args(p, FORWARD_SCANS);
  join.spans[0] = static_cast<float*>(p->workspace);
  join.s_in[0] = initial_state;
  return launch_scans(p, walk, 1, join, walk, 1, al, reinterpret_cast<hipStream_t>(stream));
}

int nugpr_decay_attention_backward(const nugpr_decay_attention* p, const nugpr_heads* q, const nugpr_heads* k, const nugpr_heads* v,
                                   const float* initial_state, const nugpr_heads* d_o, const float* d_final_state, const nugpr_heads* dq,
                                   const nugpr_heads* dk, const nugpr_heads* dv, float* d_initial_state, void* stream) {
  NUGPR_TRY(check(p));
  bool done;
  const size_t each = span_bytes(p, BACKWARD_SCANS);
  NUGPR_TRY(check_scan(p, BACKWARD_SCANS, 2 * each, &done));
  if (done) return NUGPR_OK;
  const size_t z = value_size(p);
  const nugpr_heads* every[] = {q, k, v, d_o, dq, dk, dv};
  const char* names[] = {"q", "k", "v", "d_o", "dq", "dk", "dv"};
  bool al = true;
  for (int x = 0; x < 7; ++x) {
    if (p->n_rows > 0) NUGPR_TRY(check_heads(every[x], names[x], z));
    if (!every[x]) { set_error(std::string(names[x]) + " is null"); return NUGPR_ERR_INVALID; }
    al = al && wide(every[x], x == 2 || x == 3 || x == 6 ? p->dim_v : p->dim_k, z);
  }
  const int g = p->heads / p->kv_heads, wk = p->dim_k, wv = p->dim_v;
  // (two roles read d_final_state, one of them writes d_initial_state)
  const uintptr_t from = reinterpret_cast<uintptr_t>(d_final_state), to = reinterpret_cast<uintptr_t>(d_initial_state);
  const size_t states = (size_t)p->n_seqs * p->kv_heads * wk * wv * sizeof(float);
  if (from && to && from < to + states && to < from + states) { set_error("d_initial_state overlaps d_final_state"); return NUGPR_ERR_INVALID; }
  const float scale = (float)p->scale;
  float* s_spans = static_cast<float*>(p->workspace);                       // states S, dim_k x dim_v
  float* u_spans = reinterpret_cast<float*>(static_cast<char*>(p->workspace) + each);     // gradients U, dim_k x dim_v
  ScanArgs walk = scan_args(p, BACKWARD_SCANS), adds = walk;
  walk.role[0] = role(d_o, v, k, dq, g, 1, wv, wk, 1.f, scale, 0, 1, initial_state, nullptr, s_spans);
  walk.role[1] = role(v, d_o, q, dk, 1, g, wv, wk, scale, 1.f, 1, 1, d_final_state, nullptr, u_spans);
  walk.role[2] = role(k, q, d_o, dv, 1, g, wk, wv, scale, 1.f, 1, 0, d_final_state, d_initial_state, u_spans);
  adds.role[0] = role(q, k, v, dq, g, 1, wk, wv, 1.f, scale, 0, 0, nullptr, nullptr, s_spans);
  adds.role[1] = walk.role[2];
  JoinArgs join = join_args(p, BACKWARD_SCANS);
  join.spans[0] = s_spans; join.s_in[0] = initial_state;
  join.spans[1] = u_spans; join.s_in[1] = d_final_state;
  return launch_scans(p, adds, 2, join, walk, 3, al, reinterpret_cast<hipStream_t>(stream));
}

int nugpr_decay_attention_step(const nugpr_decay_attention* p, const nugpr_heads* q, const nugpr_heads* k, const nugpr_heads* v, float* state,
                               const int32_t* slots, const nugpr_heads* o, void* stream) {
  NUGPR_TRY(check(p));
  if (!std::isfinite((float)p->scale)) { set_error("scale must be finite in float32"); return NUGPR_ERR_INVALID; }
  if (p->n_rows == 0) return NUGPR_OK;
  const size_t z = value_size(p);
  NUGPR_TRY(check_heads(q, "q", z));
  NUGPR_TRY(check_heads(k, "k", z));
  NUGPR_TRY(check_heads(v, "v", z));
  NUGPR_TRY(check_heads(o, "o", z));
  if (!p->log_decay || (p->n_seqs > 0 && !state)) { set_error("log_decay or state is null"); return NUGPR_ERR_INVALID; }
  if (reinterpret_cast<uintptr_t>(state) & 3u) { set_error("state misaligned"); return NUGPR_ERR_INVALID; }
  if (!slots && p->n_rows > p->n_seqs) { set_error("more requests than states"); return NUGPR_ERR_INVALID; }
  StepArgs a{};
  a.q = q->data; a.q_row = q->row_stride; a.q_head = q->head_stride;
  a.k = k->data; a.k_row = k->row_stride; a.k_head = k->head_stride;
  a.v = v->data; a.v_row = v->row_stride; a.v_head = v->head_stride;
  a.o = o->data; a.o_row = o->row_stride; a.o_head = o->head_stride;
  a.state = state; a.slots = slots; a.log_decay = p->log_decay; a.scale = (float)p->scale;
  a.n_states = p->n_seqs; a.kv = p->kv_heads; a.g = p->heads / p->kv_heads; a.dk = p->dim_k; a.dv = p->dim_v;
  a.slices = (p->dim_v + 31) / 32;
  const int64_t groups = p->n_rows * a.kv * a.slices;
  if (groups > (int64_t)0xffffffff / THREADS) { set_error("too many requests and heads for one call"); return NUGPR_ERR_INVALID; }
  const bool four = p->dim_v % 4 == 0 && !(reinterpret_cast<uintptr_t>(state) & 15u);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)groups), threads(THREADS);
  if (p->dtype == NUGPR_BFLOAT16) {
    if (four) hipLaunchKernelGGL((k_decay_step<Bf16, 4>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((k_decay_step<Bf16, 1>), grid, threads, 0, s, a);
  } else {
    if (four) hipLaunchKernelGGL((k_decay_step<F32, 4>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((k_decay_step<F32, 1>), grid, threads, 0, s, a);
  }
  NUGPR_HIP(hipGetLastError());
  return NUGPR_OK;
}

}  // extern "C"
