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

constexpr int C = 64;             // rows of a block
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
  ScanRole role[3];
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
__device__ void power(float g, int n, float& hi, float& lo) {
  const double p = exp((double)g * n);
  hi = (float)p;
  lo = (float)(p - (double)hi);
}

template <class TR, int D>
struct Tile {
  static constexpr int LD = D + (TR::E == 8 ? 8 : 4);       // 16 rows of a 16-byte column on different banks
  static constexpr int A_ROW = D / TR::E;                   // threads a row
  static constexpr int PASS = THREADS / A_ROW;              // rows that one load of all threads covers
  static constexpr int N = C / PASS;
};

// Rows first + dir r, r < cnt, of one head, `width` columns: 16 bytes a thread and pass; zero elsewhere.
template <class TR, int D, bool AL>
__device__ inline void fetch(u32x4* r, const void* base, int64_t stride, int64_t first, int dir, int cnt, int width) {
  using L = Tile<TR, D>;
  const int col = (threadIdx.x % L::A_ROW) * TR::E, row0 = threadIdx.x / L::A_ROW;
#pragma unroll
  for (int p = 0; p < L::N; ++p) {
    const int row = row0 + p * L::PASS;
    u32x4 v = {0, 0, 0, 0};
    if (row < cnt && col < width) {
      const typename TR::T* x = static_cast<const typename TR::T*>(base) + (first + (int64_t)dir * row) * stride + col;
      if constexpr (AL) {
        v = *reinterpret_cast<const u32x4*>(x);
      } else if constexpr (TR::E == 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col + j < width) v[j >> 1] |= (uint32_t)x[j] << (16 * (j & 1));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (col + j < width) v[j] = __builtin_bit_cast(uint32_t, x[j]);
      }
    }
    r[p] = v;
  }
}

template <class TR, int D, bool PLACED>
__device__ inline void put(typename TR::T* tile, const u32x4* r) {
  using L = Tile<TR, D>;
  const int col = (threadIdx.x % L::A_ROW) * TR::E, row0 = threadIdx.x / L::A_ROW;
#pragma unroll
  for (int p = 0; p < L::N; ++p) {
    typename TR::T* row = tile + (row0 + p * L::PASS) * L::LD;
    if constexpr (PLACED) TR::store_row(row, col, r[p]);
    else *reinterpret_cast<u32x4*>(row + col) = r[p];
  }
}

// One workgroup walks one span of one sequence and key / value head in blocks of C rows; the state stays in accumulator
// registers, its columns split among the four waves.  WALK: writes o from given start states; else: what the span adds to
// the state, for k_span_join.
// Per block and head: P^T = K Q^T (each wave 16 rows of Q), masked and decayed, goes through LDS; o^T = S^T Q^T and V^T P^T with
// the wave's columns of S and V; S += K^T (w V).  S is read as an operand where it lies (matrix_core.h).  In bfloat16 the state
// takes part with 16 of its bits and P with 8; w V, which is summed into the float32 state, with all 24.
// Values that are not finite: rows s > t must not touch o_t, but 0 x NaN in the masked part of P would; a block whose V
// has such a value takes P V row by row.
template <class TR, int D, bool AL, bool WALK>
__global__ __launch_bounds__(THREADS, 2) void k_decay_scan(const ScanArgs a) {
  using T = typename TR::T;
  using Frag = typename TR::Frag;
  using L = Tile<TR, D>;
  constexpr int KS = TR::KS, KT = KS / 16;       // accumulator tiles of a contraction step
  constexpr int NT = D / 64;                     // tiles of a wave's columns
  constexpr int PLD = C + (TR::E == 8 ? 8 : 4);
  __shared__ __align__(16) T sK[C * L::LD];
  __shared__ __align__(16) T sV[C * L::LD];
  __shared__ __align__(16) T sQ[WALK ? C * L::LD : 8];
  __shared__ __align__(16) T sP[WALK ? C * PLD : 8];
  __shared__ __align__(16) float sLam[C + 4];    // lam^i
  __shared__ __align__(16) float sW[C];          // weights of the block's rows in the state
  __shared__ int sOdd;

  const ScanRole& ro = a.role[blockIdx.y];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, kg = lane >> 4;
  const int h = blockIdx.x % a.kv, item = blockIdx.x / a.kv;

  if (WALK && item == a.items) {                 // rows that no sequence owns
    const int64_t lo = clamped(a.off[0], 0, a.n_rows), hi = clamped(a.off[a.n_seqs], lo, a.n_rows);
    const int64_t none = lo + a.n_rows - hi, per = (int64_t)ro.gq * ro.dv;
    for (int64_t e = tid; e < none * per; e += THREADS) {
      const int64_t r = e / per;
      const int c = (int)(e - r * per);
      static_cast<T*>(ro.o)[(r < lo ? r : r - lo + hi) * ro.o_row + (int64_t)(h * ro.gq + c / ro.dv) * ro.o_head + c % ro.dv] = TR::put(0.f);
    }
    return;
  }
  const int seq = sequence_of(a.off, a.n_seqs, a.n_rows, a.span_log2, item);
  if (seq < 0) return;
  const int64_t lo = clamped(a.off[seq], 0, a.n_rows), hi = clamped(a.off[seq + 1], lo, a.n_rows);
  const int64_t len = hi - lo, span = (int64_t)1 << a.span_log2;
  const int64_t c0 = (item - ((lo >> a.span_log2) + seq)) << a.span_log2;
  const bool last = c0 + span >= len, several = len > span;
  if (c0 > 0 && c0 >= len) return;
  if (!WALK && last) return;
  const int n_tok = (int)min(span, len - c0);
  const int e = ro.back;

  const float g = log_of(a.log_decay, h);
  for (int n = tid; n <= C; n += THREADS) sLam[n] = (float)exp((double)g * n);
  if (tid == 0) sOdd = 0;
  float lam_hi, lam_lo;
  power(g, C, lam_hi, lam_lo);

  // the state: rows 16 m + 4 kg .., columns col0 + 16 n + i
  f32x4 S[D / 16][NT];
  const int col0 = wave * (D / 4);
  const int64_t s_size = (int64_t)ro.dk * ro.dv;
  const int s_r = ro.s_trans ? 1 : ro.dv, s_c = ro.s_trans ? ro.dk : 1;
  const float* from = !WALK ? nullptr
                      : several ? ro.spans + ((int64_t)item * a.kv + h) * s_size
                      : ro.s_in ? ro.s_in + ((int64_t)seq * a.kv + h) * s_size : nullptr;
  bool have = from != nullptr;
#pragma unroll
  for (int m = 0; m < D / 16; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * m + 4 * kg + r, col = col0 + 16 * n + i;
        S[m][n][r] = have && row < ro.dk && col < ro.dv ? from[row * s_r + col * s_c] : 0.f;
      }

  const int gq = WALK ? ro.gq : 1, gk = ro.gk, heads = max(gq, gk);
  const int blocks = (n_tok + C - 1) / C;
  const int64_t first = e ? hi - 1 - c0 : lo + c0;
  const int dir = e ? -1 : 1;
  const T* qb = static_cast<const T*>(ro.q) + (int64_t)h * ro.gq * ro.q_head;
  const T* kb = static_cast<const T*>(ro.k) + (int64_t)h * ro.gk * ro.k_head;
  const T* vb = static_cast<const T*>(ro.v) + (int64_t)h * ro.gk * ro.v_head;
  u32x4 rq[WALK ? L::N : 1], rk[L::N], rv[L::N];
  auto fetch_block = [&](int b, int m) {
    const int64_t at = first + (int64_t)dir * b * C;
    const int cnt = min(C, n_tok - b * C);
    if (gk > 1 || m == 0) {
      fetch<TR, D, AL>(rk, kb + m * ro.k_head, ro.k_row, at, dir, cnt, ro.dk);
      fetch<TR, D, AL>(rv, vb + m * ro.v_head, ro.v_row, at, dir, cnt, ro.dv);
    }
    if constexpr (WALK)
      if (gq > 1 || m == 0) fetch<TR, D, AL>(rq, qb + m * ro.q_head, ro.q_row, at, dir, cnt, ro.dk);
  };
  f32x4 o[NT][C / 16];
  if (blocks > 0) fetch_block(0, 0);
  int kv_step = 0;
  for (int b = 0; b < blocks; ++b) {
    const int cnt = min(C, n_tok - b * C);
    for (int m = 0; m < heads; ++m) {
      const bool kv_new = gk > 1 || m == 0, q_new = WALK && (gq > 1 || m == 0);
      __syncthreads();
      if (kv_new) {
        ++kv_step;
        put<TR, D, true>(sK, rk);
        put<TR, D, false>(sV, rv);
        if (WALK) {
          bool odd = false;
#pragma unroll
          for (int p = 0; p < L::N; ++p) odd |= TR::odd(rv[p]);
          if (odd) sOdd = kv_step;
        }
        if (tid < C) sW[tid] = tid < cnt ? ro.wscale * (float)sLam[cnt - 1 - tid + e] : 0.f;
      }
      if constexpr (WALK)
        if (q_new) put<TR, D, true>(sQ, rq);
      __syncthreads();
      if (m + 1 < heads) fetch_block(b, m + 1);
      else if (b + 1 < blocks) fetch_block(b + 1, 0);

      const bool end = gq == 1 || m + 1 == heads;          // the state moves on
      const bool keep = !WALK || b + 1 < blocks || (last && ro.s_out);
      if constexpr (WALK) {
        // P^T, rows of K x the wave's 16 rows of Q
        const int t = 16 * wave + i;
        Frag qf[D / KS];
#pragma unroll
        for (int k = 0; k < D / KS; ++k) qf[k] = TR::row_frag(sQ + t * L::LD, k * KS, kg);
#pragma unroll
        for (int st = 0; st < C / 16; ++st) {
          if (st > (KT == 2 ? wave | 1 : wave)) break;     // (a product of 32 rows reads the masked tile too)
          f32x4 p = {0.f, 0.f, 0.f, 0.f};
          if (st <= wave) {
#pragma unroll
            for (int k = 0; k < D / KS; ++k) p = TR::mfma(TR::row_frag(sK + (16 * st + i) * L::LD, k * KS, kg), qf[k], p);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int d = t - (16 * st + 4 * kg + r);
              p[r] = d >= 0 ? p[r] * (ro.wscale * sLam[max(d, 0)]) : 0.f;
            }
          }
          T* to = sP + t * PLD + 16 * st + 4 * kg;
          if constexpr (KT == 2) *reinterpret_cast<u32x2*>(to) = u32x2{two_bf16(p[0], p[1]), two_bf16(p[2], p[3])};
          else *reinterpret_cast<f32x4*>(to) = p;
        }
        // o^T = S^T Q^T, rows of the state's columns
        if (gk == 1 || m == 0) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int tt = 0; tt < C / 16; ++tt) o[n][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (have) {
#pragma unroll
            for (int k = 0; k < D / KS; ++k) {
              Frag sf[NT][TR::S_PARTS];
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                f32x4 part[KT];
#pragma unroll
                for (int x = 0; x < KT; ++x) part[x] = S[k * KT + x][n];
                acc_frags(part, sf[n], TR{});
              }
#pragma unroll
              for (int tt = 0; tt < C / 16; ++tt) {
                const Frag q = TR::row_frag(sQ + (16 * tt + i) * L::LD, k * KS, kg);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                  for (int x = 0; x < TR::S_PARTS; ++x) o[n][tt] = TR::mfma(sf[n][x], q, o[n][tt]);
              }
            }
#pragma unroll
            for (int tt = 0; tt < C / 16; ++tt) {
              const float w = sLam[16 * tt + i + 1 - e];
#pragma unroll
              for (int n = 0; n < NT; ++n) o[n][tt] *= w;
            }
          }
        }
        __syncthreads();
      }
      const bool odd = WALK && sOdd == kv_step;
      if (end && keep && (have || !WALK) && (gk == 1 || m == 0)) {
        if (cnt < C) power(g, cnt, lam_hi, lam_lo);
#pragma unroll
        for (int mm = 0; mm < D / 16; ++mm)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[mm][n][r] = fmaf(S[mm][n][r], lam_hi, S[mm][n][r] * lam_lo);
      }
#pragma unroll
      for (int k = 0; k < C / KS; ++k) {
        Frag vf[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) vf[n] = TR::col_frag(sV, L::LD, k * KS, col0 + 16 * n, i, kg);
        if (WALK && !odd) {
#pragma unroll
          for (int tt = 0; tt < C / 16; ++tt)
            if (16 * tt + 15 >= k * KS) {
              // (P lies in its natural order, as the transposing reads give V)
              const Frag pf = TR::row_frag(sP + (16 * tt + i) * PLD, k * KS, kg);
#pragma unroll
              for (int n = 0; n < NT; ++n) o[n][tt] = TR::mfma(vf[n], pf, o[n][tt]);
            }
        }
        if (end && keep) {
          float w[TR::E];
#pragma unroll
          for (int j = 0; j < TR::E; ++j) w[j] = sW[k * KS + TR::col_k(j, kg)];
          Frag vw[NT][TR::PARTS];
#pragma unroll
          for (int n = 0; n < NT; ++n) weighted_frags(vf[n], w, vw[n], TR{});
#pragma unroll
          for (int mm = 0; mm < D / 16; ++mm) {
            const Frag kf = TR::col_frag_placed(sK, L::LD, k * KS, 16 * mm, i, kg);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int x = 0; x < TR::PARTS; ++x) S[mm][n] = TR::mfma(kf, vw[n][x], S[mm][n]);
          }
        }
      }
      if constexpr (WALK) {
        if (odd) {
          for (int s = 0; s < cnt; ++s)
#pragma unroll
            for (int tt = 0; tt < C / 16; ++tt) {
              const float p = TR::get(sP[(16 * tt + i) * PLD + s]);
              if (s <= 16 * tt + i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                  for (int r = 0; r < 4; ++r) o[n][tt][r] += p * TR::get(sV[s * L::LD + col0 + 16 * n + 4 * kg + r]);
            }
        }
        if (gk == 1 || m + 1 == heads) {
          T* ob = static_cast<T*>(ro.o) + (int64_t)(h * ro.gq + (gq > 1 ? m : 0)) * ro.o_head;
#pragma unroll
          for (int tt = 0; tt < C / 16; ++tt) {
            const int row = 16 * tt + i;
            if (row >= cnt) continue;
            T* orow = ob + (first + (int64_t)dir * (b * C + row)) * ro.o_row;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const int col = col0 + 16 * n + 4 * kg;
              const f32x4 x = o[n][tt] * ro.oscale;
              if constexpr (AL) {
                if (col < ro.dv) {
                  if constexpr (KT == 2) *reinterpret_cast<u32x2*>(orow + col) = u32x2{two_bf16(x[0], x[1]), two_bf16(x[2], x[3])};
                  else *reinterpret_cast<f32x4*>(orow + col) = x;
                }
              } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                  if (col + r < ro.dv) orow[col + r] = TR::put(x[r]);
              }
            }
          }
        }
      }
      if (end && (gk == 1 || m + 1 == heads)) have = true;
    }
  }
  float* to = !WALK ? ro.spans + ((int64_t)item * a.kv + h) * s_size
              : last && ro.s_out ? ro.s_out + ((int64_t)seq * a.kv + h) * s_size : nullptr;
  if (to) {
#pragma unroll
    for (int m = 0; m < D / 16; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * m + 4 * kg + r, col = col0 + 16 * n + i;
          if (row < ro.dk && col < ro.dv) to[row * s_r + col * s_c] = S[m][n][r];
        }
  }
}

// Sequences of several spans: what each span adds to the state becomes each span's start state.
struct JoinArgs {
  float* spans[2];
  const float* s_in[2];
  const int64_t* off;
  const float* log_decay;
  int64_t n_rows;
  int kv, span_log2, size;
};

__global__ __launch_bounds__(THREADS) void k_span_join(const JoinArgs a) {
  const int h = blockIdx.x % a.kv, seq = blockIdx.x / a.kv;
  const int64_t lo = clamped(a.off[seq], 0, a.n_rows), hi = clamped(a.off[seq + 1], lo, a.n_rows);
  const int spans = (int)((hi - lo + ((int64_t)1 << a.span_log2) - 1) >> a.span_log2);
  const int e = blockIdx.y * THREADS + threadIdx.x;
  if (spans < 2 || e >= a.size) return;
  float lam_hi, lam_lo;
  power(log_of(a.log_decay, h), 1 << a.span_log2, lam_hi, lam_lo);
  const int64_t stride = (int64_t)a.kv * a.size;
  const float* s_in = a.s_in[blockIdx.z];
  float* p = a.spans[blockIdx.z] + (((lo >> a.span_log2) + seq) * a.kv + h) * a.size + e;
  float cur = s_in ? s_in[((int64_t)seq * a.kv + h) * a.size + e] : 0.f;
  constexpr int AHEAD = 8;
  for (int j = 0; j < spans; j += AHEAD) {
    float add[AHEAD];
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) add[x] = j + x + 1 < spans ? p[(j + x) * stride] : 0.f;
#pragma unroll
    for (int x = 0; x < AHEAD; ++x)
      if (j + x < spans) {
        p[(j + x) * stride] = cur;
        cur = fmaf(cur, lam_hi, fmaf(cur, lam_lo, add[x]));
      }
  }
}

// One token a request: the state is read and written once, which bounds it.  A workgroup takes 32 columns of one state (V of
// them a thread and row).
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
  const float lam = expf(log_of(a.log_decay, h));
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
      for (int j = 0; j < V; ++j) S[s][j] = fmaf(S[s][j], lam, k * v[j]);
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
  return !(reinterpret_cast<uintptr_t>(x->data) & 15u) && x->row_stride % e == 0 && x->head_stride % e == 0 && width % e == 0;
}

// Rows of a span: a power of two of blocks, so many that the scans of the call give about 512 workgroups (two on
// every compute unit).
int span_log2(const nugpr_decay_attention* p, int scans) {
  int k = 6;
  while (k < 30 && ((p->n_rows * p->kv_heads * scans) >> k) > 512) ++k;
  return k;
}
int64_t span_count(const nugpr_decay_attention* p, int scans) { return (p->n_rows >> span_log2(p, scans)) + p->n_seqs; }
size_t span_bytes(const nugpr_decay_attention* p, int scans) {
  const size_t b = (size_t)span_count(p, scans) * p->kv_heads * p->dim_k * p->dim_v * sizeof(float);
  return (b + 255) / 256 * 256;
}

constexpr int FORWARD_SCANS = 1, BACKWARD_SCANS = 3;

template <class TR, int D>
int launch_scans(const ScanArgs& adds, int n_adds, const JoinArgs& join, const ScanArgs& walk, int n_walk, bool al, hipStream_t s) {
  const unsigned x = (unsigned)walk.items * walk.kv;
  // (a span that holds all rows: no sequence has several)
  if (((int64_t)1 << walk.span_log2) < walk.n_rows) {
    if (al) hipLaunchKernelGGL((k_decay_scan<TR, D, true, false>), dim3(x, n_adds), dim3(THREADS), 0, s, adds);
    else hipLaunchKernelGGL((k_decay_scan<TR, D, false, false>), dim3(x, n_adds), dim3(THREADS), 0, s, adds);
    hipLaunchKernelGGL(k_span_join, dim3((unsigned)walk.n_seqs * walk.kv, (join.size + THREADS - 1) / THREADS, n_adds), dim3(THREADS), 0, s, join);
  }
  if (al) hipLaunchKernelGGL((k_decay_scan<TR, D, true, true>), dim3(x + walk.kv, n_walk), dim3(THREADS), 0, s, walk);
  else hipLaunchKernelGGL((k_decay_scan<TR, D, false, true>), dim3(x + walk.kv, n_walk), dim3(THREADS), 0, s, walk);
  NUGPR_HIP(hipGetLastError());
  return NUGPR_OK;
}

int launch_scans(const nugpr_decay_attention* p, const ScanArgs& adds, int n_adds, const JoinArgs& join, const ScanArgs& walk, int n_walk,
                 bool al, hipStream_t s) {
  const bool narrow = p->dim_k <= 64 && p->dim_v <= 64;
  if (p->dtype == NUGPR_BFLOAT16)
    return narrow ? launch_scans<Bf16, 64>(adds, n_adds, join, walk, n_walk, al, s) : launch_scans<Bf16, 128>(adds, n_adds, join, walk, n_walk, al, s);
  return narrow ? launch_scans<F32, 64>(adds, n_adds, join, walk, n_walk, al, s) : launch_scans<F32, 128>(adds, n_adds, join, walk, n_walk, al, s);
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
  if (!std::isfinite(p->scale)) { set_error("scale must be finite"); return NUGPR_ERR_INVALID; }
  if (p->n_rows == 0 && p->n_seqs == 0) { *done = true; return NUGPR_OK; }
  if (p->n_seqs < 1 || !p->seq_offsets || !p->log_decay) { set_error("seq_offsets or log_decay is null, or there is no sequence"); return NUGPR_ERR_INVALID; }
  if ((span_count(p, scans) + 1) * p->kv_heads > (int64_t)0x7fffffff) { set_error("too many rows, sequences and heads for one call"); return NUGPR_ERR_INVALID; }
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
  if (!std::isfinite(p->scale)) { set_error("scale must be finite"); return NUGPR_ERR_INVALID; }
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
  if (groups > 0x7fffffff) { set_error("too many requests and heads for one call"); return NUGPR_ERR_INVALID; }
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
