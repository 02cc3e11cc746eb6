// A projection that all rows share beside a low-rank adapter for each request, and its gradients:
//
//   y = x W^T + h B_a,      h = scale x A_a^T                 (a: the adapter of the row's request)
//   dx = dy W + u A_a,      u = scale dy B_a^T
//   dA_a = sum u^T x,       dB_a = sum h^T dy                 over the rows of all requests that have a
//
// h and u (rows x rank, float32, in the workspace) are one kernel's work (k_low); the large products take them as a few
// more steps of their contraction (k_project, or k_project_few where there are few rows), the sums over rows are k_adapter_grad's.
#include <algorithm>
#include <cmath>

#include "matrix_core.h"
#include "nugpr_internal.h"
#include "packed_rows.h"

namespace nugpr {

namespace {

constexpr int THREADS = 256;
constexpr int LOW_LOG2 = 4;          // rows of a piece of k_low

struct Requests {
  const int64_t* off;
  const int32_t* adapter_of;         // or null: request s has adapter s
  int64_t n_rows;
  int n_seqs, n_adapters;
};

// the adapter of a request, or -1
__device__ inline int adapter(const Requests& q, int s) {
  const int a = q.adapter_of ? q.adapter_of[s] : s;
  return a >= 0 && a < q.n_adapters ? a : -1;
}

// 16 bytes of a row from column `col` on, zero past `width`; AL: aligned, and the width a multiple of them;
// NOW: nothing else is done while it is on its way
template <class TR, bool AL, bool NOW = false>
__device__ inline u32x4 run16(const typename TR::T* row, int64_t col, int64_t width) {
  u32x4 v = {0, 0, 0, 0};
  if constexpr (AL) {
    if (col < width) v = *reinterpret_cast<const u32x4*>(row + col);
  } else if (col + TR::E <= width) {
    v = NOW ? load16_now(row + col) : load16(row + col);
  } else if (col < width) {
#pragma unroll
    for (int j = 0; j < TR::E; ++j)
      if (col + j < width) {
        if constexpr (TR::E == 8) v[j >> 1] |= (uint32_t)row[col + j] << (16 * (j & 1));
        else v[j] = __builtin_bit_cast(uint32_t, row[col + j]);
      }
  }
  return v;
}

// ---- h = scale x A_a^T --------------------------------------------------------------------------------------------------
struct LowSide {
  const void* x;          // rows x width
  const void* A;          // adapters x rank x width
  float* low;             // rows x padded rank
  int64_t x_stride;
  int width;
};
struct LowArgs {
  LowSide side[2];
  Requests q;
  float scale;
  int rank, padded;
};

// A workgroup takes 16 rows of one request and all of the rank; its waves split the width, operands go from memory straight
// into registers (nothing is read twice but A, from L2), the waves' sums meet in LDS.  The way from L2 bounds it, as a
// workgroup reads as much of A as of x: 8192 rows of 4096, rank 16, bfloat16: 25 to 27 us (67 MB, 2.6 TB/s).
template <class TR, bool AL, int TILES>
__global__ __launch_bounds__(1024) void k_low(const LowArgs a) {
  using T = typename TR::T;
  extern __shared__ float red[];           // waves x 16 rows x 16 TILES
  const LowSide& sd = a.side[blockIdx.y];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6, i = lane & 15, kg = lane >> 4;
  const int item = blockIdx.x;
  const PieceOf piece = piece_of(a.q.off, a.q.n_seqs, a.q.n_rows, LOW_LOG2, item);
  const int s = piece.seq;
  if (s < 0) return;
  const int64_t lo = piece.lo, hi = piece.hi;
  const int64_t row0 = lo + ((item - ((lo >> LOW_LOG2) + s)) << LOW_LOG2);
  const int ad = adapter(a.q, s);
  if (row0 >= hi || ad < 0) return;
  const int rows = (int)min((int64_t)16, hi - row0);
  const T* x = static_cast<const T*>(sd.x) + (row0 + i) * sd.x_stride;
  const T* A = static_cast<const T*>(sd.A) + (int64_t)ad * a.rank * sd.width;
  f32x4 acc[TILES];
#pragma unroll
  for (int n = 0; n < TILES; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  // (a wave takes RUN steps side by side, 256 bytes of a row, and has all their loads on the way at once)
  constexpr int RUN = TILES > 4 ? 1 : TILES > 2 ? 2 : 4;
  for (int k0 = wave * RUN * TR::KS; k0 < sd.width; k0 += waves * RUN * TR::KS) {
    u32x4 xv[RUN], av[RUN][TILES];
#pragma unroll
    for (int u = 0; u < RUN; ++u) {
      const int col = k0 + u * TR::KS + kg * TR::E;
      xv[u] = i < rows ? run16<TR, AL, true>(x, col, sd.width) : u32x4{0, 0, 0, 0};
#pragma unroll
      for (int n = 0; n < TILES; ++n)
        av[u][n] = 16 * n + i < a.rank ? run16<TR, AL, true>(A + (int64_t)(16 * n + i) * sd.width, col, sd.width) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < RUN; ++u)
#pragma unroll
      for (int n = 0; n < TILES; ++n)
        acc[n] = TR::mfma(__builtin_bit_cast(typename TR::Frag, xv[u]), __builtin_bit_cast(typename TR::Frag, av[u][n]), acc[n]);
  }
#pragma unroll
  for (int n = 0; n < TILES; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) red[(wave * 16 + 4 * kg + r) * (16 * TILES) + 16 * n + i] = acc[n][r];
  __syncthreads();
  for (int e = tid; e < rows * a.padded; e += blockDim.x) {
    const int r = e / a.padded, j = e - r * a.padded;
    float sum = 0.f;
    if (j < a.rank)
      for (int w = 0; w < waves; ++w) sum += red[(w * 16 + r) * (16 * TILES) + j];
    sd.low[(row0 + r) * a.padded + j] = a.scale * sum;
  }
}

// ---- y = x W^T + h B_a, dx = dy W + u A_a ---------------------------------------------------------------------------------
struct ProjectArgs {
  const void *x, *W, *up;   // rows x width_k; W: n x k (NN: k x n); up: adapters x rank x n
  const float* low;         // rows x padded rank
  void* y;                  // rows x n, dense
  int64_t x_stride;
  Requests q;
  int k, n, rank, padded;
};

// What the large products share.  The accumulators' rows are the columns of y, four in a row a lane: tile (n, m) of a wave stands for
// columns wn + 16 n + 4 kg .. and row wm + 16 m + i of the workgroup's tile.
//
// The adapters are further steps of the contraction: for every request with rows in the tile, its rows of h (in bfloat16 as three
// numbers, exactly) and KS rows of B_a at a time.  sA, sB: room for BM x 128 bytes and BN x 128 bytes.
// A step waits for its loads, about a microsecond, so that with more than OWN_LANES steps in a small tile every lane works on its own
// rows and columns instead, in float32: gradients of 36 requests of one row, rank 64, 547 to 171 columns, bfloat16: 97 us with steps only, 52
// so; 256 requests of four rows, rank 8, 1000 columns: 43 and 21.  (8: 128 of 8 rows 28 instead of 19; 2: as 4.)  Larger tiles take their requests in
// steps however many there are: 4096 rows, 4096 x 4096, rank 16, 385 us in 1024 requests, 130 in 16.
constexpr int OWN_LANES = 4;
template <class TR, int BM, int BN, int MT, int NTL, int N_THREADS, bool AL>
__device__ inline void add_adapters(const ProjectArgs& a, int64_t m0, int n0, int rows, int wm, int wn, typename TR::T* sA, typename TR::T* sB,
                                    f32x4 (&acc)[NTL][MT]) {
  using T = typename TR::T;
  using Frag = typename TR::Frag;
  constexpr int KS = TR::KS, E = TR::E, BK = 128 / sizeof(T);
  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, kg = lane >> 4;
  if constexpr (MT * NTL <= 4) {
    int own[MT], count = 0;
#pragma unroll
    for (int m = 0; m < MT; ++m) own[m] = -1;
    for (int at = 0; at < a.q.n_seqs; at += 64) {
      const int mine = at + lane;
      int64_t lo = 0, hi = 0;
      int ad = -1;
      if (mine < a.q.n_seqs) {
        lo = clamped(a.q.off[mine], m0, m0 + rows);
        hi = clamped(a.q.off[mine + 1], lo, m0 + rows);
        ad = adapter(a.q, mine);
      }
      uint64_t some = __ballot(hi > lo && ad >= 0);
      while (some) {
        const int from = __builtin_ctzll(some);
        some &= some - 1;
        ++count;
        const int rlo = __shfl((int)(lo - m0), from), rhi = __shfl((int)(hi - m0), from), one = __shfl(ad, from);
#pragma unroll
        for (int m = 0; m < MT; ++m)
          if (wm + 16 * m + i >= rlo && wm + 16 * m + i < rhi) own[m] = one;
      }
    }
    if (count * ((a.rank + KS - 1) / KS) > OWN_LANES) {
      if (tid >= THREADS) return;          // (further groups of the same tile)
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        if (own[m] < 0) continue;
        const float* low = a.low + (m0 + wm + 16 * m + i) * a.padded;
#pragma unroll
        for (int n = 0; n < NTL; ++n) {
          const int col = n0 + wn + 16 * n + 4 * kg;
          const T* up = static_cast<const T*>(a.up) + (int64_t)own[m] * a.rank * a.n + col;
          if (col + 4 <= a.n) {
#pragma unroll 8
            for (int j = 0; j < a.rank; ++j) {
              T b[4];
              __builtin_memcpy(b, up + (int64_t)j * a.n, sizeof(b));
              const float h = low[j];
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[n][m][r] = fmaf(h, TR::get(b[r]), acc[n][m][r]);
            }
          } else {
            for (int j = 0; j < a.rank; ++j)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (col + r < a.n) acc[n][m][r] = fmaf(low[j], TR::get(up[(int64_t)j * a.n + r]), acc[n][m][r]);
          }
        }
      }
      return;
    }
  }
  static_assert(TR::PARTS == 1 || BM <= BN, "the third part of h lies beside B_a in sB");
  const int along_at = TR::template along_at<BK>(i, kg), third_at = TR::template along_at<KS>(i, kg);
  T* sThird = sB + KS * BN;
  int cols_at[TR::ACROSS];
  TR::template columns_at<BN>(cols_at, wn, i, kg);
  for (int at = 0; at < a.q.n_seqs; at += 64) {
    // which of 64 requests have rows here
    const int mine = at + lane;
    int64_t lo = 0, hi = 0;
    int ad = -1;
    if (mine < a.q.n_seqs) {
      lo = clamped(a.q.off[mine], m0, m0 + rows);
      hi = clamped(a.q.off[mine + 1], lo, m0 + rows);
      ad = adapter(a.q, mine);
    }
    uint64_t some = __ballot(hi > lo && ad >= 0);
    while (some) {
      const int from = __builtin_ctzll(some);
      some &= some - 1;
      const int rlo = __shfl((int)(lo - m0), from), rhi = __shfl((int)(hi - m0), from), one = __shfl(ad, from);
      const T* up = static_cast<const T*>(a.up) + (int64_t)one * a.rank * a.n;
      for (int j0 = 0; j0 < a.rank; j0 += KS) {
        __syncthreads();
        for (int c = tid; c < BM * KS / 4; c += N_THREADS) {
          const int row = c / (KS / 4), col = c % (KS / 4) * 4;
          f32x4 v = {0.f, 0.f, 0.f, 0.f};
          if (row >= rlo && row < rhi) v = *reinterpret_cast<const f32x4*>(a.low + (m0 + row) * a.padded + j0 + col);
          typename TR::Four parts[TR::PARTS];
          exact_parts(v, parts, TR{});
#pragma unroll
          for (int x = 0; x < TR::PARTS; ++x)
            *reinterpret_cast<typename TR::Four*>(x < 2 ? reinterpret_cast<char*>(sA) + TR::template unit<BK>(row, x * KS + col)
                                                        : reinterpret_cast<char*>(sThird) + TR::template unit<KS>(row, col)) = parts[x];
        }
        for (int c = tid; c < KS * BN / E; c += N_THREADS) {
          const int row = c / (BN / E), col = c % (BN / E) * E;
          *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(sB) + TR::template unit<BN>(row, col)) =
              j0 + row < a.rank ? run16<TR, AL, true>(up + (int64_t)(j0 + row) * a.n, n0 + col, a.n) : u32x4{0, 0, 0, 0};
        }
        __syncthreads();
        Frag wf[NTL], finite[NTL];
#pragma unroll
        for (int n = 0; n < NTL; ++n) {
          wf[n] = TR::template columns<BN>(sB, cols_at, 0, n);
          finite[n] = finite_frag(wf[n], TR{});
        }
        // (an adapter may hold values that are not finite: they are for the rows of its own requests, where a zero row of h
        // would make them NaN)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const int row = wm + 16 * m + i;
          const bool own = row >= rlo && row < rhi;
          Frag xf[TR::PARTS];
#pragma unroll
          for (int part = 0; part < TR::PARTS; ++part)
            xf[part] = part < 2 ? TR::template along<BK>(sA, along_at, wm + 16 * m, part * KS) : TR::template along<KS>(sThird, third_at, wm + 16 * m, 0);
#pragma unroll
          for (int n = 0; n < NTL; ++n) {
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int part = 0; part < TR::PARTS; ++part) v = TR::mfma(part ? finite[n] : wf[n], xf[part], v);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[n][m][r] += own ? v[r] : 0.f;
          }
        }
      }
    }
  }
}

template <class TR, int MT, int NTL, bool AL>
__device__ inline void store_rows(const ProjectArgs& a, int64_t m0, int n0, int rows, int wm, int wn, const f32x4 (&acc)[NTL][MT]) {
  using T = typename TR::T;
  constexpr int E = TR::E;
  const int i = threadIdx.x & 15, kg = (threadIdx.x >> 4) & 3;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int row = wm + 16 * m + i;
    if (row >= rows) continue;
    T* y = static_cast<T*>(a.y) + (m0 + row) * a.n;
#pragma unroll
    for (int n = 0; n < NTL; ++n) {
      const int col = n0 + wn + 16 * n + 4 * kg;
      const f32x4 v = acc[n][m];
      if constexpr (AL) {
        if (col < a.n) {
          if constexpr (E == 8) *reinterpret_cast<u32x2*>(y + col) = u32x2{two_bf16(v[0], v[1]), two_bf16(v[2], v[3])};
          else *reinterpret_cast<f32x4*>(y + col) = v;
        }
      } else if (col + 4 <= a.n) {
        if constexpr (E == 8) store_any(y + col, u32x2{two_bf16(v[0], v[1]), two_bf16(v[2], v[3])});
        else store_any(y + col, v);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (col + r < a.n) y[col + r] = TR::put(v[r]);
      }
    }
  }
}

// 128-byte steps of the contraction through LDS, the loads of the two steps after it in registers meanwhile.  G: groups of four waves
// that share the contraction, each a run of its steps in tiles of its own; the first one adds the others' sums to its own.  For what the wide
// tiles are not for: odd sizes, float32, few tiles, where the wait of a step and the number of steps bound it: 1501 rows, 301 to 500
// columns, float32: 14 us; 1888 rows, 620 to 142, bfloat16: 11.
template <class TR, int BM, int BN, int WM, int WN, int G, bool NN, bool AL>
__global__ __launch_bounds__(THREADS * G) void k_project(const ProjectArgs a) {
  using T = typename TR::T;
  using Frag = typename TR::Frag;
  constexpr int KS = TR::KS, E = TR::E, BK = 128 / sizeof(T), S = sizeof(T);
  constexpr int MT = BM / WM / 16, NTL = BN / WN / 16;        // a wave's tiles
  constexpr int XA = BM * BK / E / THREADS, XB = (BN * BK / E + THREADS - 1) / THREADS;
  static_assert(WM * WN == 4 && 2 * KS <= BK, "");
  __shared__ __align__(16) T tiles[G * (BM + BN) * BK];
  const int tid = threadIdx.x % THREADS, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, kg = lane >> 4;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
  T *sA = tiles + group * (BM + BN) * BK, *sB = sA + BM * BK;
  const int each = ((a.k + BK - 1) / BK + G - 1) / G * BK, k_end = min(a.k, (group + 1) * each);
  const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
  const int64_t m0 = (int64_t)blockIdx.y * BM;
  const int n0 = blockIdx.x * BN;
  const int rows = (int)min((int64_t)BM, a.q.n_rows - m0);
  const T* x = static_cast<const T*>(a.x) + m0 * a.x_stride;
  const T* W = static_cast<const T*>(a.W);
  f32x4 acc[NTL][MT];
#pragma unroll
  for (int n = 0; n < NTL; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 ra0[XA], rb0[XB], ra1[XA], rb1[XB];       // the next step and the one after it
  auto load = [&](u32x4* ra, u32x4* rb, int k0) {
#pragma unroll
    for (int p = 0; p < XA; ++p) {
      const int c = tid + p * THREADS, row = c / (BK / E), col = c % (BK / E) * E;
      ra[p] = row < rows ? run16<TR, AL>(x + (int64_t)row * a.x_stride, k0 + col, k_end) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int p = 0; p < XB; ++p) {
      const int c = tid + p * THREADS;
      u32x4 v = {0, 0, 0, 0};
      if constexpr (NN) {
        const int row = c / (BN / E), col = c % (BN / E) * E;
        if (row < BK && k0 + row < k_end) v = run16<TR, AL>(W + (int64_t)(k0 + row) * a.n, n0 + col, a.n);
      } else {
        const int row = c / (BK / E), col = c % (BK / E) * E;
        if (row < BN && n0 + row < a.n) v = run16<TR, AL>(W + (int64_t)(n0 + row) * a.k, k0 + col, k_end);
      }
      rb[p] = v;
    }
  };
  auto put = [&](const u32x4* ra, const u32x4* rb) {
#pragma unroll
    for (int p = 0; p < XA; ++p) {
      const int c = tid + p * THREADS;
      *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(sA) + TR::template unit<BK>(c / (BK / E), c % (BK / E) * E)) = ra[p];
    }
#pragma unroll
    for (int p = 0; p < XB; ++p) {
      const int c = tid + p * THREADS;
      if (c < BN * BK / E) {
        char* to = reinterpret_cast<char*>(sB);
        if constexpr (NN) *reinterpret_cast<u32x4*>(to + TR::template unit<BN>(c / (BN / E), c % (BN / E) * E)) = rb[p];
        else *reinterpret_cast<u32x4*>(to + TR::template unit<BK>(c / (BK / E), c % (BK / E) * E)) = rb[p];
      }
    }
  };
  const int along_at = TR::template along_at<BK>(i, kg);
  int cols_at[TR::ACROSS];
  TR::template columns_at<BN>(cols_at, wn, i, kg);
  auto multiply = [&]() {
#pragma unroll
    for (int k = 0; k < BK; k += KS) {
      Frag xf[MT], wf[NTL];
#pragma unroll
      for (int m = 0; m < MT; ++m) xf[m] = TR::template along<BK>(sA, along_at, wm + 16 * m, k);
#pragma unroll
      for (int n = 0; n < NTL; ++n)
        wf[n] = NN ? TR::template columns<BN>(sB, cols_at, k, n) : TR::template along<BK>(sB, along_at, wn + 16 * n, k);
#pragma unroll
      for (int n = 0; n < NTL; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = TR::mfma(wf[n], xf[m], acc[n][m]);
    }
  };
  // (all groups take the same number of steps, with zeros past the end)
  const int from = group * each, steps = min(a.k, each);
  load(ra0, rb0, from);
  if (BK < steps) load(ra1, rb1, from + BK);
  for (int k0 = 0; k0 < steps; k0 += 2 * BK) {
    __syncthreads();
    put(ra0, rb0);
    __syncthreads();
    if (k0 + 2 * BK < steps) load(ra0, rb0, from + k0 + 2 * BK);
    multiply();
    if (k0 + BK < steps) {
      __syncthreads();
      put(ra1, rb1);
      __syncthreads();
      if (k0 + 3 * BK < steps) load(ra1, rb1, from + k0 + 3 * BK);
      multiply();
    }
  }
  if constexpr (G > 1) {
    static_assert((BM + BN) * BK * S >= NTL * MT * THREADS * 16, "a group's sums fit its tiles");
    __syncthreads();
    if (group > 0)
#pragma unroll
      for (int n = 0; n < NTL; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) reinterpret_cast<f32x4*>(sA)[(n * MT + m) * THREADS + tid] = acc[n][m];
    __syncthreads();
    if (group == 0)
#pragma unroll
      for (int other = 1; other < G; ++other)
#pragma unroll
        for (int n = 0; n < NTL; ++n)
#pragma unroll
          for (int m = 0; m < MT; ++m) acc[n][m] += reinterpret_cast<const f32x4*>(sA + other * (BM + BN) * BK)[(n * MT + m) * THREADS + tid];
  }
  // (what the other groups do from here on only helps the first one's loads)
  add_adapters<TR, BM, BN, MT, NTL, THREADS * G, AL>(a, m0, n0, rows, wm, wn, tiles, tiles + BM * BK, acc);
  if (group == 0) store_rows<TR, MT, NTL, AL>(a, m0, n0, rows, wm, wn, acc);
}

// Many rows and columns in bfloat16: tiles of BM (256 or 128) x 256, eight waves of BM / 2 x 64 each.  A step of 64 indexes goes from memory straight into
// LDS (two buffers: the next step's loads run through a whole step's 64 products a wave), with one barrier a step.  A
// load writes 16 bytes a lane side by side, so the permutation of a tile's units is made on the side of memory: lane l fetches the
// unit that belongs at place l.  Rows and columns past the ends repeat the last ones and are not stored.  The matrix cores bound it: 8192
// rows, 4096 x 4096, with the adapters, under the profiler: 269 us at least, 284 in the median (1.02 and 0.97 PFLOP/s); 4096 rows, 2048 x 2048,
// tiles of 128: 42 us (0.81).
constexpr int WIDE = 256, WIDE_THREADS = 512;
template <int BM, bool NN>
__global__ __launch_bounds__(WIDE_THREADS, 2) void k_project_wide(const ProjectArgs a, int tiles_m, int tiles_n) {
  using TR = Bf16;
  using T = TR::T;
  constexpr int BK = 64, KS = 32, MT = BM / 32, NTL = 4, PASSES_A = BM * BK / 8 / WIDE_THREADS, PASSES = WIDE * BK / 8 / WIDE_THREADS;
  __shared__ __align__(16) T sA0[BM * BK];
  __shared__ __align__(16) T sB0[WIDE * BK];
  __shared__ __align__(16) T sA1[BM * BK];
  __shared__ __align__(16) T sB1[WIDE * BK];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, kg = lane >> 4;
  const int wm = wave / 4 * (BM / 2), wn = wave % 4 * 64;
  // a die (workgroup number modulo 8) takes tiles side by side: columns of eight tiles, so that what it reads stays in its L2
  int bm, bn;
  {
    const int count = tiles_m * tiles_n, die = blockIdx.x % NUM_XCD, nth = blockIdx.x / NUM_XCD;
    const int each = count / NUM_XCD, more = count % NUM_XCD;
    const int tile = die * each + min(die, more) + nth;
    const int group = tile / (8 * tiles_n), in = tile - group * 8 * tiles_n, high = min(8, tiles_m - 8 * group);
    bm = 8 * group + in % high;
    bn = in / high;
  }
  const int64_t m0 = (int64_t)bm * BM;
  const int n0 = bn * WIDE;
  const int rows = (int)min((int64_t)BM, a.q.n_rows - m0);
  const T* x = static_cast<const T*>(a.x) + m0 * a.x_stride;
  const T* W = static_cast<const T*>(a.W) + (NN ? (int64_t)0 : (int64_t)n0 * a.k);
  const int cols = min(WIDE, a.n - n0);
  const T *fa[PASSES_A], *fb[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int c = tid + p * WIDE_THREADS, row = c / 8, unit = c % 8 ^ swizzle_bytes<128>(row);
    if (p < PASSES_A) fa[p] = x + (int64_t)min(row, rows - 1) * a.x_stride + 8 * unit;
    if constexpr (NN) {
      const int r = c / 32, u = c % 32 ^ swizzle_bytes<512>(r);
      fb[p] = W + (int64_t)r * a.n + n0 + min(8 * u, cols - 8);
    } else {
      fb[p] = W + (int64_t)min(row, cols - 1) * a.k + 8 * unit;
    }
  }
  const int64_t step_b = NN ? (int64_t)BK * a.n : BK;
  typedef __attribute__((address_space(1))) const void* Global;
  typedef __attribute__((address_space(3))) void* Lds;
  auto stage = [&](T* sA, T* sB) {
#pragma unroll
    for (int p = 0; p < PASSES_A; ++p) {
      __builtin_amdgcn_global_load_lds((Global)fa[p], (Lds)(sA + (p * WIDE_THREADS + wave * 64) * 8), 16, 0, 0);
      fa[p] += BK;
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      __builtin_amdgcn_global_load_lds((Global)fb[p], (Lds)(sB + (p * WIDE_THREADS + wave * 64) * 8), 16, 0, 0);
      fb[p] += step_b;
    }
  };
  f32x4 acc[NTL][MT];
#pragma unroll
  for (int n = 0; n < NTL; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int along_at = TR::along_at<BK>(i, kg);
  int cols_at[TR::ACROSS];
  TR::columns_at<WIDE>(cols_at, wn, i, kg);
  auto multiply = [&](const T* sA, const T* sB) {
#pragma unroll
    for (int k = 0; k < BK; k += KS) {
      TR::Frag xf[MT], wf[NTL];
#pragma unroll
      for (int n = 0; n < NTL; ++n) wf[n] = NN ? TR::columns<WIDE>(sB, cols_at, k, n) : TR::along<BK>(sB, along_at, wn + 16 * n, k);
#pragma unroll
      for (int m = 0; m < MT; ++m) xf[m] = TR::along<BK>(sA, along_at, wm + 16 * m, k);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NTL; ++n) acc[n][m] = TR::mfma(wf[n], xf[m], acc[n][m]);
    }
  };
  const int steps = a.k / BK;
  stage(sA0, sB0);
  for (int s = 0; s < steps; s += 2) {
    __syncthreads();                     // (waits for this step's loads, too)
    if (s + 1 < steps) stage(sA1, sB1);
    multiply(sA0, sB0);
    if (s + 1 < steps) {
      __syncthreads();
      if (s + 2 < steps) stage(sA0, sB0);
      multiply(sA1, sB1);
    }
  }
  add_adapters<TR, BM, WIDE, MT, NTL, WIDE_THREADS, true>(a, m0, n0, rows, wm, wn, sA0, sB0, acc);
  store_rows<TR, MT, NTL, true>(a, m0, n0, rows, wm, wn, acc);
}

// Few rows (up to 16 RT): W is read once, by 16 of its rows a workgroup whose eight waves split the contraction.  The wait for its
// loads bounds it: 24 rows, 2048 x 2048, bfloat16: 8 us (8.4 MB).
constexpr int FEW_THREADS = 512;
template <class TR, int RT, bool AL>
__global__ __launch_bounds__(FEW_THREADS) void k_project_few(const ProjectArgs a) {
  using T = typename TR::T;
  using Frag = typename TR::Frag;
  constexpr int WAVES = FEW_THREADS / 64, ROWS = 16 * RT;
  __shared__ float red[WAVES][ROWS][17];
  __shared__ int sAdapter[ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, kg = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const int rows = (int)min((int64_t)ROWS, a.q.n_rows);
  const T* W = static_cast<const T*>(a.W) + (int64_t)(n0 + i) * a.k;
  const T* x = static_cast<const T*>(a.x) + i * a.x_stride;
  f32x4 acc[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
  const u32x4 none = {0, 0, 0, 0};
  // whose adapter a row has
  for (int r = wave; r < rows; r += WAVES) {
    const int s = owner_of(a.q.off, a.q.n_seqs, r);
    if (lane == 0) sAdapter[r] = s < 0 ? -1 : adapter(a.q, s);
  }
  constexpr int RUN = RT == 4 ? 4 : 8;          // steps side by side of a wave, whose loads are on the way at once
  for (int k0 = wave * RUN * TR::KS; k0 < a.k; k0 += WAVES * RUN * TR::KS) {
    u32x4 w[RUN], v[RUN][RT];
#pragma unroll
    for (int u = 0; u < RUN; ++u) {
      const int col = k0 + u * TR::KS + kg * TR::E;
      w[u] = n0 + i < a.n ? run16<TR, AL, true>(W, col, a.k) : none;
#pragma unroll
      for (int r = 0; r < RT; ++r) v[u][r] = 16 * r + i < rows ? run16<TR, AL, true>(x + 16 * r * a.x_stride, col, a.k) : none;
    }
#pragma unroll
    for (int u = 0; u < RUN; ++u)
#pragma unroll
      for (int r = 0; r < RT; ++r) acc[r] = TR::mfma(__builtin_bit_cast(Frag, w[u]), __builtin_bit_cast(Frag, v[u][r]), acc[r]);
  }
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) red[wave][16 * r + i][4 * kg + j] = acc[r][j];
  __syncthreads();
  for (int e = tid; e < rows * 16; e += FEW_THREADS) {
    const int row = e >> 4, col = e & 15;
    if (n0 + col >= a.n) continue;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += red[w][row][col];
    const int ad = sAdapter[row];
    if (ad >= 0) {
      const T* up = static_cast<const T*>(a.up) + (int64_t)ad * a.rank * a.n + n0 + col;
      const float* low = a.low + row * a.padded;
#pragma unroll 8
      for (int j = 0; j < a.rank; ++j) sum = fmaf(low[j], TR::get(up[(int64_t)j * a.n]), sum);
    }
    static_cast<T*>(a.y)[(int64_t)row * a.n + n0 + col] = TR::put(sum);
  }
}

// Few columns (up to 64) and a rank up to 32: both products with x in one pass over it.  A workgroup takes 32 rows; its waves split
// the width as k_low's do, with W's rows and those of the adapter as operands side by side.  Further requests in the same rows
// take further passes, for their adapters alone.  L2 and the matrix cores bound it: 32768 rows of 512, 20 columns, rank 4, float32: 32 to 37 us
// (67 MB, 2.0 TB/s, matrix cores busy a third of it).  With many short requests the passes are what counts: 256 rows of 512, 64 columns,
// 118 us in 256 requests, 15 in 16.
constexpr int NARROW_ROWS = 32;
template <class TR, bool AL, int WT, int JT>
__global__ __launch_bounds__(THREADS) void k_project_narrow(const ProjectArgs a, const void* A_all, float scale) {
  using T = typename TR::T;
  using Frag = typename TR::Frag;
  constexpr int WAVES = THREADS / 64, RT = NARROW_ROWS / 16, TT = WT + JT, RUN = TT > 3 ? 2 : 4;
  __shared__ float red[WAVES][NARROW_ROWS][16 * TT + 1];
  __shared__ float sH[NARROW_ROWS][16 * JT + 1], sY[NARROW_ROWS][16 * WT + 1];
  __shared__ int sAdapter[NARROW_ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, kg = lane >> 4;
  const int64_t m0 = (int64_t)blockIdx.x * NARROW_ROWS;
  const int rows = (int)min((int64_t)NARROW_ROWS, a.q.n_rows - m0);
  const T* x = static_cast<const T*>(a.x) + (m0 + i) * a.x_stride;
  const T* W = static_cast<const T*>(a.W) + (int64_t)i * a.k;
  if (tid < NARROW_ROWS) sAdapter[tid] = -1;
  const u32x4 none = {0, 0, 0, 0};
  bool first = true;
  auto pass = [&](int ad, int rlo, int rhi) {
    const T* A = static_cast<const T*>(A_all) + ((int64_t)max(ad, 0) * a.rank + i) * a.k;
    f32x4 acc[TT][RT];
#pragma unroll
    for (int n = 0; n < TT; ++n)
#pragma unroll
      for (int r = 0; r < RT; ++r) acc[n][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k0 = wave * RUN * TR::KS; k0 < a.k; k0 += WAVES * RUN * TR::KS) {
      u32x4 xv[RUN][RT], wv[RUN][TT];
#pragma unroll
      for (int u = 0; u < RUN; ++u) {
        const int col = k0 + u * TR::KS + kg * TR::E;
#pragma unroll
        for (int r = 0; r < RT; ++r) xv[u][r] = 16 * r + i < rows ? run16<TR, AL, true>(x + 16 * r * a.x_stride, col, a.k) : none;
#pragma unroll
        for (int n = 0; n < WT; ++n) wv[u][n] = first && 16 * n + i < a.n ? run16<TR, AL, true>(W + (int64_t)(16 * n) * a.k, col, a.k) : none;
#pragma unroll
        for (int n = 0; n < JT; ++n) wv[u][WT + n] = ad >= 0 && 16 * n + i < a.rank ? run16<TR, AL, true>(A + (int64_t)(16 * n) * a.k, col, a.k) : none;
      }
#pragma unroll
      for (int u = 0; u < RUN; ++u)
#pragma unroll
        for (int n = 0; n < TT; ++n)
#pragma unroll
          for (int r = 0; r < RT; ++r) acc[n][r] = TR::mfma(__builtin_bit_cast(Frag, wv[u][n]), __builtin_bit_cast(Frag, xv[u][r]), acc[n][r]);
    }
    __syncthreads();                       // (what an earlier pass left in red has been read)
#pragma unroll
    for (int n = 0; n < TT; ++n)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) red[wave][16 * r + i][16 * n + 4 * kg + j] = acc[n][r][j];
    __syncthreads();
    for (int e = tid; e < NARROW_ROWS * 16 * TT; e += THREADS) {
      const int row = e / (16 * TT), col = e % (16 * TT);
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) sum += red[w][row][col];
      if (col < 16 * WT) {
        if (first) sY[row][col] = sum;
      } else if (ad >= 0 && row >= rlo && row < rhi) {
        sH[row][col - 16 * WT] = scale * sum;
        if (col == 16 * WT) sAdapter[row] = ad;
      }
    }
    first = false;
  };
  for (int at = 0; at < a.q.n_seqs; at += 64) {
    const int mine = at + lane;
    int64_t lo = 0, hi = 0;
    int ad = -1;
    if (mine < a.q.n_seqs) {
      lo = clamped(a.q.off[mine], m0, m0 + rows);
      hi = clamped(a.q.off[mine + 1], lo, m0 + rows);
      ad = adapter(a.q, mine);
    }
    uint64_t some = __ballot(hi > lo && ad >= 0);
    while (some) {
      const int from = __builtin_ctzll(some);
      some &= some - 1;
      pass(__shfl(ad, from), __shfl((int)(lo - m0), from), __shfl((int)(hi - m0), from));
    }
  }
  if (first) pass(-1, 0, 0);
  __syncthreads();
  for (int e = tid; e < rows * a.n; e += THREADS) {
    const int row = e / a.n, col = e - row * a.n, ad = sAdapter[row];
    float sum = sY[row][col];
    if (ad >= 0) {
      const T* up = static_cast<const T*>(a.up) + (int64_t)ad * a.rank * a.n + col;
#pragma unroll 4
      for (int j = 0; j < a.rank; ++j) sum = fmaf(sH[row][j], TR::get(up[(int64_t)j * a.n]), sum);
    }
    static_cast<T*>(a.y)[(m0 + row) * a.n + col] = TR::put(sum);
  }
}

// ---- dA_a = sum u^T x, dB_a = sum h^T dy ----------------------------------------------------------------------------------
struct GradSide {
  const void* x;           // rows x width
  const float* low;        // rows x padded rank
  void* out;               // adapters x rank x width
  float* part;             // the same in float32 for each part of the rows, or null: there is one
  int64_t x_stride;
  int width, tiles;        // column tiles
};
struct GradArgs {
  GradSide side[2];
  Requests q;
  int rank, padded;
  int64_t per;             // rows of a part
};

constexpr int GRAD_COLS = 128, GRAD_ROWS = 64;

// A workgroup takes 128 columns of one adapter's gradient and a part of the rows, and of these the requests that have the adapter.
// The wait for 64 rows at a time bounds it: 4096 rows, 2048 + 2048 columns, rank 16, 8 adapters, bfloat16: 22 us (34 MB), and
// 4 for the sum over two parts.
template <class TR, int JT, bool AL>
__global__ __launch_bounds__(THREADS) void k_adapter_grad(const GradArgs a) {
  using T = typename TR::T;
  using Frag = typename TR::Frag;
  constexpr int KS = TR::KS, E = TR::E, PAD = 16 / sizeof(T), LDX = GRAD_COLS + PAD, LDJ = 16 * JT + PAD;
  constexpr int X = GRAD_ROWS * GRAD_COLS / E / THREADS;
  __shared__ __align__(16) T sX[GRAD_ROWS * LDX];
  __shared__ __align__(16) T sL[TR::PARTS][GRAD_ROWS * LDJ];
  const int side = (int)blockIdx.x < a.side[0].tiles ? 0 : 1;
  const GradSide& sd = a.side[side];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, kg = lane >> 4;
  const int n0 = (blockIdx.x - (side ? a.side[0].tiles : 0)) * GRAD_COLS, ad = blockIdx.y;
  const int64_t p0 = blockIdx.z * a.per, p1 = min(a.q.n_rows, p0 + a.per);
  const T* x = static_cast<const T*>(sd.x);
  f32x4 acc[2][JT];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int j = 0; j < JT; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int at = 0; at < a.q.n_seqs; at += 64) {
    const int mine = at + lane;
    int64_t lo = 0, hi = 0;
    if (mine < a.q.n_seqs && adapter(a.q, mine) == ad) {
      lo = clamped(a.q.off[mine], p0, p1);
      hi = clamped(a.q.off[mine + 1], lo, p1);
    }
    uint64_t some = __ballot(hi > lo);
    while (some) {
      const int from = __builtin_ctzll(some);
      some &= some - 1;
      const int64_t rlo = __shfl((long long)lo, from), rhi = __shfl((long long)hi, from);
      u32x4 v[X];
      f32x4 w[JT];
      auto load = [&](int64_t r0) {
        const int rows = (int)min((int64_t)GRAD_ROWS, rhi - r0);
#pragma unroll
        for (int p = 0; p < X; ++p) {
          const int c = tid + p * THREADS, row = c / (GRAD_COLS / E), col = c % (GRAD_COLS / E) * E;
          v[p] = row < rows ? run16<TR, AL>(x + (r0 + row) * sd.x_stride, n0 + col, sd.width) : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int p = 0; p < JT; ++p) {
          const int c = tid + p * THREADS, row = c / (4 * JT), col = c % (4 * JT) * 4;
          w[p] = row < rows && col < a.padded ? *reinterpret_cast<const f32x4*>(sd.low + (r0 + row) * a.padded + col) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
      };
      load(rlo);
      for (int64_t r0 = rlo; r0 < rhi; r0 += GRAD_ROWS) {
        __syncthreads();
#pragma unroll
        for (int p = 0; p < X; ++p) {
          const int c = tid + p * THREADS;
          *reinterpret_cast<u32x4*>(sX + c / (GRAD_COLS / E) * LDX + c % (GRAD_COLS / E) * E) = v[p];
        }
#pragma unroll
        for (int p = 0; p < JT; ++p) {
          const int c = tid + p * THREADS, row = c / (4 * JT), col = c % (4 * JT) * 4;
          typename TR::Four parts[TR::PARTS];
          exact_parts(w[p], parts, TR{});
#pragma unroll
          for (int x = 0; x < TR::PARTS; ++x) *reinterpret_cast<typename TR::Four*>(sL[x] + row * LDJ + col) = parts[x];
        }
        __syncthreads();
        if (r0 + GRAD_ROWS < rhi) load(r0 + GRAD_ROWS);
#pragma unroll
        for (int k = 0; k < GRAD_ROWS; k += KS) {
          Frag xf[2], finite[2];
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            xf[m] = TR::col_frag(sX, LDX, k, 32 * wave + 16 * m, i, kg);
            finite[m] = finite_frag(xf[m], TR{});
          }
#pragma unroll
          for (int part = 0; part < TR::PARTS; ++part)
#pragma unroll
            for (int j = 0; j < JT; ++j) {
              const Frag lf = TR::col_frag(sL[part], LDJ, k, 16 * j, i, kg);
#pragma unroll
              for (int m = 0; m < 2; ++m) acc[m][j] = TR::mfma(part ? finite[m] : xf[m], lf, acc[m][j]);
            }
        }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < JT; ++j) {
    const int row = 16 * j + i;
    if (row >= a.rank) continue;
    const int64_t at = ((int64_t)ad * a.rank + row) * sd.width;
    float* part = sd.part ? sd.part + (int64_t)blockIdx.z * a.q.n_adapters * a.rank * sd.width + at : nullptr;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int col = n0 + 32 * wave + 16 * m + 4 * kg + r;
        if (col >= sd.width) continue;
        if (part) part[col] = acc[m][j][r];
        else static_cast<T*>(sd.out)[at + col] = TR::put(acc[m][j][r]);
      }
  }
}

struct SumArgs {
  const float* part[2];
  void* out[2];
  int64_t count[2];
  int parts;
};
template <class TR>
__global__ __launch_bounds__(THREADS) void k_sum_grads(const SumArgs a) {
  const int64_t e = (int64_t)blockIdx.x * THREADS + threadIdx.x, n = a.count[blockIdx.y];
  if (e >= n) return;
  const float* p = a.part[blockIdx.y] + e;
  float sum = 0.f;
#pragma unroll 8
  for (int k = 0; k < a.parts; ++k) sum += p[k * n];
  static_cast<typename TR::T*>(a.out[blockIdx.y])[e] = TR::put(sum);
}

// ---- host -----------------------------------------------------------------------------------------------------------------
int check(const nugpr_adapter* p) {
  if (!p) { set_error("problem is null"); return NUGPR_ERR_INVALID; }
  if (p->dtype != NUGPR_FLOAT32 && p->dtype != NUGPR_BFLOAT16) { set_error("dtype must be NUGPR_FLOAT32 or NUGPR_BFLOAT16"); return NUGPR_ERR_INVALID; }
  if (p->dim_in < 1 || p->dim_in > 65536 || p->dim_out < 1 || p->dim_out > 65536) { set_error("dim_in and dim_out must be 1..65536"); return NUGPR_ERR_INVALID; }
  if (p->rank < 1 || p->rank > 128) { set_error("rank must be 1..128"); return NUGPR_ERR_INVALID; }
  if (p->n_adapters < 0 || p->n_adapters > 65535) { set_error("n_adapters must be 0..65535"); return NUGPR_ERR_INVALID; }
  if (p->n_rows < 0 || p->n_rows > (int64_t)4 << 20) { set_error("n_rows must be 0..2^22"); return NUGPR_ERR_INVALID; }
  if (p->n_seqs < 0 || p->n_seqs > 1 << 22) { set_error("n_seqs must be 0..2^22"); return NUGPR_ERR_INVALID; }
  return NUGPR_OK;
}

size_t value_size(const nugpr_adapter* p) { return p->dtype == NUGPR_BFLOAT16 ? 2 : 4; }
int padded_rank(const nugpr_adapter* p) { const int k = p->dtype == NUGPR_BFLOAT16 ? 32 : 16; return (p->rank + k - 1) / k * k; }
size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }
size_t low_bytes(const nugpr_adapter* p) { return rounded((size_t)p->n_rows * padded_rank(p) * sizeof(float)); }
int grad_tiles(int width) { return (width + GRAD_COLS - 1) / GRAD_COLS; }
// parts of the rows in the sums over them: about 512 workgroups, of 256 rows at least
int grad_parts(const nugpr_adapter* p) {
  const int64_t tiles = (int64_t)(grad_tiles(p->dim_in) + grad_tiles(p->dim_out)) * p->n_adapters;
  if (tiles == 0) return 1;
  int64_t parts = 512 / tiles;
  if (parts > p->n_rows / 256) parts = p->n_rows / 256;
  return parts < 1 ? 1 : (int)parts;
}
size_t part_bytes(const nugpr_adapter* p, int width) {
  const int parts = grad_parts(p);
  return parts == 1 ? 0 : rounded((size_t)parts * p->n_adapters * p->rank * width * sizeof(float));
}

bool wide(const void* x, int64_t stride, size_t value) {
  return !(reinterpret_cast<uintptr_t>(x) & 15u) && stride % (16 / (int64_t)value) == 0;
}

int check_call(const nugpr_adapter* p, size_t need) {
  if (!std::isfinite((float)p->scale)) { set_error("scale must be finite in float32"); return NUGPR_ERR_INVALID; }
  const size_t z = value_size(p);
  if (p->n_seqs > 0 && !p->seq_offsets) { set_error("seq_offsets is null"); return NUGPR_ERR_INVALID; }
  if (!p->W || (p->n_adapters > 0 && (!p->A || !p->B))) { set_error("W, A or B is null"); return NUGPR_ERR_INVALID; }
  if ((reinterpret_cast<uintptr_t>(p->W) | reinterpret_cast<uintptr_t>(p->A) | reinterpret_cast<uintptr_t>(p->B)) % z) {
    set_error("W, A or B misaligned");
    return NUGPR_ERR_INVALID;
  }
  if (need && (!p->workspace || (reinterpret_cast<uintptr_t>(p->workspace) & 255u))) { set_error("workspace is null or not 256-byte aligned"); return NUGPR_ERR_WORKSPACE; }
  if (p->workspace_bytes < need) { set_error("workspace smaller than nugpr_adapter_workspace_bytes()"); return NUGPR_ERR_WORKSPACE; }
  return NUGPR_OK;
}

int check_rows(const void* x, int64_t stride, const char* name, size_t z) {
  if (!x) { set_error(std::string(name) + " is null"); return NUGPR_ERR_INVALID; }
  if (reinterpret_cast<uintptr_t>(x) % z) { set_error(std::string(name) + " misaligned"); return NUGPR_ERR_INVALID; }
  if (stride < 0) { set_error(std::string(name) + ": negative stride"); return NUGPR_ERR_INVALID; }
  return NUGPR_OK;
}

Requests requests(const nugpr_adapter* p) {
  return Requests{p->seq_offsets, p->adapter_of, p->n_rows, p->n_adapters > 0 ? p->n_seqs : 0, p->n_adapters};
}

template <class TR, bool AL>
void launch_low(const LowArgs& a, int sides, hipStream_t s) {
  const unsigned items = (unsigned)((a.q.n_rows >> LOW_LOG2) + a.q.n_seqs);
  const int tiles = (a.rank + 15) / 16;
  // (so many waves that each has about two runs of loads, 4 to 16; few pieces: 16)
  const int width = sides > 1 ? max(a.side[0].width, a.side[1].width) : a.side[0].width, runs = width / (4 * TR::KS);
  int waves = items * sides < 512 || runs >= 24 ? 16 : runs >= 12 ? 8 : 4;
  if (tiles > 2 || items > 0xffffffffu / 1024) waves = min(waves, 8);      // (the threads of a launch are counted in 32 bits)
  const dim3 grid(items, sides), threads(64 * waves);
  const size_t lds = (size_t)waves * 16 * 16 * (tiles <= 1 ? 1 : tiles <= 2 ? 2 : tiles <= 4 ? 4 : 8) * sizeof(float);
  if (tiles <= 1) hipLaunchKernelGGL((k_low<TR, AL, 1>), grid, threads, lds, s, a);
  else if (tiles <= 2) hipLaunchKernelGGL((k_low<TR, AL, 2>), grid, threads, lds, s, a);
  else if (tiles <= 4) hipLaunchKernelGGL((k_low<TR, AL, 4>), grid, threads, lds, s, a);
  else hipLaunchKernelGGL((k_low<TR, AL, 8>), grid, threads, lds, s, a);
}

template <class TR, int BM, int BN, int WM, int WN, int G, bool NN, bool AL>
void launch_tiles(const ProjectArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_project<TR, BM, BN, WM, WN, G, NN, AL>), dim3((a.n + BN - 1) / BN, (unsigned)((a.q.n_rows + BM - 1) / BM)), dim3(THREADS * G), 0, s, a);
}

template <class TR, bool NN, bool AL>
void launch_project(const ProjectArgs& a, hipStream_t s) {
  if (!NN && a.q.n_rows <= 64) {
    const dim3 grid((a.n + 15) / 16);
    if (a.q.n_rows <= 16) hipLaunchKernelGGL((k_project_few<TR, 1, AL>), grid, dim3(FEW_THREADS), 0, s, a);
    else if (a.q.n_rows <= 32) hipLaunchKernelGGL((k_project_few<TR, 2, AL>), grid, dim3(FEW_THREADS), 0, s, a);
    else hipLaunchKernelGGL((k_project_few<TR, 4, AL>), grid, dim3(FEW_THREADS), 0, s, a);
    return;
  }
  if constexpr (TR::E == 8 && AL) {
    // (from 192 tiles on, three quarters of the compute units)
    const int64_t tn = (a.n + WIDE - 1) / WIDE, t256 = (a.q.n_rows + 255) / 256, t128 = (a.q.n_rows + 127) / 128;
    if (a.k % 64 == 0 && t256 * tn >= 192) {
      hipLaunchKernelGGL((k_project_wide<256, NN>), dim3((unsigned)(t256 * tn)), dim3(WIDE_THREADS), 0, s, a, (int)t256, (int)tn);
      return;
    }
    if (a.k % 64 == 0 && t128 * tn >= 192) {
      hipLaunchKernelGGL((k_project_wide<128, NN>), dim3((unsigned)(t128 * tn)), dim3(WIDE_THREADS), 0, s, a, (int)t128, (int)tn);
      return;
    }
  }
  // The fewer tiles there are, the smaller they are and the more groups share their contraction.  128 x 4096 rows and columns, contraction
  // 4096, 128 tiles of 64 x 64: 52 us with these, 36 with four groups, 31 with tiles of 32 x 32 as well; 512 x 2048, 2048 (256):
  // 29, 22, 30; with two groups 24; 2048 x 1024, 2048 (512): 31, 34, 48; 28.  In float32, whose products last longer, smaller tiles rather
  // than groups: 1501 x 500, 301 (192): 51, 51, 49; tiles of 32 x 32 with one group 43.
  const int64_t large = ((a.q.n_rows + 127) / 128) * ((a.n + 127) / 128), small = ((a.q.n_rows + 63) / 64) * ((a.n + 63) / 64);
  if (large >= 256) return launch_tiles<TR, 128, 128, 2, 2, 1, NN, AL>(a, s);
  if (small <= 128) return launch_tiles<TR, 32, 32, 2, 2, 4, NN, AL>(a, s);
  if constexpr (TR::E == 8) {
    if (small <= 256) return launch_tiles<TR, 64, 64, 2, 2, 4, NN, AL>(a, s);
    if (small <= 512) return launch_tiles<TR, 64, 64, 2, 2, 2, NN, AL>(a, s);
  } else {
    if (small <= 256) return launch_tiles<TR, 32, 32, 2, 2, 1, NN, AL>(a, s);
    if (a.n <= 32) return launch_tiles<TR, 128, 32, 4, 1, 1, NN, AL>(a, s);
  }
  launch_tiles<TR, 64, 64, 2, 2, 1, NN, AL>(a, s);
}

template <class TR, bool AL>
void launch_grad(const GradArgs& a, const SumArgs& sum, hipStream_t s) {
  const int tiles = (a.rank + 15) / 16;
  const dim3 grid(a.side[0].tiles + a.side[1].tiles, a.q.n_adapters, sum.parts);
  if (tiles <= 1) hipLaunchKernelGGL((k_adapter_grad<TR, 1, AL>), grid, dim3(THREADS), 0, s, a);
  else if (tiles <= 2) hipLaunchKernelGGL((k_adapter_grad<TR, 2, AL>), grid, dim3(THREADS), 0, s, a);
  else if (tiles <= 4) hipLaunchKernelGGL((k_adapter_grad<TR, 4, AL>), grid, dim3(THREADS), 0, s, a);
  else hipLaunchKernelGGL((k_adapter_grad<TR, 8, AL>), grid, dim3(THREADS), 0, s, a);
  if (sum.parts > 1) {
    const int64_t most = sum.count[0] > sum.count[1] ? sum.count[0] : sum.count[1];
    hipLaunchKernelGGL((k_sum_grads<TR>), dim3((unsigned)((most + THREADS - 1) / THREADS), 2), dim3(THREADS), 0, s, sum);
  }
}

template <class TR, bool AL, int WT>
void launch_narrow(const ProjectArgs& a, const nugpr_adapter* p, hipStream_t s) {
  const dim3 grid((unsigned)((a.q.n_rows + NARROW_ROWS - 1) / NARROW_ROWS));
  if (p->rank <= 16) hipLaunchKernelGGL((k_project_narrow<TR, AL, WT, 1>), grid, dim3(THREADS), 0, s, a, p->A, (float)p->scale);
  else hipLaunchKernelGGL((k_project_narrow<TR, AL, WT, 2>), grid, dim3(THREADS), 0, s, a, p->A, (float)p->scale);
}

template <class TR, bool AL>
int run_forward(const nugpr_adapter* p, const void* x, int64_t x_stride, void* y, hipStream_t s) {
  const Requests q = requests(p);
  // (one pass over x; each further request with rows in a workgroup's 32 costs it a pass more, which takes the longer the wider x is, so that wide
  // x with fewer rows than keep the card busy go the general way: 2048 rows of 2048, 64 columns: 21 us, the general way 16; 32768 rows of 512, 20 columns, float32: 34 and 59)
  if (p->dim_out <= 64 && p->rank <= 32 && q.n_rows > 64 && (p->dim_in <= 1024 || q.n_rows >= 16384)) {
    const ProjectArgs a{x, p->W, p->B, nullptr, y, x_stride, q, p->dim_in, p->dim_out, p->rank, padded_rank(p)};
    if (p->dim_out <= 16) launch_narrow<TR, AL, 1>(a, p, s);
    else if (p->dim_out <= 32) launch_narrow<TR, AL, 2>(a, p, s);
    else launch_narrow<TR, AL, 4>(a, p, s);
    NUGPR_HIP(hipGetLastError());
    return NUGPR_OK;
  }
  LowArgs l{};
  l.q = q; l.scale = (float)p->scale; l.rank = p->rank; l.padded = padded_rank(p);
  l.side[0] = LowSide{x, p->A, static_cast<float*>(p->workspace), x_stride, p->dim_in};
  if (q.n_seqs > 0) launch_low<TR, AL>(l, 1, s);
  const ProjectArgs a{x, p->W, p->B, l.side[0].low, y, x_stride, q, p->dim_in, p->dim_out, p->rank, l.padded};
  launch_project<TR, false, AL>(a, s);
  NUGPR_HIP(hipGetLastError());
  return NUGPR_OK;
}

template <class TR, bool AL>
int run_backward(const nugpr_adapter* p, const void* x, int64_t x_stride, const void* dy, int64_t dy_stride, void* dx, void* dA, void* dB,
                 hipStream_t s) {
  const Requests q = requests(p);
  char* ws = static_cast<char*>(p->workspace);
  const size_t each = low_bytes(p);
  float *low = reinterpret_cast<float*>(ws), *up = reinterpret_cast<float*>(ws + each);
  LowArgs l{};
  l.q = q; l.scale = (float)p->scale; l.rank = p->rank; l.padded = padded_rank(p);
  l.side[0] = LowSide{x, p->A, low, x_stride, p->dim_in};
  l.side[1] = LowSide{dy, p->B, up, dy_stride, p->dim_out};
  if (q.n_seqs > 0 && q.n_rows > 0) launch_low<TR, AL>(l, 2, s);
  if (dx && q.n_rows > 0) {
    const ProjectArgs a{dy, p->W, p->A, up, dx, dy_stride, q, p->dim_out, p->dim_in, p->rank, l.padded};
    launch_project<TR, true, AL>(a, s);
  }
  if (p->n_adapters > 0) {
    GradArgs g{};
    SumArgs sum{};
    const int parts = grad_parts(p);
    float* pa = reinterpret_cast<float*>(ws + 2 * each);
    float* pb = reinterpret_cast<float*>(ws + 2 * each + part_bytes(p, p->dim_in));
    g.q = q; g.rank = p->rank; g.padded = l.padded;
    g.per = (q.n_rows + parts - 1) / parts;
    g.side[0] = GradSide{x, up, dA, parts > 1 ? pa : nullptr, x_stride, p->dim_in, grad_tiles(p->dim_in)};
    g.side[1] = GradSide{dy, low, dB, parts > 1 ? pb : nullptr, dy_stride, p->dim_out, grad_tiles(p->dim_out)};
    sum.parts = parts;
    sum.part[0] = pa; sum.part[1] = pb; sum.out[0] = dA; sum.out[1] = dB;
    sum.count[0] = (int64_t)p->n_adapters * p->rank * p->dim_in;
    sum.count[1] = (int64_t)p->n_adapters * p->rank * p->dim_out;
    launch_grad<TR, AL>(g, sum, s);
  }
  NUGPR_HIP(hipGetLastError());
  return NUGPR_OK;
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

size_t nugpr_adapter_workspace_bytes(const nugpr_adapter* p, int32_t backward) {
  if (check(p) != NUGPR_OK) return 0;
  return 256 + (backward ? 2 * low_bytes(p) + part_bytes(p, p->dim_in) + part_bytes(p, p->dim_out) : low_bytes(p));
}

int nugpr_adapter_forward(const nugpr_adapter* p, const void* x, int64_t x_stride, void* y, void* stream) {
  NUGPR_TRY(check(p));
  NUGPR_TRY(check_call(p, low_bytes(p)));
  if (p->n_rows == 0) return NUGPR_OK;
  const size_t z = value_size(p);
  NUGPR_TRY(check_rows(x, x_stride, "x", z));
  NUGPR_TRY(check_rows(y, p->dim_out, "y", z));
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool al = wide(x, x_stride, z) && wide(p->W, p->dim_in, z) && wide(p->A, p->dim_in, z) && wide(p->B, p->dim_out, z) && wide(y, p->dim_out, z);
  if (p->dtype == NUGPR_BFLOAT16) return al ? run_forward<Bf16, true>(p, x, x_stride, y, s) : run_forward<Bf16, false>(p, x, x_stride, y, s);
  return al ? run_forward<F32, true>(p, x, x_stride, y, s) : run_forward<F32, false>(p, x, x_stride, y, s);
}

int nugpr_adapter_backward(const nugpr_adapter* p, const void* x, int64_t x_stride, const void* d_y, int64_t dy_stride, void* dx, void* dA,
                           void* dB, void* stream) {
  NUGPR_TRY(check(p));
  NUGPR_TRY(check_call(p, 2 * low_bytes(p) + part_bytes(p, p->dim_in) + part_bytes(p, p->dim_out)));
  const size_t z = value_size(p);
  if (p->n_rows > 0) {
    NUGPR_TRY(check_rows(x, x_stride, "x", z));
    NUGPR_TRY(check_rows(d_y, dy_stride, "d_y", z));
  }
  if (p->n_adapters > 0) {
    NUGPR_TRY(check_rows(dA, p->dim_in, "dA", z));
    NUGPR_TRY(check_rows(dB, p->dim_out, "dB", z));
  }
  if (dx) NUGPR_TRY(check_rows(dx, p->dim_in, "dx", z));
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool al = wide(x, x_stride, z) && wide(d_y, dy_stride, z) && wide(p->W, p->dim_in, z) && wide(p->A, p->dim_in, z) &&
                  wide(p->B, p->dim_out, z) && wide(dx, p->dim_in, z);
  if (p->dtype == NUGPR_BFLOAT16)
    return al ? run_backward<Bf16, true>(p, x, x_stride, d_y, dy_stride, dx, dA, dB, s) : run_backward<Bf16, false>(p, x, x_stride, d_y, dy_stride, dx, dA, dB, s);
  return al ? run_backward<F32, true>(p, x, x_stride, d_y, dy_stride, dx, dA, dB, s) : run_backward<F32, false>(p, x, x_stride, d_y, dy_stride, dx, dA, dB, s);
}

}  // extern "C"
