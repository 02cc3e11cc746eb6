// Gradients of the selective scan (selective_scan.hip has the formulas): two walks over the rows.
//
// The first goes forward and keeps the states at every tile's begin; of a sequence's later spans it also finds what they add to the state and to the
// gradient before them (selective_scan.hip's k_scan_join then has the states and gradients at the spans' ends).  The second goes through
// the tiles from the last to the first: forward inside a tile, whose states and factors stay in registers, then back.
//
// G lanes have one channel, S of its states each, and a wave 64 / G channels, so that sums over a channel's states stay inside groups of neighbouring
// lanes and waves need not wait for each other; only B and C, and their gradients' sums over the workgroup's channels, pass between waves, with one
// barrier a tile and two buffers in turn.
#include "selective_scan.h"

namespace nugpr {

namespace {

// Lanes of a channel, waves of a workgroup, states of a lane.
template <int G_, int WAVES_, int S_>
struct Shape {
  static constexpr int G = G_, WAVES = WAVES_, S = S_;
  static constexpr int CW = 64 / G;               // channels of a wave
  static constexpr int CB = CW * WAVES;           // of a workgroup
  static constexpr int V = CW / 4;                // of a lane that takes up or stores rows: four lanes a row
  static constexpr int NS = G * S;                // places for a channel's states
  static constexpr int THREADS = 64 * WAVES;
  static constexpr int PAIRS = (TILE_ROWS * NS + THREADS - 1) / THREADS;      // values of a tile's B (and C) that a thread takes up
  static constexpr bool ROOM = G < 16;            // in LDS, for what only some lanes read
};

// A tile's rows as memory has them: V channels of one row, and PAIRS values of B and C.  OUT: what the gradients need beside the states.
template <class TR, class H, bool OUT>
struct Incoming {
  typedef typename TR::T T;
  Values<TR, H::V> x, dt, z, dy;
  T b[H::PAIRS], c[H::PAIRS];
  const T *px, *pdt, *pz, *pdy;                   // the lane's, of the tile that is loaded next
  int64_t row0;                                   // that tile's first row
  __device__ __forceinline__ void begin(const ScanArgs& a, const Place& p, int wave, int lane, int64_t first) {
    const int64_t row = first + lane / 4;
    const int at = p.channel + wave * H::CW + lane % 4 * H::V;
    px = static_cast<const T*>(a.x) + row * a.x_row + at;
    pdt = static_cast<const T*>(a.dt) + row * a.dt_row + at;
    if (OUT) pz = static_cast<const T*>(a.z) + row * a.z_row + at;
    if (OUT) pdy = static_cast<const T*>(a.dy) + row * a.dy_row + at;
    row0 = first;
  }
  // n_rows of the tile, then on by `way` tiles; valid: channels of the wave
  __device__ __forceinline__ void load(const ScanArgs& a, const Place& p, int lane, int n_rows, int valid, int way) {
    if (n_rows == TILE_ROWS && valid >= H::CW) {
      x.load_all(px);
      dt.load_all(pdt);
      if (OUT && a.z) z.load_all(pz);
      if (OUT) dy.load_all(pdy);
    } else {
      const int mine = lane / 4 < n_rows ? valid - lane % 4 * H::V : 0;
      x.load(px, mine);
      dt.load(pdt, mine);
      if (OUT && a.z) z.load(pz, mine);
      if (OUT) dy.load(pdy, mine);
    }
#pragma unroll
    for (int k = 0; k < H::PAIRS; ++k) {
      const int at = k * H::THREADS + threadIdx.x, row = at / H::NS, n = at % H::NS;
      b[k] = c[k] = T(0);
      if (row < n_rows && n < a.states) {
        b[k] = (static_cast<const T*>(a.B) + p.group * a.B_head + n)[(row0 + row) * a.B_row];
        if (OUT) c[k] = (static_cast<const T*>(a.C) + p.group * a.C_head + n)[(row0 + row) * a.C_row];
      }
    }
    const int64_t rows = (int64_t)way * TILE_ROWS;
    row0 += rows;
    px += rows * a.x_row;
    pdt += rows * a.dt_row;
    if (OUT) pz += rows * a.z_row;
    if (OUT) pdy += rows * a.dy_row;
  }
};

template <class H>
struct alignas(16) Tile {
  float2 du[H::WAVES][TILE_ROWS][H::CW];          // d and u, every wave's own
  float e[H::WAVES][TILE_ROWS][H::CW];
  // B, then C, two buffers of each; then as many zeros as lanes without a channel read in their place: d = u = e = 0 does not silence an infinity
  float rows[4 + (H::ROOM ? 3 : 0)][TILE_ROWS][H::NS];
  static constexpr int C = 2, NONE = 4;
};

// Rows and channels that there are not: d = u = e = 0, which leaves a state, and a gradient, as it is.
template <class TR, class H, bool OUT>
__device__ __forceinline__ void fill_tile(Tile<H>& tile, const ScanArgs& a, const Incoming<TR, H, OUT>& in, int wave, int lane, int buffer, int n_rows,
                                          int valid, const float* bias) {
  constexpr int V = H::V;
  const int r = lane / 4, col = lane % 4 * V;
  float d[V];
#pragma unroll
  for (int j = 0; j < V; ++j) d[j] = in.dt.get(j) + bias[j];
  if (a.softplus)
#pragma unroll
    for (int j = 0; j < V; ++j) d[j] = softplus_of<TR>(d[j]);
  if (n_rows < TILE_ROWS || valid < H::CW)
#pragma unroll
    for (int j = 0; j < V; ++j) d[j] = r < n_rows && col + j < valid ? d[j] : 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) tile.du[wave][r][col + j] = float2{d[j], d[j] * in.x.get(j)};
  if constexpr (OUT) {
    float e[V];
#pragma unroll
    for (int j = 0; j < V; ++j) e[j] = in.dy.get(j);
    if (a.z)
#pragma unroll
      for (int j = 0; j < V; ++j) e[j] *= in.z.get(j) * sigmoid_of<TR>(in.z.get(j));
#pragma unroll
    for (int j = 0; j < V; ++j) tile.e[wave][r][col + j] = e[j];
  }
#pragma unroll
  for (int k = 0; k < H::PAIRS; ++k) {
    const int at = k * H::THREADS + threadIdx.x;
    if (H::PAIRS * H::THREADS == TILE_ROWS * H::NS || at < TILE_ROWS * H::NS) {
      (&tile.rows[buffer][0][0])[at] = TR::get(in.b[k]);
      if (OUT) (&tile.rows[Tile<H>::C + buffer][0][0])[at] = TR::get(in.c[k]);
    }
  }
}

template <int S>
__device__ __forceinline__ void load_states(float (&h)[S], const float* from, int n) {
#pragma unroll
  for (int s = 0; s < S; ++s) h[s] = s < n ? from[s] : 0.f;
}
template <int S>
__device__ __forceinline__ void store_states(const float (&h)[S], float* to, int n) {
#pragma unroll
  for (int s = 0; s < S; ++s)
    if (s < n) to[s] = h[s];
}
template <int S>
__device__ __forceinline__ void read_states(float (&v)[S], const float* lds) {
  if constexpr (S == 4) {
    const float4 x = *reinterpret_cast<const float4*>(lds);
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
  } else {
    const float2 x = *reinterpret_cast<const float2*>(lds);
    v[0] = x.x; v[1] = x.y;
  }
}

// The lane's place in what the first walk keeps of a tile.
template <class H>
__device__ __forceinline__ float* kept(const ScanArgs& a, int64_t tile, int block) {
  return a.tiles + ((tile * a.blocks + block) * H::THREADS + threadIdx.x) * H::S;
}
__device__ __forceinline__ int64_t first_tile(const Place& p) { return p.piece.lo / TILE_ROWS + p.piece.seq + (p.from - p.piece.lo) / TILE_ROWS; }

// The first walk.  Factors multiply up over a span for what it adds to the gradient before it; of a sequence's first span that is not wanted, so that
// the walk of sequences that are not cut is the states' alone.  The vector pipe bounds it, busy 80 % of the time: 8 x 2048 rows, 2048 channels, 16 states,
// bfloat16: 172 us.
//
// EXACT: the states fill the lanes' places.  Else those that there are not stay zero (nothing is multiplied by a zero there, where an
// infinity would become NaN): `n` are the lane's.
template <class TR, class H, bool EXACT>
__global__ __launch_bounds__(H::THREADS) void k_scan_tiles(const ScanArgs a) {
  constexpr int S = H::S;
  __shared__ Tile<H> tile;
  const int item = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks;
  Place p;
  if (!find(a, item, block, p)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int ch = lane / H::G, group = lane % H::G, valid = p.valid - wave * H::CW;
  const bool live = ch < valid;
  const int n = live ? min(S, a.states - group * S) : 0;
  const int64_t each = (int64_t)a.dim * a.states, of_lane = (int64_t)(p.channel + wave * H::CW + ch) * a.states + group * S;
  float h[S], a2[S], product[S], g[S], bias[H::V];
  load_states(a2, a.A + of_lane, n);
#pragma unroll
  for (int s = 0; s < S; ++s) {
    a2[s] = rate_of(a2[s]);
    product[s] = 1.f;
    g[s] = 0.f;
  }
  const float* start = p.span == 0 && a.s_in ? a.s_in + p.piece.seq * each : nullptr;
  load_states(h, start + of_lane, start ? n : 0);
#pragma unroll
  for (int j = 0; j < H::V; ++j) {
    const int c = lane % 4 * H::V + j;
    bias[j] = a.bias && c < valid ? a.bias[p.channel + wave * H::CW + c] : 0.f;
  }
  float passed = 0.f;                              // sum of d
  // (a sequence's first span has no state before it whose gradient were wanted)
  auto walk = [&](auto later) __attribute__((always_inline)) {
    constexpr bool LATER = decltype(later)::value;
    int64_t number = first_tile(p);
    int buffer = 0;
    Incoming<TR, H, LATER> in;
    in.begin(a, p, wave, lane, p.from);
    if (p.from < p.to) in.load(a, p, lane, (int)min((int64_t)TILE_ROWS, p.to - p.from), valid, 1);
    for (int64_t t0 = p.from; t0 < p.to; t0 += TILE_ROWS, ++number, buffer ^= 1) {
      __builtin_memcpy(kept<H>(a, number, block), h, sizeof h);
      if (LATER && live && group == 0) a.tile_steps[number * a.dim + p.channel + wave * H::CW + ch] = passed;
      fill_tile(tile, a, in, wave, lane, buffer, (int)min((int64_t)TILE_ROWS, p.to - t0), valid, bias);
      __syncthreads();
      if (t0 + TILE_ROWS < p.to) in.load(a, p, lane, (int)min((int64_t)TILE_ROWS, p.to - t0 - TILE_ROWS), valid, 1);
#pragma unroll
      for (int t = 0; t < TILE_ROWS; ++t) {
        const float2 du = tile.du[wave][t][ch];
        float b[S], c[S];
        read_states(b, &tile.rows[buffer][t][group * S]);
        if (LATER) read_states(c, &tile.rows[Tile<H>::C + buffer][t][group * S]);
        const float e = LATER ? tile.e[wave][t][ch] : 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s) {
          const bool there = EXACT || s < n;
          const float f = exp2_of((there ? du.x : 0.f) * a2[s]);
          h[s] = fmaf(f, h[s], (there ? du.y : 0.f) * b[s]);
          if (LATER) {
            product[s] *= f;
            g[s] = fmaf(product[s], (there ? e : 0.f) * c[s], g[s]);
          }
        }
        passed += du.x;
      }
    }
  };
  if (p.span > 0) walk(std::true_type{});
  else walk(std::false_type{});
  if (p.span == 0 && p.last) return;
  if (!p.last) store_states(h, a.adds + item * each + of_lane, n);
  if (p.span > 0) store_states(g, a.back + item * each + of_lane, n);
  if (live && group == 0) a.steps[(int64_t)item * a.dim + p.channel + wave * H::CW + ch] = passed;
}

__device__ __forceinline__ void swap_halves(float& x, float& y) {
  const auto v = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y), false, false);
  x = __builtin_bit_cast(float, (uint32_t)v[0]);
  y = __builtin_bit_cast(float, (uint32_t)v[1]);
}
__device__ __forceinline__ void swap_rows(float& x, float& y) {
  const auto v = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y), false, false);
  x = __builtin_bit_cast(float, (uint32_t)v[0]);
  y = __builtin_bit_cast(float, (uint32_t)v[1]);
}
// v of another lane: of those quad by quad, mirrored among 8 or 16, four above or below
enum { SWAP_ONE = 0xb1, SWAP_TWO = 0x4e, MIRROR_16 = 0x140, MIRROR_8 = 0x141, FROM_ABOVE_4 = 0x104, FROM_BELOW_4 = 0x114 };
template <int WHICH>
__device__ __forceinline__ float moved(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), WHICH, 0xf, 0xf, true));
}
// of the lane four above or below, whose number differs in the third bit
__device__ __forceinline__ float across_four(float v) {
  const int x = __builtin_bit_cast(int, v);
  const int lower = __builtin_amdgcn_update_dpp(0, x, FROM_ABOVE_4, 0xf, 0x5, false);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(lower, x, FROM_BELOW_4, 0xf, 0xa, false));
}

// Sums over the G lanes of a channel of four rows' numbers: lane l gets that of row l % 4.  Two numbers are joined in one register at a step.
template <int G>
__device__ __forceinline__ float sums_of_states(float (&v)[4], int lane) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (G > 8) v[i] += moved<MIRROR_16>(v[i]);
    if (G > 4) v[i] += moved<MIRROR_8>(v[i]);
  }
  const bool odd = lane & 1, upper = lane & 2;
  const float x = (odd ? v[1] : v[0]) + moved<SWAP_ONE>(odd ? v[0] : v[1]);
  const float y = (odd ? v[3] : v[2]) + moved<SWAP_ONE>(odd ? v[2] : v[3]);
  return (upper ? y : x) + moved<SWAP_TWO>(upper ? x : y);
}

// Numbers of two states (or of two pairs of them) joined in one register, for two rows: the sum with the lane eight on among 16, of the first in the
// lower eight lanes and of the second in the upper; then, of what these leave of four states, the same with the lane four on or back.  An addition that
// writes a part of the lanes does what otherwise takes two selections and an addition; the compiler does not make it.  (s_nop: what a vector
// instruction has just written can be read so, and swapped, two steps later.)
__device__ __forceinline__ void join_eight_on(float& x, float& y, float a0, float a1, float b0, float b1) {
  asm("s_nop 1\n\t"
      "v_add_f32_dpp %0, %2, %2 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %1, %4, %4 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %0, %3, %3 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %1, %5, %5 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "s_nop 1"
      : "=&v"(x), "=&v"(y)
      : "v"(a0), "v"(a1), "v"(b0), "v"(b1));
}
__device__ __forceinline__ void join_four_states(float& x, float& y, const float (&a)[4], const float (&b)[4]) {
  float p, q, r, s;
  asm("s_nop 1\n\t"
      "v_add_f32_dpp %2, %6, %6 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %3, %7, %7 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %2, %8, %8 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %3, %9, %9 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %4, %10, %10 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %5, %11, %11 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %4, %12, %12 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %5, %13, %13 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %0, %2, %2 row_shl:4 row_mask:0xf bank_mask:0x5\n\t"
      "v_add_f32_dpp %0, %3, %3 row_shr:4 row_mask:0xf bank_mask:0xa\n\t"
      "v_add_f32_dpp %1, %4, %4 row_shl:4 row_mask:0xf bank_mask:0x5\n\t"
      "v_add_f32_dpp %1, %5, %5 row_shr:4 row_mask:0xf bank_mask:0xa\n\t"
      "s_nop 1"
      : "=&v"(x), "=&v"(y), "=&v"(p), "=&v"(q), "=&v"(r), "=&v"(s)
      : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]));
}

// Without that room: channels that there are not have no part in sums over channels.
template <int S>
__device__ __forceinline__ void silence(float (&v)[4][S], bool live) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int s = 0; s < S; ++s) v[i][s] = live ? v[i][s] : 0.f;
}

// dA += x d, where the tile has row T.  Whether it has is the same for all lanes, and no lane's business: d = 0 would not silence an x that is not
// finite, a selection a number takes an instruction of the vector pipe each, and a branch keeps the rows on its sides apart.  (exec: all lanes, as everywhere
// in the walk.)
template <int T, int S>
__device__ __forceinline__ void add_where_row(float (&dA)[S], const float (&x)[S], const float (&d)[S], int rows) {
  if constexpr (S == 4)
    asm("s_cmp_gt_i32 %12, %13\n\t"
        "s_cselect_b64 exec, -1, 0\n\t"
        "v_fmac_f32_e32 %0, %4, %8\n\t"
        "v_fmac_f32_e32 %1, %5, %9\n\t"
        "v_fmac_f32_e32 %2, %6, %10\n\t"
        "v_fmac_f32_e32 %3, %7, %11\n\t"
        "s_mov_b64 exec, -1"
        : "+v"(dA[0]), "+v"(dA[1]), "+v"(dA[2]), "+v"(dA[3])
        : "v"(x[0]), "v"(x[1]), "v"(x[2]), "v"(x[3]), "v"(d[0]), "v"(d[1]), "v"(d[2]), "v"(d[3]), "s"(rows), "n"(T)
        : "scc");
  else
    asm("s_cmp_gt_i32 %6, %7\n\t"
        "s_cselect_b64 exec, -1, 0\n\t"
        "v_fmac_f32_e32 %0, %2, %4\n\t"
        "v_fmac_f32_e32 %1, %3, %5\n\t"
        "s_mov_b64 exec, -1"
        : "+v"(dA[0]), "+v"(dA[1])
        : "v"(x[0]), "v"(x[1]), "v"(d[0]), "v"(d[1]), "s"(rows), "n"(T)
        : "scc");
}

// Four rows' numbers, one register each, to one: lane l gets the sum, over the lanes that differ in the upper two bits, of row l / 16.
__device__ __forceinline__ float join_rows(float a, float b, float c, float d) {
  swap_halves(a, c);
  swap_halves(b, d);
  float x = a + c, y = b + d;
  swap_rows(x, y);
  return x + y;
}

// Sums over the wave's channels of four rows' numbers for the lane's S states, to out[4][NS] in LDS.
template <class H>
__device__ __forceinline__ void sums_of_channels(float (&v)[4][H::S], float* out, int lane) {
  constexpr int S = H::S;
  out += lane / 16 * H::NS + lane % H::G * S;
  if constexpr (H::G == 16) {
    float4 z;
    z.x = join_rows(v[0][0], v[1][0], v[2][0], v[3][0]);
    z.y = join_rows(v[0][1], v[1][1], v[2][1], v[3][1]);
    z.z = join_rows(v[0][2], v[1][2], v[2][2], v[3][2]);
    z.w = join_rows(v[0][3], v[1][3], v[2][3], v[3][3]);
    *reinterpret_cast<float4*>(out) = z;
  } else if constexpr (H::G == 8) {                // lower eight lanes: states 0 and 1
    float a[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) join_eight_on(a[i], b[i], v[i][0], v[i][2], v[i][1], v[i][3]);
    *reinterpret_cast<float2*>(out + (lane & 8 ? 2 : 0)) = float2{join_rows(a[0], a[1], a[2], a[3]), join_rows(b[0], b[1], b[2], b[3])};
  } else if constexpr (S == 4) {                   // lanes by four: states 0, 1, 2, 3
    float a[4];
    join_four_states(a[0], a[1], v[0], v[1]);
    join_four_states(a[2], a[3], v[2], v[3]);
    out[lane % 16 / 4] = join_rows(a[0], a[1], a[2], a[3]);
  } else {
    float a[4];
    join_eight_on(a[0], a[1], v[0][0], v[0][1], v[1][0], v[1][1]);
    join_eight_on(a[2], a[3], v[2][0], v[2][1], v[3][0], v[3][1]);
    float x = join_rows(a[0], a[1], a[2], a[3]);
    x += across_four(x);
    if (!(lane & 4)) out[lane & 8 ? 1 : 0] = x;
  }
}

// The second walk.  A tile's 16 states and factors, 32 S registers, are what lets it go back without computing them again or dividing by a factor that may be
// zero; with them two waves fit into a SIMD, and the vector pipe is busy 73 % of the time: 8 x 2048 rows, 2048 channels, 16 states, bfloat16, 494 us, where
// its instructions alone take 375.  (In float32, 9 to 16 states with a gate, 17 to 19 registers a lane are in memory: x, dt, z and dy of a tile wait for its end.  16
// states: 644 us, the pipe busy 58 %.)  The rest are waits for LDS that two waves cannot fill.  (Half tiles, with three waves a SIMD, took longer; waves that share
// out a channel's states, as forward, with more barriers a tile, 160 us more.)
template <class TR, class H, bool EXACT, bool GATE>
__global__ __launch_bounds__(H::THREADS, 2) void k_scan_backward(const ScanArgs a) {
  typedef typename TR::T T;
  constexpr int S = H::S, V = H::V;
  // A branch between the quarters of a tile, for its registers: the states of rows that there are not, which it clears, are used nowhere.  Without it the float32
  // kernel of 9 to 16 states with a gate has 25 registers in memory instead of 17 (8 x 2048 rows, 2048 channels, 16 states: 906 us instead of 845), and 64
  // states take 1414 us instead of 1367 (8 x 1024 rows, bfloat16); with it other kernels take longer (bfloat16, 16 states: 667 us instead of 651, 4096 sequences
  // of 4 rows 1960 instead of 1863; 10 states 755 instead of 750, though two registers are in memory there without it).
  constexpr bool APART = H::NS == 64 || (H::NS == 16 && GATE && sizeof(T) == 4);
  __shared__ Tile<H> tile;
  __shared__ float part[GATE ? 3 : 2][H::WAVES][TILE_ROWS][H::CW];       // sums over the states: du, dd, y, every wave's own
  __shared__ alignas(16) float sums[2][2][H::WAVES][TILE_ROWS][H::NS];               // over a wave's channels: dB, dC
  __shared__ float of_channel[2][H::CB];                                 // bias and D
  __shared__ alignas(16) float starts[H::ROOM ? H::THREADS : 1][S];      // the lanes' states at the span's begin, where there is room
  const int item = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks;
  if (item >= a.items) {
    const int who = blockIdx.x - a.items * a.blocks;
    clear_rows<TR>(a, who, a.dx, a.dx_row);
    clear_rows<TR>(a, who, a.ddt, a.ddt_row);
    clear_rows<TR>(a, who, a.dz, a.dz_row);
    return;
  }
  Place p;
  const bool found = find(a, item, block, p);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int ch = lane / H::G, group = lane % H::G, valid = p.valid - wave * H::CW;
  const int r = lane / 4, col = lane % 4 * V;
  const int n = ch < valid ? min(S, a.states - group * S) : 0;
  const int channel = p.channel + wave * H::CW;
  const int64_t each = (int64_t)a.dim * a.states, of_lane = (int64_t)(channel + ch) * a.states + group * S;
  float dA[S], dD[V], dbias[V];
#pragma unroll
  for (int s = 0; s < S; ++s) dA[s] = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) dD[j] = dbias[j] = 0.f;
  if (found) {
    float g[S], a2[S];
    if (threadIdx.x < H::CB) {
      const bool mine = (int)threadIdx.x < p.valid;
      of_channel[0][threadIdx.x] = mine && a.bias ? a.bias[p.channel + threadIdx.x] : 0.f;
      of_channel[1][threadIdx.x] = mine && a.D ? a.D[p.channel + threadIdx.x] : 0.f;
    }
    if (H::ROOM && p.valid < H::CB)
      for (int at = threadIdx.x; at < 3 * TILE_ROWS * H::NS; at += H::THREADS) (&tile.rows[Tile<H>::NONE][0][0])[at] = 0.f;
    __syncthreads();
    const float* bias = &of_channel[0][wave * H::CW + col];
    const float* D = &of_channel[1][wave * H::CW + col];
    load_states(a2, a.A + of_lane, n);
#pragma unroll
    for (int s = 0; s < S; ++s) a2[s] = rate_of(a2[s]);
    const float* end = p.last && p.span == 0 ? (a.ds_end ? a.ds_end + p.piece.seq * each : nullptr) : a.back + item * each;
    load_states(g, end + of_lane, end ? n : 0);
    const int tiles = (int)((p.to - p.from + TILE_ROWS - 1) / TILE_ROWS);
    const int64_t number = first_tile(p), stride = (int64_t)a.groups * a.states;
    // (of the group's blocks this one's parts of dB and dC)
    const int64_t part_at = (int64_t)(block % (a.blocks / a.groups)) * a.n_rows * stride + p.group * a.states;
    // dB and dC of a tile from the waves' sums
    auto gather = [&](int buffer, int64_t t0, int rows) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < H::PAIRS; ++k) {
        const int at = k * H::THREADS + threadIdx.x, row = at / H::NS, state = at % H::NS;
        if (row < rows && state < a.states) {
          const int64_t to = part_at + (t0 + row) * stride + state;
          float b = 0.f, c = 0.f;
#pragma unroll
          for (int w = 0; w < H::WAVES; ++w) {
            b += sums[buffer][0][w][row][state];
            c += sums[buffer][1][w][row][state];
          }
          a.dB[to] = b;
          a.dC[to] = c;
        }
      }
    };
    Incoming<TR, H, true> in;
    in.begin(a, p, wave, lane, p.from + (int64_t)(tiles - 1) * TILE_ROWS);
    if (tiles > 0) in.load(a, p, lane, (int)(p.to - p.from - (int64_t)(tiles - 1) * TILE_ROWS), valid, -1);
    // the states at the next tile's begin, and the span's steps before it, on their way while a tile is worked through
    float begin[S], passed = 0.f;
    const auto load_begin = [&](int k) __attribute__((always_inline)) {
      __builtin_memcpy(begin, kept<H>(a, number + k, block), sizeof begin);
      if (p.span > 0 && ch < valid) passed = a.tile_steps[(number + k) * a.dim + channel + ch];
    };
    if (tiles > 0) load_begin(tiles - 1);
    if (H::ROOM && p.span > 0) {
      float start[S];
      load_states(start, a.adds + item * each + of_lane, n);
      __builtin_memcpy(starts[threadIdx.x], start, sizeof start);
    }
    int buffer = 0;
    for (int k = tiles - 1; k >= 0; --k, buffer ^= 1) {
      const int64_t t0 = p.from + (int64_t)k * TILE_ROWS;
      const int rows = (int)min((int64_t)TILE_ROWS, p.to - t0);
      float h[TILE_ROWS + 1][S], f[TILE_ROWS][S];                        // h_{t-1} and on, a_t
#pragma unroll
      for (int s = 0; s < S; ++s) h[0][s] = ch < valid ? begin[s] : 0.f;
      if (p.span > 0) {                                                  // (its walk began at zero)
        float start[S];
        if constexpr (H::ROOM) read_states(start, starts[threadIdx.x]);
        else load_states(start, a.adds + item * each + of_lane, n);
#pragma unroll
        for (int s = 0; s < S; ++s) h[0][s] = start[s] == 0.f ? h[0][s] : fmaf(exp2_of(a2[s] * passed), start[s], h[0][s]);
      }
      fill_tile(tile, a, in, wave, lane, buffer, rows, valid, bias);
      const Values<TR, V> x_now = in.x, dt_now = in.dt, z_now = in.z, dy_now = in.dy;
      __syncthreads();
      if (k + 1 < tiles) gather(buffer ^ 1, t0 + TILE_ROWS, (int)min((int64_t)TILE_ROWS, p.to - t0 - TILE_ROWS));
      if (k > 0) {
        in.load(a, p, lane, TILE_ROWS, valid, -1);
        load_begin(k - 1);
      }
      const float* B = &tile.rows[H::ROOM && ch >= valid ? Tile<H>::NONE : buffer][0][group * S];
      const float* C = B + Tile<H>::C * TILE_ROWS * H::NS;
      repeat<TILE_ROWS / 4>([&](auto q) __attribute__((always_inline)) {
        float of_c[4][S], y[4];
        repeat<4>([&](auto i) __attribute__((always_inline)) {
          constexpr int t = 4 * q + i;
          const float2 du = tile.du[wave][t][ch];
          const float e = tile.e[wave][t][ch];
          float b[S], c[S];
          read_states(b, B + t * H::NS);
          if (GATE) read_states(c, C + t * H::NS);
          y[i] = 0.f;
#pragma unroll
          for (int s = 0; s < S; ++s) {
            const bool there = EXACT || s < n;
            f[t][s] = exp2_of((there ? du.x : 0.f) * a2[s]);
            h[t + 1][s] = fmaf(f[t][s], h[t][s], (there ? du.y : 0.f) * b[s]);
            of_c[i][s] = (there ? e : 0.f) * h[t + 1][s];
            if (GATE) y[i] = fmaf(c[s], h[t + 1][s], y[i]);
          }
        });
        if constexpr (GATE) part[2][wave][4 * q + lane % 4][ch] = sums_of_states<H::G>(y, lane);
        if (!H::ROOM && valid < H::CW) silence(of_c, ch < valid);
        sums_of_channels<H>(of_c, &sums[buffer][1][wave][4 * q][0], lane);
        if (APART && 4 * q + 4 > rows)
          repeat<4>([&](auto i) __attribute__((always_inline)) {
#pragma unroll
            for (int s = 0; s < S; ++s) h[4 * q + i + 1][s] = 4 * q + i + 1 >= rows ? 0.f : h[4 * q + i + 1][s];
          });
        __builtin_amdgcn_sched_barrier(0);         // (what comes later is not read earlier: its registers are needed)
      });
      repeat<TILE_ROWS / 4>([&](auto back) __attribute__((always_inline)) {
        constexpr int q = TILE_ROWS / 4 - 1 - back;
        float of_b[4][S], by_u[4], by_d[4];
        repeat<4>([&](auto j) __attribute__((always_inline)) {
          constexpr int i = 3 - j, t = 4 * q + i;
          const float2 du = tile.du[wave][t][ch];
          const float e = tile.e[wave][t][ch];
          float b[S], c[S];
          read_states(b, B + t * H::NS);
          read_states(c, C + t * H::NS);
          by_u[i] = by_d[i] = 0.f;
          float x[S], d[S];
#pragma unroll
          for (int s = 0; s < S; ++s) {
            const bool there = EXACT || s < n;
            g[s] = fmaf(there ? e : 0.f, c[s], g[s]);
            of_b[i][s] = g[s] * (there ? du.y : 0.f);
            by_u[i] = fmaf(b[s], g[s], by_u[i]);
            g[s] *= f[t][s];
            x[s] = g[s] * h[t][s];
            d[s] = there ? du.x : 0.f;
            by_d[i] = fmaf(x[s], a2[s], by_d[i]);
          }
          add_where_row<t>(dA, x, d, rows);
        });
        part[0][wave][4 * q + lane % 4][ch] = sums_of_states<H::G>(by_u, lane);
        part[1][wave][4 * q + lane % 4][ch] = sums_of_states<H::G>(by_d, lane);
        if (!H::ROOM && valid < H::CW) silence(of_b, ch < valid);
        sums_of_channels<H>(of_b, &sums[buffer][0][wave][4 * q][0], lane);
        __builtin_amdgcn_sched_barrier(0);
      });
      // (what the wave's lanes have stored for each other)
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      float dx[V], ddt[V], dz[V];
      const bool there = r < rows;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = tile.du[wave][r][col + j].x, e = tile.e[wave][r][col + j], x = x_now.get(j), raw = dt_now.get(j) + bias[j];
        const float du = part[0][wave][r][col + j], dd = part[1][wave][r][col + j];
        dx[j] = a.D ? fmaf(D[j], e, d * du) : d * du;
        ddt[j] = fmaf(x, du, LN_2 * dd);
        if (a.softplus) ddt[j] *= sigmoid_of<TR>(raw);
        if (there && col + j < valid) {
          dD[j] = fmaf(e, x, dD[j]);
          dbias[j] += ddt[j];
        }
        dz[j] = 0.f;
        if constexpr (GATE) {
          const float z = z_now.get(j), s = sigmoid_of<TR>(z), y = part[2][wave][r][col + j];
          dz[j] = dy_now.get(j) * (a.D ? fmaf(D[j], x, y) : y) * s * fmaf(z, 1.f - s, 1.f);
        }
      }
      if (there) {
        const int64_t row = t0 + r;
        Values<TR, V> o;
        o.put(dx);
        o.store(static_cast<T*>(a.dx) + row * a.dx_row + channel + col, valid - col);
        o.put(ddt);
        o.store(static_cast<T*>(a.ddt) + row * a.ddt_row + channel + col, valid - col);
        if constexpr (GATE) {
          o.put(dz);
          o.store(static_cast<T*>(a.dz) + row * a.dz_row + channel + col, valid - col);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    if (tiles > 0) gather(buffer ^ 1, p.from, (int)min((int64_t)TILE_ROWS, p.to - p.from));
    if (p.span == 0 && a.ds_in) store_states(g, a.ds_in + p.piece.seq * each + of_lane, n);
  }
  // (items that are no span have sums too: zero)
  store_states(dA, a.dA + item * each + of_lane, n);
  auto of_rows = [&](const float (&v)[V], float* to) __attribute__((always_inline)) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) part[0][wave][r][col + j] = v[j];
    __syncthreads();
    if (lane < H::CW && lane < valid) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < TILE_ROWS; ++k) s += part[0][wave][k][lane];
      to[channel + lane] = s;
    }
  };
  if (a.D) of_rows(dD, a.dD + (int64_t)item * a.dim);
  if (a.bias) of_rows(dbias, a.dbias + (int64_t)item * a.dim);
}

// The gradients that are sums, from their parts in their order.  The first workgroups have dB and dC, from the channel blocks' parts (zero where no
// sequence owns the row), then those of dA, dD and dbias, from the spans' parts, each wave of a workgroup a quarter of them.  (15 us for 16384 rows, 2048
// channels: 32 parts of dB and dC, 67 MB.)
struct Sums {
  int64_t rows;       // workgroups of dB, and of dC
  int64_t channels;   // of dA, and of dD, and of dbias: 64 sums each
};
template <class TR>
__global__ __launch_bounds__(256) void k_scan_sums(const ScanArgs a, const Sums w) {
  typedef typename TR::T T;
  __shared__ float part[4][64];
  if (blockIdx.x < 2 * w.rows) {
    const bool is_C = blockIdx.x >= w.rows;
    const int64_t stride = (int64_t)a.groups * a.states, total = a.n_rows * stride, at = (blockIdx.x - (is_C ? w.rows : 0)) * 256 + threadIdx.x;
    if (at >= total) return;
    const int64_t row = at / stride;
    const int group = (int)(at % stride) / a.states, n = (int)(at % stride) % a.states, parts = a.blocks / a.groups;
    const int64_t first = clamped(a.off[0], 0, a.n_rows), last = clamped(a.off[a.n_seqs], first, a.n_rows);
    const float* from = (is_C ? a.dC : a.dB) + at;
    float s = 0.f;
    if (row >= first && row < last)
#pragma unroll 8
      for (int k = 0; k < parts; ++k) s += from[k * total];
    if (is_C) static_cast<T*>(a.dC_out)[row * a.dC_row + group * a.dC_head + n] = TR::put(s);
    else static_cast<T*>(a.dB_out)[row * a.dB_row + group * a.dB_head + n] = TR::put(s);
    return;
  }
  const int64_t block = blockIdx.x - 2 * w.rows;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, which = (int)(block / w.channels);
  const float* from = which == 0 ? a.dA : which == 1 ? a.dD : a.dbias;
  float* to = which == 0 ? a.dA_out : which == 1 ? a.dD_out : a.dbias_out;
  const int64_t size = (int64_t)a.dim * (which == 0 ? a.states : 1), at = block % w.channels * 64 + lane;
  if (!to || at - lane >= size) return;
  const int each = (a.items + 3) / 4, end = min(a.items, (wave + 1) * each);
  float s = 0.f;
  if (at < size)
#pragma unroll 8
    for (int k = wave * each; k < end; ++k) s += from[k * size + at];
  part[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && at < size) to[at] = part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
}

// f(shape, whether the states fill it).  That they do is known at 16 and 32 states, the usual numbers, which saves a selection an operand: 8 x 2048 rows, 2048
// channels, bfloat16, 655 us instead of 762 without it; 8 x 1024, 32 states, 600 instead of 702.  (8 and 64 states fill theirs too, and go without.)
typedef Shape<4, 4, 2> To8;
typedef Shape<4, 4, 4> To16;
typedef Shape<8, 8, 4> To32;
typedef Shape<16, 8, 4> To64;
template <class F>
void with_shape(int states, F f) {
  if (states <= 8) f(To8{}, std::false_type{});
  else if (states == 16) f(To16{}, std::true_type{});
  else if (states < 16) f(To16{}, std::false_type{});
  else if (states == 32) f(To32{}, std::true_type{});
  else if (states < 32) f(To32{}, std::false_type{});
  else f(To64{}, std::false_type{});
}

template <class TR>
void launch(const ScanArgs& a, bool one_span, void (*join)(const ScanArgs&, bool, hipStream_t), hipStream_t s) {
  if (a.items > 0)
    with_shape(a.states, [&](auto shape, auto exact) {
      typedef decltype(shape) H;
      constexpr bool EXACT = decltype(exact)::value;
      const dim3 spans((unsigned)(a.items * a.blocks)), all((unsigned)(a.items * a.blocks + ZERO_GROUPS)), threads(H::THREADS);
      hipLaunchKernelGGL((k_scan_tiles<TR, H, EXACT>), spans, threads, 0, s, a);
      if (!one_span) join(a, true, s);
      if (a.z) hipLaunchKernelGGL((k_scan_backward<TR, H, EXACT, true>), all, threads, 0, s, a);
      else hipLaunchKernelGGL((k_scan_backward<TR, H, EXACT, false>), all, threads, 0, s, a);
    });
  const int64_t values = a.n_rows * a.groups * a.states, each = (int64_t)a.dim * a.states;
  const Sums w{(values + 255) / 256, (each + 63) / 64};
  hipLaunchKernelGGL(k_scan_sums<TR>, dim3((unsigned)(2 * w.rows + 3 * w.channels)), dim3(256), 0, s, a, w);
}

}  // namespace

int scan_backward_width(int states) {
  int w = 0;
  with_shape(states, [&](auto shape, auto) { w = decltype(shape)::CB; });
  return w;
}

int scan_backward_threads(int states) {
  int t = 0;
  with_shape(states, [&](auto shape, auto) { t = decltype(shape)::THREADS; });
  return t;
}

int scan_backward_states(int states) {
  int n = 0;
  with_shape(states, [&](auto shape, auto) { n = decltype(shape)::S; });
  return n;
}

int launch_scan_backward(int dtype, const ScanArgs& a, bool one_span, void (*join)(const ScanArgs&, bool, hipStream_t), hipStream_t s) {
  if (dtype == NUGPR_BFLOAT16) launch<Bf16>(a, one_span, join, s);
  else launch<F32>(a, one_span, join, s);
  NUGPR_HIP(hipGetLastError());
  return NUGPR_OK;
}

}  // namespace nugpr
