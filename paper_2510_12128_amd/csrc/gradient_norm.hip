// The 2-norm of the gradients of a model, many tensors of any sizes, and their clipping to a bound:
//   norm = sqrt(sum of g^2 over all values),   g <- g min(1, bound / norm).
// Squares are summed in 64 bits: those of float32 values neither overflow nor vanish there.
//
// The tensors' addresses travel as kernel arguments, TABLE of them a launch, so that a call copies nothing and can be captured.
// Tensors are cut into chunks; a workgroup takes every so many chunks, adds up its squares and stores the sum at its place;
// whoever needs the norm adds all these sums in one fixed order.
#include <algorithm>
#include <new>
#include <vector>

#include "call_checks.h"
#include "row_values.h"

namespace nugpr {

namespace {

constexpr int THREADS = 256;
constexpr int TABLE = 232, TABLE_OUT = 155;      // tensors of a launch, without and with a place to go to: kernel arguments below 4096 bytes
constexpr int CHUNK = 16384;          // values
constexpr int GROUPS = 2048;          // workgroups of a call, about: partial sums that every clipping workgroup adds up

struct Tensor {
  void* data;
  uint32_t first;       // its first chunk
  uint32_t tail;        // values of its last chunk; the upper bits: its type, and that of where it goes
};
constexpr uint32_t BF16_DATA = 1u << 31, BF16_OUT = 1u << 30;

template <int N, bool OUT>
struct Table {
  Tensor t[N];
  void* out[OUT ? N : 1];
  double* sums;
  float* norm;
  double bound;
  int n;                // tensors
  uint32_t chunks;
  int n_sums;           // partial sums of the whole call
  int sums_from;        // of them, this launch's
};
typedef Table<TABLE, false> InPlace;
typedef Table<TABLE_OUT, true> ToOut;
static_assert(sizeof(InPlace) < 4000 && sizeof(ToOut) < 4000, "kernel arguments");

// A chunk: its tensor is the last that begins at or before it.  (Empty tensors begin where the next one does.)
struct Chunk {
  int tensor, count;
  int64_t from;
};
template <int N, bool OUT>
__device__ inline Chunk chunk_at(const Table<N, OUT>& a, uint32_t chunk) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int k = 0; k < (N + 63) / 64; ++k) {
    const int at = k * 64 + lane;
    n += __popcll(__ballot(at < a.n && a.t[min(at, N - 1)].first <= chunk));
  }
  n = __builtin_amdgcn_readfirstlane(n - 1);
  const uint32_t first = a.t[n].first, end = n + 1 < a.n ? a.t[n + 1].first : a.chunks;
  return Chunk{n, chunk + 1 == end ? (int)(a.t[n].tail & 0xffffu) : CHUNK, (int64_t)(chunk - first) * CHUNK};
}

__device__ inline double sum_of_workgroup(double x) {
  __shared__ double part[THREADS / 64];
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  if (!(threadIdx.x & 63)) part[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < THREADS / 64; ++k) s += part[k];
  return s;
}

template <class TR>
__device__ double squares(const typename TR::T* p, int count) {
  constexpr int V = TR::E;
  double s0 = 0.0, s1 = 0.0;
  for (int i = threadIdx.x * V; i < count; i += THREADS * V) {
    Values<TR, V> v;
    v.load(p + i, count - i);
#pragma unroll
    for (int j = 0; j < V; j += 2) {
      const double a = v.get(j), b = v.get(j + 1);
      s0 = fma(a, a, s0);
      s1 = fma(b, b, s1);
    }
  }
  return s0 + s1;
}

// Memory bounds it: 252 million bfloat16 values in 82 us, 6.2 TB/s (reads alone run faster than a copy).  The squares go to two sums of 64 bits a thread,
// which the loads hide.
__global__ __launch_bounds__(THREADS) void k_square_sums(const InPlace a) {
  double s = 0.0;
  for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const Chunk k = chunk_at(a, c);
    const Tensor& t = a.t[k.tensor];
    if (t.tail & BF16_DATA) s += squares<Bf16>(static_cast<const uint16_t*>(t.data) + k.from, k.count);
    else s += squares<F32>(static_cast<const float*>(t.data) + k.from, k.count);
  }
  s = sum_of_workgroup(s);
  if (threadIdx.x == 0) a.sums[a.sums_from + blockIdx.x] = s;
}

__device__ inline double norm_of(const double* sums, int n) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += THREADS) s += sums[i];
  return sqrt(sum_of_workgroup(s));
}

__global__ __launch_bounds__(THREADS) void k_norm(const double* sums, int n, float* norm) {
  const double x = norm_of(sums, n);
  if (threadIdx.x == 0) *norm = (float)x;
}

// (The product in 64 bits: a factor below float32's range times a large value is not lost.  To bfloat16 by way of float32, as its instruction rounds: off by
// 2^-24 more than half a step.)
template <class FROM, class TO>
__device__ void scaled(const typename FROM::T* p, typename TO::T* q, int count, double factor) {
  constexpr int V = 4;
  for (int i = threadIdx.x * V; i < count; i += THREADS * V) {
    Values<FROM, V> v;
    v.load(p + i, count - i);
    float x[V];
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = (float)(v.get(j) * factor);
    Values<TO, V> o;
    o.put(x);
    o.store(q + i, count - i);
  }
}

// Every workgroup adds up the partial sums for itself, 16 KB from L2, which saves a launch between two others; in place within the bound that is all it
// does (5 us).  Beyond it memory bounds this too: 252 million bfloat16 values in place in 162 us, 6.2 TB/s, and 303 with the norm, whose reads wait for what the
// call before has written (two reads and a write are 296 at the rate of a copy); float32, half as many values, 330.
template <int N, bool OUT>
__global__ __launch_bounds__(THREADS) void k_clip(const Table<N, OUT> a) {
  const double norm = norm_of(a.sums, a.n_sums);
  if (a.sums_from == 0 && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  const double factor = norm <= a.bound ? 1.0 : a.bound / norm;
  if (!OUT && factor == 1.0) return;
  for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const Chunk k = chunk_at(a, c);
    const Tensor& t = a.t[k.tensor];
    void* out = OUT ? a.out[k.tensor] : t.data;
    if (OUT && factor == 1.0 && out == t.data) continue;           // (of its own type, then: others may not overlap)
    if (t.tail & BF16_DATA) {
      const uint16_t* p = static_cast<const uint16_t*>(t.data) + k.from;
      if (!OUT || t.tail & BF16_OUT) scaled<Bf16, Bf16>(p, static_cast<uint16_t*>(out) + k.from, k.count, factor);
      else scaled<Bf16, F32>(p, static_cast<float*>(out) + k.from, k.count, factor);
    } else {
      const float* p = static_cast<const float*>(t.data) + k.from;
      if (OUT && t.tail & BF16_OUT) scaled<F32, Bf16>(p, static_cast<uint16_t*>(out) + k.from, k.count, factor);
      else scaled<F32, F32>(p, static_cast<float*>(out) + k.from, k.count, factor);
    }
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------
size_t size_of(int dtype) { return dtype == NUGPR_BFLOAT16 ? 2 : 4; }

int check_counts(const nugpr_gradient* g, int32_t n) {
  if (n < 0 || (n > 0 && !g)) return invalid("gradients is null or their number negative");
  int64_t total = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (g[i].dtype != NUGPR_FLOAT32 && g[i].dtype != NUGPR_BFLOAT16) return invalid("dtype must be NUGPR_FLOAT32 or NUGPR_BFLOAT16");
    if (g[i].count < 0 || g[i].count > (int64_t)1 << 40 || (total += g[i].count) > (int64_t)1 << 40) return invalid("counts must be 0..2^40 in all");
  }
  return NUGPR_OK;
}

int launches(int32_t n) { return (int)(((int64_t)n + TABLE - 1) / TABLE); }

// Most workgroups of one launch, by how many launches share the partial sums.
int64_t most_groups(int32_t n) { return std::max<int64_t>(64, GROUPS / std::max(1, launches(n))); }

int64_t chunks_of(int64_t count) { return (count + CHUNK - 1) / CHUNK; }

// Chunks of launch k.
int64_t chunks_in(const nugpr_gradient* g, int32_t n, int k) {
  int64_t c = 0;
  for (int32_t i = k * TABLE; i < std::min<int64_t>(n, (int64_t)(k + 1) * TABLE); ++i) c += chunks_of(g[i].count);
  return c;
}

int64_t sums_in(const nugpr_gradient* g, int32_t n) {
  int64_t s = 0;
  for (int k = 0; k < launches(n); ++k) s += std::min(chunks_in(g, n, k), most_groups(n));
  return s;
}

size_t workspace_of(const nugpr_gradient* g, int32_t n) { return 256 + ((size_t)sums_in(g, n) * sizeof(double) + 255) / 256 * 256; }

int check_call(const nugpr_gradient* g, int32_t n, const float* norm, const void* ws, size_t bytes) {
  if (const int c = check_counts(g, n)) return c;
  if (!norm || reinterpret_cast<uintptr_t>(norm) % 4) return invalid("norm is null or misaligned");
  for (int32_t i = 0; i < n; ++i)
    if (g[i].count > 0 && (!g[i].data || reinterpret_cast<uintptr_t>(g[i].data) % size_of(g[i].dtype))) return invalid("a gradient's data is null or misaligned");
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u)) { set_error("workspace is null or not 256-byte aligned"); return NUGPR_ERR_WORKSPACE; }
  if (bytes < workspace_of(g, n)) { set_error("workspace smaller than nugpr_gradient_norm_workspace_bytes()"); return NUGPR_ERR_WORKSPACE; }
  return NUGPR_OK;
}

// Refuses tensors that are written and share memory with another one.
int check_written(const nugpr_gradient* g, int32_t n) try {
  struct Range { uintptr_t lo, hi; bool written; };
  std::vector<Range> r;
  r.reserve(2 * (size_t)n);
  for (int32_t i = 0; i < n; ++i) {
    if (g[i].count == 0) continue;
    const uintptr_t at = reinterpret_cast<uintptr_t>(g[i].data), to = reinterpret_cast<uintptr_t>(g[i].out);
    const bool in_place = !to || (to == at && g[i].out_dtype == g[i].dtype);
    r.push_back({at, at + (uintptr_t)g[i].count * size_of(g[i].dtype), in_place});
    if (in_place) continue;
    if (g[i].out_dtype != NUGPR_FLOAT32 && g[i].out_dtype != NUGPR_BFLOAT16) return invalid("out_dtype must be NUGPR_FLOAT32 or NUGPR_BFLOAT16");
    if (to % size_of(g[i].out_dtype)) return invalid("a gradient's out is misaligned");
    r.push_back({to, to + (uintptr_t)g[i].count * size_of(g[i].out_dtype), true});
  }
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
  uintptr_t read_to = 0, written_to = 0;       // the ends of what has begun
  for (const Range& x : r) {
    if (x.lo < written_to || (x.written && x.lo < read_to)) return invalid("tensors that are written overlap others");
    (x.written ? written_to : read_to) = std::max(x.written ? written_to : read_to, x.hi);
  }
  return NUGPR_OK;
} catch (const std::bad_alloc&) {
  return invalid("no host memory for the tensors' ranges");
}

// Every launch of a kernel over the tables; `groups` at most.  The sums' places are those of the first kernel's workgroups.
template <class T, class F>
void for_tables(const nugpr_gradient* g, int32_t n, double* sums, float* norm, double bound, int64_t most, F launch) {
  constexpr int N = sizeof(T::t) / sizeof(Tensor);
  constexpr bool OUT = sizeof(T::out) > sizeof(void*);
  T a;
  a.sums = sums; a.norm = norm; a.bound = bound;
  a.n_sums = (int)sums_in(g, n);
  a.sums_from = 0;
  for (int64_t from = 0; from < n; from += N) {
    a.n = (int)std::min<int64_t>(N, n - from);
    uint32_t chunk = 0;
    for (int i = 0; i < a.n; ++i) {
      const nugpr_gradient& x = g[from + i];
      const int64_t chunks = chunks_of(x.count);
      a.t[i] = Tensor{x.data, chunk, (uint32_t)(x.count - std::max<int64_t>(chunks - 1, 0) * CHUNK)};
      if (x.dtype == NUGPR_BFLOAT16) a.t[i].tail |= BF16_DATA;
      if (OUT) a.out[i] = x.out ? x.out : x.data;
      if (OUT && (x.out ? x.out_dtype : x.dtype) == NUGPR_BFLOAT16) a.t[i].tail |= BF16_OUT;
      chunk += (uint32_t)chunks;
    }
    a.chunks = chunk;
    const int64_t groups = std::min<int64_t>(chunk, most);
    if (groups > 0) launch(a, dim3((unsigned)groups));
    a.sums_from += (int)groups;
  }
}

}  // namespace

}  // namespace nugpr

using namespace nugpr;

extern "C" {

size_t nugpr_gradient_norm_workspace_bytes(const nugpr_gradient* g, int32_t n) {
  if (check_counts(g, n) != NUGPR_OK) return 0;
  return workspace_of(g, n);
}

int nugpr_gradient_norm(const nugpr_gradient* g, int32_t n, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  if (const int c = check_call(g, n, norm, workspace, workspace_bytes)) return c;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  double* sums = static_cast<double*>(workspace);
  for_tables<InPlace>(g, n, sums, norm, 0.0, most_groups(n), [&](const InPlace& a, dim3 grid) { hipLaunchKernelGGL(k_square_sums, grid, dim3(THREADS), 0, s, a); });
  hipLaunchKernelGGL(k_norm, dim3(1), dim3(THREADS), 0, s, sums, (int)sums_in(g, n), norm);
  NUGPR_HIP(hipGetLastError());
  return NUGPR_OK;
}

int nugpr_clip_gradients(const nugpr_gradient* g, int32_t n, double max_norm, float* norm, void* workspace, size_t workspace_bytes,
                         void* stream) {
  if (const int c = check_call(g, n, norm, workspace, workspace_bytes)) return c;
  if (!(max_norm >= 0.0)) return invalid("max_norm must be >= 0");
  if (const int c = check_written(g, n)) return c;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  double* sums = static_cast<double*>(workspace);
  if (sums_in(g, n) == 0) {
    hipLaunchKernelGGL(k_norm, dim3(1), dim3(THREADS), 0, s, sums, 0, norm);
  } else {
    for_tables<InPlace>(g, n, sums, norm, max_norm, most_groups(n),
                        [&](const InPlace& a, dim3 grid) { hipLaunchKernelGGL(k_square_sums, grid, dim3(THREADS), 0, s, a); });
    bool elsewhere = false;
    for (int32_t i = 0; i < n; ++i) elsewhere |= g[i].out && (g[i].out != g[i].data || g[i].out_dtype != g[i].dtype);
    if (elsewhere)
      for_tables<ToOut>(g, n, sums, norm, max_norm, GROUPS,
                        [&](const ToOut& a, dim3 grid) { hipLaunchKernelGGL((k_clip<TABLE_OUT, true>), grid, dim3(THREADS), 0, s, a); });
    else
      for_tables<InPlace>(g, n, sums, norm, max_norm, GROUPS,
                          [&](const InPlace& a, dim3 grid) { hipLaunchKernelGGL((k_clip<TABLE, false>), grid, dim3(THREADS), 0, s, a); });
  }
  NUGPR_HIP(hipGetLastError());
  return NUGPR_OK;
}

}  // extern "C"
