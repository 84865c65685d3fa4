// The global norm of many gradients, and the gradients clipped by it.
//
// Two passes: squares summed in float64 (of float32 and bfloat16 values they neither
// overflow nor underflow), then g * factor, factor = max_norm / max(norm, max_norm).
// The gradients are cut into chunks of 16384 elements; workgroups take chunks in turn,
// and find a chunk's tensor by bisection in a table that comes with the launch's
// arguments (so nothing is copied to the device, and a captured launch holds it).  More
// tensors than a table takes are several launches, whose workgroups add to the same
// partial sums.  The last workgroup of the last launch adds those in order.
//
// The second pass goes backwards, from what the first left in the Infinity Cache.
#include "clip.hpp"
#include "device_common.hpp"
#include "wave_ops.hpp"

namespace vtrace {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int64_t kChunk = 16384;
constexpr int kTable = 96;  // tensors of a launch: 24 bytes each, and the head, within 4 KB of arguments

constexpr size_t kFactorOffset = 8;  // in the workspace's header, behind the counter and the error flag

struct ClipTable {
  const void* in[kTable];
  void* out[kTable];
  int64_t size_type[kTable];       // 2 size + (bfloat16)
  uint32_t first_chunk[kTable + 1];  // of each tensor, in this launch
  int count;
  int first, last;  // launches of the call
  float max_norm;
  float* norm;
  unsigned int* ticket;
  float* factor;
  double* partials;
};
static_assert(sizeof(ClipTable) <= 3072, "kernel arguments");

struct Piece {
  const char* in;
  char* out;
  int64_t n;
  bool bf16;
};

__device__ __forceinline__ Piece piece_of(const ClipTable& t, uint32_t chunk) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (t.first_chunk[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  Piece p;
  const int64_t off = static_cast<int64_t>(chunk - t.first_chunk[lo]) * kChunk;
  const int64_t left = (t.size_type[lo] >> 1) - off;
  p.bf16 = t.size_type[lo] & 1;
  p.n = left < kChunk ? left : kChunk;
  p.in = static_cast<const char*>(t.in[lo]) + off * (p.bf16 ? 2 : 4);
  p.out = static_cast<char*>(t.out[lo]) + off * (p.bf16 ? 2 : 4);
  return p;
}

__device__ __forceinline__ void add_square(double& sum, float x) {
  const double d = x;
  sum = fma(d, d, sum);
}
__device__ __forceinline__ void add_squares(double& sum, unsigned word, bool bf16) {
  if (bf16) {
    add_square(sum, __uint_as_float(word << 16));
    add_square(sum, __uint_as_float(word & 0xffff0000u));
  } else {
    add_square(sum, __uint_as_float(word));
  }
}

// Elements before the first 16-byte boundary of p.
template <typename T>
__device__ __forceinline__ int64_t before_boundary(const T* p, int64_t n) {
  const int64_t k = static_cast<int64_t>((16 - reinterpret_cast<uintptr_t>(p) % 16) % 16 / sizeof(T));
  return k < n ? k : n;
}

template <typename T>
__device__ __forceinline__ void sum_piece(const Piece& p, double (&sum)[4]) {
  constexpr int kPer = 16 / sizeof(T);
  const T* const in = reinterpret_cast<const T*>(p.in);
  const int64_t head = before_boundary(in, p.n);
  const int64_t vectors = (p.n - head) / kPer, tail = head + vectors * kPer;
  const v4u* const vec = reinterpret_cast<const v4u*>(in + head);
  for (int64_t i = threadIdx.x; i < vectors; i += 4 * kThreads) {
    v4u x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const v4u zero = {0u, 0u, 0u, 0u};
      x[u] = i + u * kThreads < vectors ? vec[i + u * kThreads] : zero;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int w = 0; w < 4; ++w) add_squares(sum[w], x[u][w], sizeof(T) == 2);
  }
  if (threadIdx.x < head) add_square(sum[0], logit_to_float(in[threadIdx.x]));
  if (tail + threadIdx.x < p.n) add_square(sum[1], logit_to_float(in[tail + threadIdx.x]));
}

__device__ __forceinline__ float scaled(float x, float factor) { return x * factor; }
__device__ __forceinline__ uint16_t scaled(uint16_t x, float factor) { return to_bf16(logit_to_float(x) * factor); }

template <typename T>
__device__ __forceinline__ unsigned scaled_word(unsigned w, float factor) {
  if constexpr (sizeof(T) == 4) return __float_as_uint(__uint_as_float(w) * factor);
  return pack_bf16x2(__uint_as_float(w << 16) * factor, __uint_as_float(w & 0xffff0000u) * factor);
}

template <typename T>
__device__ __forceinline__ void scale_piece(const Piece& p, float factor) {
  constexpr int kPer = 16 / sizeof(T);
  const T* const in = reinterpret_cast<const T*>(p.in);
  T* const out = reinterpret_cast<T*>(p.out);
  if (reinterpret_cast<uintptr_t>(in) % 16 != reinterpret_cast<uintptr_t>(out) % 16) {
    for (int64_t i = threadIdx.x; i < p.n; i += kThreads) out[i] = scaled(in[i], factor);
    return;
  }
  const int64_t head = before_boundary(in, p.n);
  const int64_t vectors = (p.n - head) / kPer, tail = head + vectors * kPer;
  const v4u* const from = reinterpret_cast<const v4u*>(in + head);
  v4u* const to = reinterpret_cast<v4u*>(out + head);
  for (int64_t i = threadIdx.x; i < vectors; i += 4 * kThreads) {
    v4u x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u * kThreads < vectors) x[u] = from[i + u * kThreads];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i + u * kThreads >= vectors) continue;
#pragma unroll
      for (int w = 0; w < 4; ++w) x[u][w] = scaled_word<T>(x[u][w], factor);
      to[i + u * kThreads] = x[u];
    }
  }
  if (threadIdx.x < head) out[threadIdx.x] = scaled(in[threadIdx.x], factor);
  if (tail + threadIdx.x < p.n) out[tail + threadIdx.x] = scaled(in[tail + threadIdx.x], factor);
}

__device__ __forceinline__ double block_sum(double x, double* scratch) {
  x = wave_sum(x);
  if (threadIdx.x % kWave == 0) scratch[threadIdx.x / kWave] = x;
  __syncthreads();
  x = scratch[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) x += scratch[w];
  __syncthreads();
  return x;
}

__global__ __launch_bounds__(kThreads) void clip_norm_kernel(ClipTable t) {
  __shared__ double s_red[kWaves];
  __shared__ int s_last;
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  const uint32_t chunks = t.first_chunk[t.count];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Piece p = piece_of(t, c);
    if (p.bf16) sum_piece<uint16_t>(p, sum);
    else sum_piece<float>(p, sum);
  }
  double total = block_sum((sum[0] + sum[1]) + (sum[2] + sum[3]), s_red);
  if (threadIdx.x == 0) {
    if (!t.first) total += __hip_atomic_load(t.partials + blockIdx.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(t.partials + blockIdx.x, total, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (!t.last) return;
  // As finish_ticket: the partial's store has completed before the ticket is drawn.
  if (threadIdx.x == 0) {
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    const unsigned prev = __hip_atomic_fetch_add(t.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = prev == gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  double all = 0.0;
  for (unsigned i = threadIdx.x; i < gridDim.x; i += kThreads)
    all += __hip_atomic_load(t.partials + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  all = block_sum(all, s_red);
  if (threadIdx.x == 0) {
    const double norm = sqrt(all), bound = t.max_norm;
    *t.norm = static_cast<float>(norm);
    // norm <= max_norm gives exactly 1; a NaN norm gives NaN.
    *t.factor = norm <= bound ? 1.0f : static_cast<float>(bound / norm);
    __hip_atomic_store(t.ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

__global__ __launch_bounds__(kThreads) void clip_scale_kernel(ClipTable t) {
  const float factor = *t.factor;
  const uint32_t chunks = t.first_chunk[t.count];
  for (uint32_t k = blockIdx.x; k < chunks; k += gridDim.x) {
    const Piece p = piece_of(t, chunks - 1 - k);
    if (factor == 1.0f && p.in == p.out) continue;  // clipping in place changes nothing
    if (p.bf16) scale_piece<uint16_t>(p, factor);
    else scale_piece<float>(p, factor);
  }
}

int64_t chunks_of(int64_t size) { return (size + kChunk - 1) / kChunk; }

// Tensors [from, from + n) of the call, for one launch: as many as a table takes, and
// whose chunks a 32-bit number counts.
int64_t fill(const ClipItem* items, int64_t count, int64_t from, ClipTable* t) {
  uint64_t chunks = 0;
  int n = 0;
  while (from + n < count && n < kTable) {
    const ClipItem& item = items[from + n];
    if (n > 0 && chunks + chunks_of(item.size) > 0x7fffffff) break;
    t->in[n] = item.in;
    t->out[n] = item.out;
    t->size_type[n] = 2 * item.size + (item.bf16 ? 1 : 0);
    t->first_chunk[n] = static_cast<uint32_t>(chunks);
    chunks += chunks_of(item.size);
    ++n;
  }
  t->first_chunk[n] = static_cast<uint32_t>(chunks);
  t->count = n;
  return n;
}

}  // namespace

size_t clip_workspace_bytes() { return kWsHeaderBytes + kClipMostBlocks * sizeof(double); }

hipError_t launch_clip(const ClipItem* items, int64_t count, bool scale, float max_norm, float* norm, void* ws,
                       hipStream_t st) {
  char* const base = static_cast<char*>(ws);
  ClipTable t = {};
  t.max_norm = max_norm;
  t.norm = norm;
  t.ticket = reinterpret_cast<unsigned int*>(base + kWsTicketOffset);
  t.factor = reinterpret_cast<float*>(base + kFactorOffset);
  t.partials = reinterpret_cast<double*>(base + kWsHeaderBytes);
  int64_t chunks = 0;
  for (int64_t i = 0; i < count && chunks < kClipMostBlocks; ++i) chunks += chunks_of(items[i].size);
  const unsigned blocks = static_cast<unsigned>(chunks < 1 ? 1 : chunks < kClipMostBlocks ? chunks : kClipMostBlocks);
  int64_t from = 0;
  do {
    const int64_t n = fill(items, count, from, &t);
    t.first = from == 0;
    t.last = from + n == count;
    hipLaunchKernelGGL(clip_norm_kernel, dim3(blocks), dim3(kThreads), 0, st, t);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    from += n;
  } while (from < count);
  if (!scale || count == 0) return hipSuccess;
  from = 0;
  do {
    const int64_t n = fill(items, count, from, &t);
    hipLaunchKernelGGL(clip_scale_kernel, dim3(blocks), dim3(kThreads), 0, st, t);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    from += n;
  } while (from < count);
  return hipSuccess;
}

}  // namespace vtrace
