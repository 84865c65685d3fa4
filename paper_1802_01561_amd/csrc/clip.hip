// The global norm of many gradients, and the gradients clipped by it.
//
// Two passes: squares summed in float64 (of float32 and bfloat16 values they neither
// overflow nor underflow), then g * factor, factor = max_norm / max(norm, max_norm).
// The gradients are cut into chunks; a workgroup finds a chunk's tensor by bisection in a
// table that comes with the launch's arguments (so nothing is copied to the device, and a
// captured launch holds it).  More tensors than a table takes are several launches, whose
// workgroups add to the same partial sums.  The last workgroup of the last launch adds
// those in order.
//
// Bound by memory: 1.2e9 elements, mostly bfloat16, in 290 tensors (2.4 GB read twice and
// written once) 430 + 895 us, 5.6 and 5.4 TB/s (torch's copy of 8 GB: 4.8).  The norm's
// workgroups take several chunks (one partial sum each); the second pass has a workgroup a
// chunk (2048 workgroups in turn: 1060 us).  Walking it backwards, from what the first pass
// left in the Infinity Cache, gained nothing.  Outputs whose place in 16 bytes is not their
// gradient's are written element by element: 60 M float32 290 us, at the same place 113.
#include "clip.hpp"
#include "device_common.hpp"
#include "tickets.hpp"
#include "wave_ops.hpp"

namespace vtrace {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
// Elements of a chunk; short calls take smaller ones to have more workgroups.
constexpr int kChunkBits = 14, kSmallChunkBits = 12;
constexpr int64_t kSmallCall = int64_t(1) << 24;

// Tensors of a launch: as many as 4 KB of arguments hold.
template <bool kOut>
struct ClipTable {
  static constexpr int kMost = kOut ? 140 : 196;
  const void* in[kMost];
  void* out[kOut ? kMost : 1];
  int64_t size_type[kMost];         // 2 size + (bfloat16)
  uint32_t first_chunk[kMost + 1];  // of each tensor, in this launch
  int count;
  int chunk_bits;
  int first, last;  // launches of the call
  float max_norm;
  float* norm;
  unsigned int* ticket;
  unsigned int* counters;
  float* factor;
  double* partials;
};
static_assert(sizeof(ClipTable<true>) <= 4096 && sizeof(ClipTable<false>) <= 4096, "kernel arguments");

struct Piece {
  const char* in;
  char* out;
  int64_t n;
  bool bf16;
};

template <bool kOut>
__device__ __forceinline__ Piece piece_of(const ClipTable<kOut>& t, uint32_t chunk) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (t.first_chunk[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  Piece p;
  const int64_t off = static_cast<int64_t>(chunk - t.first_chunk[lo]) << t.chunk_bits;
  const int64_t left = (t.size_type[lo] >> 1) - off;
  p.bf16 = t.size_type[lo] & 1;
  const int64_t whole = int64_t(1) << t.chunk_bits;
  p.n = left < whole ? left : whole;
  p.in = static_cast<const char*>(t.in[lo]) + off * (p.bf16 ? 2 : 4);
  p.out = kOut ? static_cast<char*>(t.out[lo]) + off * (p.bf16 ? 2 : 4) : nullptr;
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
  constexpr int kPer = 16 / sizeof(T), kUnroll = 8;
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
  for (int64_t i = threadIdx.x; i < vectors; i += kUnroll * kThreads) {
    v4u x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (i + u * kThreads < vectors) x[u] = from[i + u * kThreads];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (i + u * kThreads >= vectors) continue;
#pragma unroll
      for (int w = 0; w < 4; ++w) x[u][w] = scaled_word<T>(x[u][w], factor);
      // Past the caches: nothing reads the outputs soon (60 M float32: 147 -> 117 us).
      __builtin_nontemporal_store(x[u], &to[i + u * kThreads]);
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

__global__ __launch_bounds__(kThreads) void clip_norm_kernel(ClipTable<false> t) {
  __shared__ double s_red[kWaves];
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
  if (!t.last || !last_workgroup(t.ticket, t.counters)) return;
  double all = 0.0;
  for (unsigned i = threadIdx.x; i < gridDim.x; i += kThreads)
    all += __hip_atomic_load(t.partials + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  all = block_sum(all, s_red);
  if (threadIdx.x == 0) {
    const double norm = sqrt(all), bound = t.max_norm;
    *t.norm = static_cast<float>(norm);
    // norm <= max_norm gives exactly 1; a NaN norm gives NaN.
    *t.factor = norm <= bound ? 1.0f : static_cast<float>(bound / norm);
  }
}

__global__ __launch_bounds__(kThreads) void clip_scale_kernel(ClipTable<true> t) {
  const float factor = *t.factor;
  const Piece p = piece_of(t, blockIdx.x);
  if (factor == 1.0f && p.in == p.out) return;  // clipping in place changes nothing
  if (p.bf16) scale_piece<uint16_t>(p, factor);
  else scale_piece<float>(p, factor);
}

int64_t chunks_of(int64_t size, int bits) { return (size + (int64_t(1) << bits) - 1) >> bits; }

// Tensors [from, from + n) of the call, for one launch: as many as a table takes, and
// whose chunks a launch has workgroups for (2^32 threads).
constexpr uint64_t kMostChunks = (uint64_t(1) << 32) / kThreads - 1;
template <bool kOut>
int64_t fill(const ClipItem* items, int64_t count, int64_t from, ClipTable<kOut>* t) {
  uint64_t chunks = 0;
  int n = 0;
  while (from + n < count && n < ClipTable<kOut>::kMost) {
    const ClipItem& item = items[from + n];
    if (n > 0 && chunks + chunks_of(item.size, t->chunk_bits) > kMostChunks) break;
    t->in[n] = item.in;
    if (kOut) t->out[n] = item.out;
    t->size_type[n] = 2 * item.size + (item.bf16 ? 1 : 0);
    t->first_chunk[n] = static_cast<uint32_t>(chunks);
    chunks += chunks_of(item.size, t->chunk_bits);
    ++n;
  }
  t->first_chunk[n] = static_cast<uint32_t>(chunks);
  t->count = n;
  return n;
}

}  // namespace

size_t clip_workspace_bytes() { return kWsDataOffset + kClipMostBlocks * sizeof(double); }

namespace {

template <bool kOut>
hipError_t launch_pass(const ClipItem* items, int64_t count, int bits, unsigned blocks, float max_norm, float* norm,
                       void* ws, hipStream_t st) {
  char* const base = static_cast<char*>(ws);
  ClipTable<kOut> t = {};
  t.chunk_bits = bits;
  t.max_norm = max_norm;
  t.norm = norm;
  t.ticket = reinterpret_cast<unsigned int*>(base + kWsTicketOffset);
  t.factor = reinterpret_cast<float*>(base + kWsFactorOffset);
  t.counters = reinterpret_cast<unsigned int*>(base + kWsHeaderBytes);
  t.partials = reinterpret_cast<double*>(base + kWsDataOffset);
  int64_t from = 0;
  do {
    const int64_t n = fill(items, count, from, &t);
    t.first = from == 0;
    t.last = from + n == count;
    if constexpr (kOut) hipLaunchKernelGGL(clip_scale_kernel, dim3(t.first_chunk[n]), dim3(kThreads), 0, st, t);
    else hipLaunchKernelGGL(clip_norm_kernel, dim3(blocks), dim3(kThreads), 0, st, t);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    from += n;
  } while (from < count);
  return hipSuccess;
}

}  // namespace

hipError_t launch_clip(const ClipItem* items, int64_t count, bool scale, float max_norm, float* norm, void* ws,
                       hipStream_t st) {
  int64_t elements = 0, chunks = 0;
  for (int64_t i = 0; i < count && elements <= kSmallCall; ++i) elements += items[i].size;
  const int bits = elements <= kSmallCall ? kSmallChunkBits : kChunkBits;
  for (int64_t i = 0; i < count && chunks < kClipMostBlocks; ++i) chunks += chunks_of(items[i].size, bits);
  const unsigned blocks = static_cast<unsigned>(chunks < 1 ? 1 : chunks < kClipMostBlocks ? chunks : kClipMostBlocks);
  const hipError_t e = launch_pass<false>(items, count, bits, blocks, max_norm, norm, ws, st);
  if (e != hipSuccess || !scale || count == 0) return e;
  return launch_pass<true>(items, count, bits, blocks, max_norm, norm, ws, st);
}

}  // namespace vtrace
