// The vocabulary's rows as a network's inputs, and their gradient:
//   rows[n, :] = scale table[a_n, :],   d_table[v, :] = scale sum over {n : a_n = v} of d_rows[n, :].
//
// Both are bound by memory.  The gradient's steps are put in the order of their tokens (stable:
// a token's steps stay in theirs, so that sums are the same in every call), cut into chunks of
// as many steps, and a chunk's runs of one token are summed in registers.  A run inside a chunk
// is a row of the result; what a run leaves in a chunk that it enters or leaves is a partial
// sum, added to the others of its run by a second launch.  No atomics: a frequent token's
// thousands of steps are read by as many chunks as anything else.
//
// Sums are float32 within a chunk (at most kMostChunk steps) and float64 over the chunks.
#include "device_common.hpp"
#include "embed.hpp"
#include "wave_ops.hpp"

#include <algorithm>

namespace vtrace {
namespace {

constexpr int kThreads = 256;
// A thread's elements of a row: one 16-byte vector of bfloat16, two of float32.
constexpr int kUnit = 8;

struct Unit {
  float x[kUnit];
};
// The same as it lies in memory.
template <typename T>
struct Raw {
  v4u w[kUnit * sizeof(T) / 16];
};

template <typename T>
__device__ __forceinline__ Raw<T> load_raw(const T* p) {
  Raw<T> r;
#pragma unroll
  for (unsigned h = 0; h < sizeof(r.w) / 16; ++h) r.w[h] = reinterpret_cast<const v4u*>(p)[h];
  return r;
}
__device__ __forceinline__ Unit values(const Raw<uint16_t>& r) {
  Unit u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u.x[2 * i] = __uint_as_float(r.w[0][i] << 16);
    u.x[2 * i + 1] = __uint_as_float(r.w[0][i] & 0xffff0000u);
  }
  return u;
}
__device__ __forceinline__ Unit values(const Raw<float>& r) {
  Unit u;
#pragma unroll
  for (int i = 0; i < kUnit; ++i) u.x[i] = __uint_as_float(r.w[i / 4][i % 4]);
  return u;
}
template <typename T>
__device__ __forceinline__ Unit load_unit(const T* p) {
  return values(load_raw(p));
}
template <bool kPast>
__device__ __forceinline__ void store_vector(v4u* p, const v4u& w) {
  if constexpr (kPast) __builtin_nontemporal_store(w, p);
  else *p = w;
}
// kPast: past the caches.
template <bool kPast = false>
__device__ __forceinline__ void store_unit(uint16_t* p, const Unit& u) {
  v4u w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(u.x[2 * i], u.x[2 * i + 1]);
  store_vector<kPast>(reinterpret_cast<v4u*>(p), w);
}
template <bool kPast = false>
__device__ __forceinline__ void store_unit(float* p, const Unit& u) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    v4u w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(u.x[4 * h + i]);
    store_vector<kPast>(reinterpret_cast<v4u*>(p) + h, w);
  }
}

// How many threads share a row: a power of two, up to a workgroup.
int row_lanes_log2(int64_t H, int most_log2) {
  int bits = 0;
  while (bits < most_log2 && (int64_t(kUnit) << bits) < H) ++bits;
  return bits;
}
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int64_t kCachedBytes = int64_t(1) << 27;  // half of the Infinity Cache

// kRows rows a group of threads, their loads in flight together.  Outputs larger than what the
// caches hold go past them: 65536 rows of 2048 bfloat16 87 -> 60 us (2 or 8 rows a group: 88, 108),
// 4.5 TB/s of stores and 1.4 of distinct rows; 48 rows 2.9 us, a launch.
template <typename In, typename Out, int kRows, bool kPast>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedArgs a, int lanes_log2) {
  const int groups = kThreads >> lanes_log2, lanes = 1 << lanes_log2;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kRows * groups + (threadIdx.x >> lanes_log2);
  const int lane = threadIdx.x & (lanes - 1), units = static_cast<int>(a.H / kUnit);
  int32_t token[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int64_t n = first + r * groups;
    token[r] = a.tokens[n < a.N ? n : a.N - 1];
    if (n < a.N && lane == 0 && token[r] != -1 && (token[r] < 0 || token[r] >= a.V)) raise_error_flag(a.error_flag);
  }
  for (int c = lane; c < units; c += lanes) {
    // (Loads under a condition would be waited for one by one: tokens that are none read row 0.)
    Raw<In> row[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int64_t t = token[r] >= 0 && token[r] < a.V ? token[r] : 0;
      row[r] = load_raw(static_cast<const In*>(a.table) + t * a.H + c * kUnit);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int64_t n = first + r * groups;
      if (n >= a.N) continue;
      const bool valid = token[r] >= 0 && token[r] < a.V;
      Unit u = values(row[r]);
#pragma unroll
      for (int i = 0; i < kUnit; ++i) u.x[i] = valid ? u.x[i] * a.scale : token[r] == -1 ? 0.0f : NAN;
      store_unit<kPast>(static_cast<Out*>(a.rows) + n * a.H + c * kUnit, u);
    }
  }
}

// ---- The steps in the order of their tokens. ----

// Up to here every step's place is counted directly, N^2 comparisons in one launch.  Onto 32768 rows of 256,
// us so and sorted by digits: 4096 steps 16.3, 30.2; 8192 21.6, 33.3; 12288 32.7, 35.8; 16384 44.0, 39.0; onto
// 131072 rows of 1024: 12288 44.3, 46.3; 16384 52.2, 46.9.
constexpr int64_t kMostRanked = 12288;
constexpr int kRankThreads = 1024;

__device__ __forceinline__ bool invalid(int32_t token, int64_t V) { return token != -1 && (token < 0 || token >= V); }

// A workgroup's 16 steps: each 16 threads count one 64th of all steps that come before them, from
// LDS, where all tokens are.  Tokens compare as unsigned numbers, so that what is no token of the
// vocabulary comes last.  Bound by the comparisons where N is some thousands (with 64 steps a
// workgroup, which leaves most CUs without one, 3200 steps 9.7 us, so 5.5).
constexpr int kRankSteps = 16;
__global__ __launch_bounds__(kRankThreads) void embed_rank_kernel(EmbedArgs a) {
  constexpr int kSlices = kRankThreads / kRankSteps;
  __shared__ __align__(16) uint32_t s_token[kMostRanked];
  __shared__ int s_rank[kSlices][kRankSteps];
  const int step = threadIdx.x % kRankSteps, slice = threadIdx.x / kRankSteps;
  const int N = static_cast<int>(a.N);
  const int n0 = blockIdx.x * kRankSteps, n = n0 + step;
  // In fours, whose last one is filled up with what comes behind everything.
  const int fours = (N + 3) / 4;
  for (int j = threadIdx.x; j < 4 * fours; j += kRankThreads) s_token[j] = j < N ? static_cast<uint32_t>(a.tokens[j]) : 0xffffffffu;
  __syncthreads();
  const uint32_t mine = n < N ? s_token[n] : 0xffffffffu;
  const int per = (fours + kSlices - 1) / kSlices;
  const int from = slice * per < fours ? slice * per : fours, to = from + per < fours ? from + per : fours;
  auto inside = [&](int j) { return j < from ? from : j > to ? to : j; };
  const int own = inside(n0 / 4), behind = inside((n0 + kRankSteps) / 4);
  int rank = 0;
#pragma unroll 4
  for (int j = from; j < own; ++j) {
    const v4u t = *reinterpret_cast<const v4u*>(s_token + 4 * j);
#pragma unroll
    for (int q = 0; q < 4; ++q) rank += t[q] <= mine;
  }
  for (int j = 4 * own; j < 4 * behind; ++j) rank += s_token[j] < mine || (s_token[j] == mine && j < n);
#pragma unroll 4
  for (int j = behind; j < to; ++j) {
    const v4u t = *reinterpret_cast<const v4u*>(s_token + 4 * j);
#pragma unroll
    for (int q = 0; q < 4; ++q) rank += t[q] < mine;
  }
  s_rank[slice][step] = rank;
  __syncthreads();
  // Sums over the slices: four threads of a wave a step, then their sums.
  if (threadIdx.x >= kWave) return;
  int at = 0;
#pragma unroll
  for (int w = 0; w < kSlices / 4; ++w) at += s_rank[4 * w + slice][step];
  at += __shfl_xor(at, 16, kWave);
  at += __shfl_xor(at, 32, kWave);
  if (slice != 0 || n >= N) return;
  a.keys[0][at] = mine;
  a.steps[0][at] = static_cast<uint32_t>(n);
  if (invalid(static_cast<int32_t>(mine), a.V)) raise_error_flag(a.error_flag);
}

// More steps: passes over digits of the token, from the lowest up, each of them stable: of 65536 steps
// two passes, 5 us to count and 9 to move.  A pass
// counts every block's digits, adds the counts up in the order (digit, block), and moves.
constexpr int kMostDigitBits = 9, kMostDigits = 1 << kMostDigitBits;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kSortItems = 2048;  // of a block
constexpr int kSortRounds = kSortItems / kSortThreads;  // of 64 consecutive items a wave
constexpr int kScanThreads = 1024;

// What is no token of the vocabulary is V.
__device__ __forceinline__ uint32_t sort_key(const EmbedArgs& a, int from, int64_t i) {
  if (from >= 0) return a.keys[from][i];
  const uint32_t t = static_cast<uint32_t>(a.tokens[i]);
  return t < static_cast<uint32_t>(a.V) ? t : static_cast<uint32_t>(a.V);
}

// A wave's items of a block, `kSortRounds` times 64 in their order: what each has before it of the
// same digit among them, and in s_at how many there are of each digit.  Frequent tokens give most
// lanes the same digit: lanes find each other by its bits and one of them counts.
struct SortItems {
  uint32_t key[kSortRounds];
  int rank[kSortRounds];
  int64_t first;
};
__device__ __forceinline__ void rank_items(const EmbedArgs& a, int from, int shift, int bits, uint32_t* s_at, SortItems* t) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  t->first = static_cast<int64_t>(blockIdx.x) * kSortItems + wave * (kSortRounds * kWave) + lane;
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) t->key[r] = sort_key(a, from, t->first + r * kWave < a.N ? t->first + r * kWave : a.N - 1);
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const bool in = t->first + r * kWave < a.N;
    const int d = (t->key[r] >> shift) & ((1 << bits) - 1);
    unsigned long long same = __ballot(in);
    for (int b = 0; b < bits; ++b) {
      const unsigned long long set = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? set : ~set;
    }
    const int before = __popcll(same & ((1ull << lane) - 1));
    const uint32_t at = s_at[d];
    __builtin_amdgcn_wave_barrier();  // every lane has read before one of them writes
    if (in && before == 0) s_at[d] = at + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    t->rank[r] = at + before;
  }
}

__global__ __launch_bounds__(kSortThreads) void embed_count_kernel(EmbedArgs a, int from, int shift, int bits) {
  __shared__ uint32_t s_at[kSortWaves][kMostDigits];
  for (int d = threadIdx.x; d < kSortWaves * kMostDigits; d += kSortThreads) s_at[d / kMostDigits][d % kMostDigits] = 0;
  __syncthreads();
  SortItems t;
  rank_items(a, from, shift, bits, s_at[threadIdx.x / kWave], &t);
  if (from < 0) {
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
      if (t.first + r * kWave < a.N && invalid(a.tokens[t.first + r * kWave], a.V)) raise_error_flag(a.error_flag);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < 1 << bits; d += kSortThreads) {
    uint32_t n = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) n += s_at[w][d];
    a.counts[static_cast<int64_t>(d) * gridDim.x + blockIdx.x] = n;
  }
}

// counts[i] = sum of counts[0 .. i), by one workgroup.
__global__ __launch_bounds__(kScanThreads) void embed_scan_kernel(uint32_t* counts, int64_t n) {
  constexpr int kWaves = kScanThreads / kWave, kItems = 4;
  __shared__ uint32_t s_sum[2][kWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  uint32_t total = 0;
  int flip = 0;
  for (int64_t base = 0; base < n; base += kScanThreads * kItems, flip ^= 1) {
    const int64_t first = base + static_cast<int64_t>(threadIdx.x) * kItems;
    uint32_t x[kItems], mine = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      x[i] = first + i < n ? counts[first + i] : 0;
      mine += x[i];
    }
    uint32_t upto = mine;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t y = __shfl_up(upto, o, kWave);
      if (lane >= o) upto += y;
    }
    if (lane == kWave - 1) s_sum[flip][wave] = upto;
    __syncthreads();
    uint32_t at = total + upto - mine;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t s = s_sum[flip][w];
      if (w < wave) at += s;
      total += s;
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      if (first + i < n) counts[first + i] = at;
      at += x[i];
    }
  }
}

// kScans: up to kMostSelfScanned blocks add up the counts themselves.
constexpr int kMostSelfScanned = 64;
template <bool kScans>
__global__ __launch_bounds__(kSortThreads) void embed_move_kernel(EmbedArgs a, int from, int to, int shift, int bits) {
  __shared__ uint32_t s_at[kSortWaves][kMostDigits];
  __shared__ uint32_t s_digits[kMostDigits / kWave];
  uint32_t own = 0, all = 0;  // a thread's digit: in the blocks before this one, and in all
  if constexpr (kScans) {
    if (static_cast<int>(threadIdx.x) < 1 << bits) {
      const uint32_t* const counts = a.counts + static_cast<int64_t>(threadIdx.x) * gridDim.x;
#pragma unroll 16
      for (unsigned b = 0; b < gridDim.x; ++b) {
        const uint32_t n = counts[b];
        all += n;
        if (b < blockIdx.x) own += n;
      }
    }
  }
  for (int d = threadIdx.x; d < kSortWaves * kMostDigits; d += kSortThreads) s_at[d / kMostDigits][d % kMostDigits] = 0;
  __syncthreads();
  SortItems t;
  const int wave = threadIdx.x / kWave;
  rank_items(a, from, shift, bits, s_at[wave], &t);
  uint32_t step[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const int64_t i = t.first + r * kWave;
    step[r] = from < 0 ? static_cast<uint32_t>(i) : a.steps[from][i < a.N ? i : a.N - 1];
  }
  if constexpr (kScans) {
    // And those of all smaller digits.
    uint32_t upto = all;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t y = __shfl_up(upto, o, kWave);
      if (static_cast<int>(threadIdx.x) % kWave >= o) upto += y;
    }
    if (threadIdx.x % kWave == kWave - 1 && threadIdx.x < kMostDigits) s_digits[threadIdx.x / kWave] = upto;
    own += upto - all;
  }
  __syncthreads();
  if constexpr (kScans) {
    for (int w = 0; w < wave && w < kMostDigits / kWave; ++w) own += s_digits[w];
  }
  for (int d = threadIdx.x; d < 1 << bits; d += kSortThreads) {
    uint32_t at = kScans ? own : a.counts[static_cast<int64_t>(d) * gridDim.x + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t n = s_at[w][d];
      s_at[w][d] = at;
      at += n;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    if (t.first + r * kWave >= a.N) continue;
    const uint32_t at = s_at[wave][(t.key[r] >> shift) & ((1 << bits) - 1)] + t.rank[r];
    a.keys[to][at] = t.key[r];
    a.steps[to][at] = step[r];
  }
}

// ---- Sums. ----

constexpr int kLeastChunk = 4, kMostChunk = 128;
constexpr int kWorkgroups = 1024;  // least, where chunks are longer than the shortest
constexpr int kBatch = 8;  // rows of a chunk in flight
constexpr int kFillRows = 256;  // most rows of a workgroup that fills
constexpr int64_t kFillBytes = 65536;

// A run's sum, scaled and (with `was`) added to what its row held.
template <typename Out>
__device__ __forceinline__ void write_row(Out* p, const Unit& sum, float scale, bool accumulate, const Unit& was) {
  Unit u;
#pragma unroll
  for (int i = 0; i < kUnit; ++i) u.x[i] = accumulate ? fmaf(sum.x[i], scale, was.x[i]) : sum.x[i] * scale;
  store_unit(p, u);
}

// The place of the first sorted step whose token is not before v, by a workgroup: 256 places at a
// time.
__device__ __forceinline__ int64_t first_step_of(const EmbedArgs& a, int64_t v) {
  __shared__ int s_before[kThreads / kWave];
  int64_t lo = 0, hi = a.N;
  while (lo < hi) {
    const int64_t stride = (hi - lo + kThreads - 1) / kThreads, at = lo + threadIdx.x * stride;
    const unsigned long long before = __ballot(at < hi && a.keys[0][at] < v);
    if (threadIdx.x % kWave == 0) s_before[threadIdx.x / kWave] = __popcll(before);
    __syncthreads();
    int n = 0;
#pragma unroll
    for (int w = 0; w < kThreads / kWave; ++w) n += s_before[w];
    __syncthreads();
    if (n == 0) return lo;
    const int64_t end = lo + n * stride;
    lo += (n - 1) * stride + 1;
    hi = end < hi ? end : hi;
  }
  return lo;
}

// Zeros in the rows of tokens that no step has: workgroup `block` of those that do this.  Rows are
// vectors of 16 bytes, 1 << lanes_log2 threads each.
template <typename Out>
__device__ void fill_rows(const EmbedArgs& a, int64_t block, int rows, int lanes_log2) {
  __shared__ int s_present[kFillRows];
  const int64_t v0 = block * rows, v1 = v0 + rows < a.V ? v0 + rows : a.V;
  if (static_cast<int>(threadIdx.x) < rows) s_present[threadIdx.x] = 0;
  const int64_t first = first_step_of(a, v0);  // behind a barrier, unless there is no step
  __syncthreads();
  // The steps of these rows: all of them, or after some a search for each row that is not met yet.
  constexpr int kMostLooks = 4;
  int64_t i = first + threadIdx.x;
  for (int look = 0; look < kMostLooks; ++look, i += kThreads) {
    const uint32_t key = i < a.N ? a.keys[0][i] : 0xffffffffu;
    if (key < v1) s_present[key - v0] = 1;
    if (!__syncthreads_or(i == first + (look + 1) * kThreads - 1 && key < v1)) break;
    if (look + 1 < kMostLooks || static_cast<int>(threadIdx.x) >= v1 - v0) continue;
    const int64_t v = v0 + threadIdx.x;
    int64_t lo = first, hi = a.N;
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (a.keys[0][mid] < v) lo = mid + 1;
      else hi = mid;
    }
    if (lo < a.N && a.keys[0][lo] == v) s_present[threadIdx.x] = 1;
  }
  __syncthreads();
  const int lanes = 1 << lanes_log2, vectors = static_cast<int>(a.H * sizeof(Out) / 16);
  const v4u zero = {0u, 0u, 0u, 0u};
  for (int r = threadIdx.x >> lanes_log2; r < v1 - v0; r += kThreads >> lanes_log2) {
    if (s_present[r]) continue;
    v4u* const row = reinterpret_cast<v4u*>(static_cast<Out*>(a.d_table) + (v0 + r) * a.H);
    for (int c = threadIdx.x & (lanes - 1); c < vectors; c += lanes) row[c] = zero;
  }
}

__device__ __forceinline__ float* partial_row(const EmbedArgs& a, int64_t chunk, int which) {
  return a.partials + (2 * chunk + which) * a.H;
}

// Chunks of the sorted steps, one a group of threads (and a slab of the row, where it has more
// than a workgroup's units); then, in further workgroups, the rows that no step has.
// Bound by memory where steps or rows are many: 65536 steps of 2048 bfloat16 added to 20088 rows 97 us,
// 4.5 TB/s; 3200 steps of 1024 and 32768 rows 14 us, 5.2 TB/s, most of it the rows of no step.
// Slot 0 of a chunk's partial sums is that of the run that comes from the chunk before it,
// slot 1 of the one that begins here and goes on behind it.
template <typename In, typename Out, bool kAccumulate>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(EmbedArgs a, int lanes_log2, int slabs, int64_t sum_blocks,
                                                             int fill, int fill_lanes_log2) {
  if constexpr (!kAccumulate) {
    if (blockIdx.x >= sum_blocks) {
      fill_rows<Out>(a, blockIdx.x - sum_blocks, fill, fill_lanes_log2);
      return;
    }
  }
  const int lanes = 1 << lanes_log2;
  const int64_t chunk = static_cast<int64_t>(blockIdx.x / slabs) * (kThreads >> lanes_log2) + (threadIdx.x >> lanes_log2);
  const int64_t begin = chunk * a.chunk;
  const int unit = static_cast<int>(blockIdx.x % slabs) * kThreads + (threadIdx.x & (lanes - 1));
  if (begin >= a.N || unit >= static_cast<int>(a.H / kUnit)) return;
  const int64_t end = begin + a.chunk < a.N ? begin + a.chunk : a.N;
  const uint32_t* const keys = a.keys[0];
  const uint32_t V = static_cast<uint32_t>(a.V);
  const int64_t column = static_cast<int64_t>(unit) * kUnit;
  const In* const d_rows = static_cast<const In*>(a.d_rows) + column;
  Out* const d_table = static_cast<Out*>(a.d_table) + column;
  const uint32_t previous = begin > 0 ? keys[begin - 1] : 0xffffffffu;
  bool first = true;  // the chunk's first run, which may come from the chunk before
  Unit sum = {};
  for (int64_t i = begin; i < end; i += kBatch) {
    // Tokens one step further than the batch: a run ends where the next one differs.  (Loads under
    // a condition would be waited for one by one: what is behind the end is read at the last
    // step, and where no run ends a step's own row in place of the table's.)
    uint32_t key[kBatch + 1], step[kBatch];
#pragma unroll
    for (int b = 0; b <= kBatch; ++b) key[b] = keys[i + b < a.N ? i + b : a.N - 1];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) step[b] = a.steps[0][i + b < end ? i + b : end - 1];
#pragma unroll
    for (int b = 0; b <= kBatch; ++b)
      if (i + b >= a.N) key[b] = 0xffffffffu;
    if (key[0] >= V) break;
    Raw<In> row[kBatch];
    Raw<Out> was[kAccumulate ? kBatch : 1];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const In* const from = d_rows + static_cast<int64_t>(step[b]) * a.H;
      row[b] = load_raw(from);
      if constexpr (kAccumulate) {
        const void* const other = sizeof(Out) > sizeof(In) ? static_cast<const void*>(d_table) : from;
        const void* const held = d_table + static_cast<int64_t>(key[b]) * a.H;
        was[b] = load_raw(static_cast<const Out*>(key[b] < V && key[b] != key[b + 1] ? held : other));
      }
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (i + b >= end || key[b] >= V) continue;
      const Unit u = values(row[b]);
#pragma unroll
      for (int e = 0; e < kUnit; ++e) sum.x[e] += u.x[e];
      const bool ends = key[b] != key[b + 1];
      if (!ends && i + b + 1 < end) continue;
      if (first && previous == key[b]) store_unit(partial_row(a, chunk, 0) + column, sum);
      else if (!ends) store_unit(partial_row(a, chunk, 1) + column, sum);
      else write_row(d_table + static_cast<int64_t>(key[b]) * a.H, sum, a.scale, kAccumulate, kAccumulate ? values(was[kAccumulate ? b : 0]) : Unit{});
      first = false;
#pragma unroll
      for (int e = 0; e < kUnit; ++e) sum.x[e] = 0.0f;
    }
  }
}

// The run that begins in a chunk and goes on behind it: its parts, in order, in float64; the
// groups of a workgroup take turns with them.  5 us, a launch; 11 of 65536 steps of 2048 where one
// token has 3900 of them, eight parts in flight.
constexpr int kJoinThreads = 256;
template <typename Out>
__global__ __launch_bounds__(kJoinThreads) void embed_join_kernel(EmbedArgs a, int lanes_log2, int slabs) {
  __shared__ double s_sum[kJoinThreads][kUnit];
  const int64_t chunk = blockIdx.x / slabs;
  const int64_t begin = chunk * a.chunk, end = begin + a.chunk;
  const uint32_t* const keys = a.keys[0];
  if (end >= a.N) return;
  const uint32_t run = keys[end - 1], after = keys[end], before = begin > 0 ? keys[begin - 1] : 0xffffffffu;
  if (run >= static_cast<uint32_t>(a.V) || after != run || before == run) return;
  // The last chunk that begins with it: as many as there are threads at a time.
  int64_t last = chunk + 1;
  for (bool more = true; more;) {
    const int64_t at = (last + 1 + threadIdx.x) * a.chunk;
    const int n = __syncthreads_count(at < a.N && keys[at] == run);
    last += n;
    more = n == kJoinThreads;
  }
  const int lanes = 1 << lanes_log2, groups = kJoinThreads >> lanes_log2, group = threadIdx.x >> lanes_log2;
  const int unit = static_cast<int>(blockIdx.x % slabs) * lanes + (threadIdx.x & (lanes - 1));
  const bool in = unit < static_cast<int>(a.H / kUnit);
  const int64_t column = static_cast<int64_t>(unit) * kUnit;
  double sum[kUnit] = {};
  if (in) {
    // Parts: this chunk's own, and of each that follows the first.  Eight in flight.
    constexpr int kParts = 8;
    for (int64_t c = chunk + group; c <= last; c += groups * kParts) {
      Raw<float> part[kParts];
#pragma unroll
      for (int k = 0; k < kParts; ++k) {
        const int64_t at = c + k * groups <= last ? c + k * groups : last;
        part[k] = load_raw(static_cast<const float*>(partial_row(a, at, at == chunk ? 1 : 0) + column));
      }
#pragma unroll
      for (int k = 0; k < kParts; ++k) {
        if (c + k * groups > last) continue;
        const Unit u = values(part[k]);
#pragma unroll
        for (int e = 0; e < kUnit; ++e) sum[e] += static_cast<double>(u.x[e]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kUnit; ++e) s_sum[threadIdx.x][e] = sum[e];
  __syncthreads();
  if (group != 0 || !in) return;
  for (int g = 1; g < groups; ++g)
#pragma unroll
    for (int e = 0; e < kUnit; ++e) sum[e] += s_sum[g * lanes + threadIdx.x][e];
  Unit u;
#pragma unroll
  for (int e = 0; e < kUnit; ++e) u.x[e] = static_cast<float>(sum[e]);
  Out* const to = static_cast<Out*>(a.d_table) + static_cast<int64_t>(run) * a.H + column;
  write_row(to, u, a.scale, a.accumulate, a.accumulate ? load_unit(static_cast<const Out*>(to)) : Unit{});
}

template <typename In, typename Out>
hipError_t launch_sums(const EmbedArgs& a, hipStream_t st) {
  const int lanes = row_lanes_log2(a.H, 8);
  const int64_t slabs = ceil_div(a.H / kUnit, kThreads), chunks = ceil_div(a.N, a.chunk);
  const int64_t sums = ceil_div(chunks, kThreads >> lanes) * slabs;
  int64_t fill = 0, fills = 0;
  if (!a.accumulate) {
    fill = kFillBytes / (a.H * static_cast<int64_t>(sizeof(Out)));
    fill = fill < 1 ? 1 : fill > kFillRows ? kFillRows : fill;
    fills = ceil_div(a.V, fill);
  }
  const int fill_lanes = row_lanes_log2(a.H * static_cast<int64_t>(sizeof(Out)) / 2, 8);  // 16 bytes each
  const dim3 grid(static_cast<unsigned>(sums + fills));
  if (a.accumulate)
    hipLaunchKernelGGL((embed_sum_kernel<In, Out, true>), grid, dim3(kThreads), 0, st, a, lanes, static_cast<int>(slabs), sums, 0, 0);
  else
    hipLaunchKernelGGL((embed_sum_kernel<In, Out, false>), grid, dim3(kThreads), 0, st, a, lanes, static_cast<int>(slabs), sums,
                       static_cast<int>(fill), fill_lanes);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || chunks < 2) return e;
  const int join_lanes = row_lanes_log2(a.H, 6);
  const int64_t join_slabs = ceil_div(a.H / kUnit, int64_t(1) << join_lanes);
  hipLaunchKernelGGL(embed_join_kernel<Out>, dim3(static_cast<unsigned>(chunks * join_slabs)), dim3(kJoinThreads), 0, st, a,
                     join_lanes, static_cast<int>(join_slabs));
  return hipGetLastError();
}

int token_bits(int64_t V) {
  int all = 1;  // keys are 0 .. V
  while ((V >> all) != 0) ++all;
  return all;
}
int passes_of(int64_t V, int* bits) {
  const int all = token_bits(V), passes = (all + kMostDigitBits - 1) / kMostDigitBits;
  *bits = (all + passes - 1) / passes;
  return passes;
}

// Which of the two buffers the first pass fills, so that the last one fills buffer 0.
hipError_t launch_order(const EmbedArgs& a, const EmbedPlan& p, hipStream_t st) {
  if (p.ranks) {
    hipLaunchKernelGGL(embed_rank_kernel, dim3(static_cast<unsigned>(ceil_div(a.N, kRankSteps))), dim3(kRankThreads), 0, st, a);
    return hipGetLastError();
  }
  int bits = 0;
  const int passes = passes_of(a.V, &bits);
  const int64_t blocks = ceil_div(a.N, kSortItems);
  int from = -1;
  for (int pass = 0; pass < passes; ++pass) {
    const int to = (passes - 1 - pass) % 2;
    const dim3 grid(static_cast<unsigned>(blocks));
    hipLaunchKernelGGL(embed_count_kernel, grid, dim3(kSortThreads), 0, st, a, from, pass * bits, bits);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (blocks <= kMostSelfScanned) {
      hipLaunchKernelGGL(embed_move_kernel<true>, grid, dim3(kSortThreads), 0, st, a, from, to, pass * bits, bits);
    } else {
      hipLaunchKernelGGL(embed_scan_kernel, dim3(1), dim3(kScanThreads), 0, st, a.counts, blocks << bits);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(embed_move_kernel<false>, grid, dim3(kSortThreads), 0, st, a, from, to, pass * bits, bits);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    from = to;
  }
  return hipSuccess;
}

template <typename In, typename Out>
hipError_t launch_lookup(const EmbedArgs& a, hipStream_t st) {
  const int lanes = row_lanes_log2(a.H, 8), groups = kThreads >> lanes;
  auto launch = [&](auto kernel, int rows) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(ceil_div(a.N, rows * groups))), dim3(kThreads), 0, st, a, lanes);
  };
  if (a.N < 4096 * groups) launch(embed_kernel<In, Out, 1, false>, 1);
  else if (a.N * a.H * static_cast<int64_t>(sizeof(Out)) < kCachedBytes) launch(embed_kernel<In, Out, 4, false>, 4);
  else launch(embed_kernel<In, Out, 4, true>, 4);
  return hipGetLastError();
}

}  // namespace

EmbedPlan plan_embed_grad(int64_t N, int64_t V, int64_t H) {
  EmbedPlan p = {};
  p.ranks = N <= kMostRanked;
  // Chunks as long as leave a thousand workgroups: four a CU, with kBatch rows each in flight.
  const int lanes = row_lanes_log2(H, 8);
  const int64_t slabs = ceil_div(H / kUnit, kThreads), groups = kThreads >> lanes;
  p.chunk = kLeastChunk;
  while (p.chunk < kMostChunk && N * slabs / (groups * p.chunk * 2) >= kWorkgroups) p.chunk *= 2;
  size_t at = kWsDataOffset;
  auto take = [&](size_t bytes) {
    const size_t begin = at;
    at += (bytes + 255) / 256 * 256;
    return begin;
  };
  const int buffers = p.ranks ? 1 : 2;
  for (int b = 0; b < buffers; ++b) {
    p.keys_at[b] = take(N * 4);
    p.steps_at[b] = take(N * 4);
  }
  // What is taken is enough for fewer steps, fewer tokens and shorter rows too, so that the bytes for
  // the largest call serve all of them.  Fewer tokens may be sorted in fewer passes of more bits.
  if (!p.ranks) p.counts_at = take((ceil_div(N, kSortItems) << std::min(token_bits(V), kMostDigitBits)) * 4);
  // Chunks that are twice as long halve the partial sums, and fewer steps have more of them: chunks that
  // are not of kMostChunk are less than 2 kWorkgroups groups / slabs, whose rows have at most kThreads kUnit slabs /
  // groups elements (and one row for the chunk that is not whole).
  const int64_t least = ceil_div(N, kLeastChunk) * H, most = int64_t(2) * kWorkgroups * kThreads * kUnit + H;
  p.partials_at = take(std::max({ceil_div(N, p.chunk) * H, ceil_div(N, kMostChunk) * H, std::min(least, most)}) * 2 * 4);
  p.bytes = at;
  return p;
}

void attach_embed_grad(EmbedArgs* a, const EmbedPlan& p, void* ws) {
  char* const base = static_cast<char*>(ws);
  a->error_flag = reinterpret_cast<unsigned int*>(base + kWsFlagOffset);
  for (int b = 0; b < 2; ++b) {
    a->keys[b] = reinterpret_cast<uint32_t*>(base + p.keys_at[b]);
    a->steps[b] = reinterpret_cast<uint32_t*>(base + p.steps_at[b]);
  }
  a->counts = reinterpret_cast<uint32_t*>(base + p.counts_at);
  a->partials = reinterpret_cast<float*>(base + p.partials_at);
  a->chunk = p.chunk;
}

hipError_t launch_embed(const EmbedArgs& a, hipStream_t st) {
  if (a.table_bf16) return a.steps_bf16 ? launch_lookup<uint16_t, uint16_t>(a, st) : launch_lookup<uint16_t, float>(a, st);
  return a.steps_bf16 ? launch_lookup<float, uint16_t>(a, st) : launch_lookup<float, float>(a, st);
}

hipError_t launch_embed_grad(const EmbedArgs& a, const EmbedPlan& p, hipStream_t st) {
  const hipError_t e = launch_order(a, p, st);
  if (e != hipSuccess) return e;
  if (a.steps_bf16) return a.table_bf16 ? launch_sums<uint16_t, uint16_t>(a, st) : launch_sums<uint16_t, float>(a, st);
  return a.table_bf16 ? launch_sums<float, uint16_t>(a, st) : launch_sums<float, float>(a, st);
}

}  // namespace vtrace
