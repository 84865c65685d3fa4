// The vocabulary layer: workspaces, launches, and the small kernels around the tiles
// (vocab_logits.hip, vocab_products.hip) and the few-step kernel (vocab_stream.hip).
#include "vocab_impl.hpp"

namespace vtrace {
namespace {

// Tiles that d_hidden's product is split up to: two rounds.
__host__ __device__ constexpr int most_split_tiles(int size) { return 2 * resident_tiles(size); }

__host__ __device__ inline int hidden_tile(const VocabArgs& a) { return a.small_hidden ? kSmallTile : kTile; }

constexpr int kListThreads = 1024;
constexpr int kListItems = 8;  // tokens per thread and pass

// How d_hidden's product is split for `count` active steps, and what it then takes (us):
// every CU has `rounds` tiles one after the other, each of them with its share of a piece's
// steps (round_cost), and in the end the parts are added, at 5 TB/s.  Considered are no parts,
// and as many as fill one round (or half a one) or two.
struct Split {
  int parts;
  double cost;
};
__host__ __device__ inline Split best_split(const VocabArgs& a, int count, int size) {
  const int tiles_n = (count + size - 1) / size, tiles = tiles_n * ((static_cast<int>(a.H) + size - 1) / size);
  const int steps = static_cast<int>(a.g_pitch / kTileK), resident = resident_tiles(size);
  Split best = {1, INFINITY};
  for (int halves = 0; halves <= 4; halves += halves < 2 ? 1 : 2) {
    int parts = tiles == 0 ? 1 : halves * resident / 2 / tiles;
    if (parts > steps) parts = steps;
    if (parts < 1) parts = 1;
    const int share = (steps + parts - 1) / parts;
    parts = (steps + share - 1) / share;  // as few as have that share
    const int rounds = (tiles * parts + resident - 1) / resident;
    const double bytes = 4.0 * parts * tiles_n * size * static_cast<double>(a.H);
    const double cost = static_cast<double>(a.pieces) * rounds * round_cost(size, share * (a.grad_bf16 ? 1 : 2)) + bytes / 5e6;
    if (cost < best.cost) best = {parts, cost};
  }
  return best;
}

// active[0 .. count) = the steps with a token, in order.  One workgroup: a pass over
// 8192 tokens counts, scans and writes.  For the gradient it also chooses the number of
// parts of d_hidden's product, which depends on the count.
template <bool kGrad>
__global__ __launch_bounds__(kListThreads) void vocab_list_kernel(VocabArgs a) {
  constexpr int kWaves = kListThreads / kWave;
  __shared__ int s_count[2][kWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int total = 0;
  int flip = 0;
  for (int64_t base = 0; base < a.N; base += kListThreads * kListItems, flip ^= 1) {
    const int64_t first = base + static_cast<int64_t>(threadIdx.x) * kListItems;
    int32_t token[kListItems];
    int mine = 0;
#pragma unroll
    for (int j = 0; j < kListItems; ++j) {
      token[j] = first + j < a.N ? a.tokens[first + j] : kNoToken;
      mine += token[j] != kNoToken;
    }
    int upto = mine;  // of this wave's lanes up to this one
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int x = __shfl_up(upto, o, kWave);
      if (lane >= o) upto += x;
    }
    if (lane == kWave - 1) s_count[flip][wave] = upto;
    __syncthreads();
    int at = total + upto - mine;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int n = s_count[flip][w];
      if (w < wave) at += n;
      total += n;
    }
#pragma unroll
    for (int j = 0; j < kListItems; ++j) {
      if (token[j] != kNoToken) a.active[at++] = static_cast<int32_t>(first + j);
    }
  }
  if (threadIdx.x == 0) *a.active_count = total;
  if (kGrad && threadIdx.x == 0) *a.splits = best_split(a, total, hidden_tile(a)).parts;
}

// A step's outputs from the joined statistics: sums of 2^d and of 2^d d, d = (z - c) log2 e.
template <bool kDot>
__device__ __forceinline__ void store_step(const VocabArgs& a, int64_t step, int64_t row, double c, double sum,
                                           double dot) {
  constexpr double kLn2 = 0.6931471805599453;
  const int32_t token = a.tokens[step];
  const double log_s = log(sum);
  const bool valid = token >= 0 && token < a.V;
  if (!valid) raise_error_flag(a.error_flag);
  a.log_sums[step] = static_cast<float>(c + log_s);
  a.log_probs[step] = valid ? static_cast<float>(static_cast<double>(a.token_logit[row]) - c - log_s) : NAN;
  if constexpr (kDot) a.entropy[step] = static_cast<float>(log_s - kLn2 * (dot / sum));
}
template <bool kDot>
__device__ __forceinline__ void store_no_step(const VocabArgs& a, int64_t step) {
  a.log_probs[step] = 0.0f;
  a.log_sums[step] = 0.0f;
  if constexpr (kDot) a.entropy[step] = 0.0f;
}

// One piece's statistics, added to sums about c.  An empty piece (nothing but -inf
// logits) has the sum 0 and no maximum.
template <bool kDot>
__device__ __forceinline__ void add_piece(const VocabArgs& a, int64_t o, float c, double& sum, double& dot) {
  const float p = a.part_sum[o];
  const double d = p == 0.0f ? 0.0 : (static_cast<double>(a.part_max[o]) - static_cast<double>(c)) * static_cast<double>(kLog2eF);
  const double ratio = static_cast<double>(__builtin_amdgcn_exp2f(static_cast<float>(d)));
  const double e = ratio * static_cast<double>(p);
  sum += e;
  if constexpr (kDot) dot += fma(e, d, ratio * static_cast<double>(a.part_dot[o]));
}
__device__ __forceinline__ float piece_top(const VocabArgs& a, int64_t o) {
  return a.part_sum[o] == 0.0f ? -INFINITY : a.part_max[o];
}

// Joins the pieces' statistics of the tiles: 16 steps a workgroup, 32 threads over the
// pieces of each.  The kernel also writes the zeros of the steps without a token.
constexpr int kJoinThreads = 512;
constexpr int kJoinRows = 16;
template <bool kDot>
__global__ __launch_bounds__(kJoinThreads) void vocab_join_kernel(VocabArgs a) {
  constexpr int kParts = kJoinThreads / kJoinRows;
  __shared__ float s_top[kParts][kJoinRows];
  __shared__ double s_sum[kParts][kJoinRows], s_dot[kParts][kJoinRows];
  const int r = threadIdx.x % kJoinRows, part = threadIdx.x / kJoinRows;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kJoinRows + r;
  if (part == 0 && row < a.N && a.tokens[row] == kNoToken) store_no_step<kDot>(a, row);
  const bool in = row < *a.active_count;
  float top = -INFINITY;
  if (in) {
#pragma unroll 8
    for (int64_t j = part; j < a.pieces; j += kParts) top = fmaxf(top, piece_top(a, j * a.row_pitch + row));
  }
  s_top[part][r] = top;
  __syncthreads();
#pragma unroll 8
  for (int q = 0; q < kParts; ++q) top = fmaxf(top, s_top[q][r]);
  const float c = top == -INFINITY ? 0.0f : top;
  double sum = 0.0, dot = 0.0;
  if (in) {
#pragma unroll 8
    for (int64_t j = part; j < a.pieces; j += kParts) add_piece<kDot>(a, j * a.row_pitch + row, c, sum, dot);
  }
  s_sum[part][r] = sum;
  if constexpr (kDot) s_dot[part][r] = dot;
  __syncthreads();
  if (part != 0 || !in) return;
  sum = 0.0;
  dot = 0.0;
#pragma unroll 8
  for (int q = 0; q < kParts; ++q) {
    sum += s_sum[q][r];
    if constexpr (kDot) dot += s_dot[q][r];
  }
  store_step<kDot>(a, a.active[row], row, c, sum, dot);
}

// The same for few steps: a workgroup a step.
constexpr int kJoinFewThreads = 256;
template <bool kDot>
__global__ __launch_bounds__(kJoinFewThreads) void vocab_join_few_kernel(VocabArgs a) {
  __shared__ float s_top[kJoinFewThreads / kWave];
  __shared__ double s_red[3 * (kJoinFewThreads / kWave)];
  const int64_t row = blockIdx.x;
  if (a.tokens[row] == kNoToken) {
    if (threadIdx.x == 0) store_no_step<kDot>(a, row);
    return;
  }
  float top = -INFINITY;
#pragma unroll 4
  for (int64_t j = threadIdx.x; j < a.pieces; j += kJoinFewThreads) top = fmaxf(top, piece_top(a, row * a.pieces + j));
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
  if (threadIdx.x % kWave == 0) s_top[threadIdx.x / kWave] = top;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kJoinFewThreads / kWave; ++q) top = fmaxf(top, s_top[q]);
  const float c = top == -INFINITY ? 0.0f : top;
  double sum = 0.0, dot = 0.0, unused = 0.0;
#pragma unroll 4
  for (int64_t j = threadIdx.x; j < a.pieces; j += kJoinFewThreads) add_piece<kDot>(a, row * a.pieces + j, c, sum, dot);
  block_sum3<kJoinFewThreads>(sum, dot, unused, s_red);
  if (threadIdx.x == 0) store_step<kDot>(a, row, row, c, sum, dot);
}

// The tiles' operands by active step: hidden states side by side with zeros behind each
// row's end and behind the last row (up to a whole tile), the tokens, and (kGrad) the
// scalars that the gradient's epilogue needs.  A wave a row; in kGrad the same waves clear
// d_hidden of the steps without a token.  (The copy takes 14 us of the largest step's 10 ms,
// and makes every operand of the products one of plain rows.)
//
// With l = log-sum, lp = log p and G = p (c + d_h' lp) + d_lp 1[v = a] (c = -d_lp - d_h
// entropy, d_h' = -d_h), the epilogue has p = 2^(z K - l2), K the float32 log2 e and l2 the
// rounded l log2 e; what the rounding of l2 does to p is a factor of each step's own, and
// goes into c0 and c1 here.  Rows behind the last get an l2 that makes p 0.
//
// kOwnList: up to 8192 steps each workgroup counts the tokens for itself and places its own
// steps, and the list is a by-product (640 steps: 5 us in place of 9 for two launches).
constexpr int kGatherThreads = 256;
constexpr int64_t kOwnListMost = 8192;
template <bool kGrad>
__device__ __forceinline__ void gather_row(const VocabArgs& a, int64_t row, int64_t step, bool in, int lane);

template <bool kGrad, bool kOwnList>
__global__ __launch_bounds__(kGatherThreads) void vocab_gather_kernel(VocabArgs a) {
  constexpr int kWaves = kGatherThreads / kWave;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
  int64_t count;
  const bool here = row < a.N, idle = here && a.tokens[row] == kNoToken;
  if constexpr (kOwnList) {
    __shared__ int s_before[kWaves], s_all[kWaves];
    int before = 0, all = 0;  // active steps before this row's, and all of them
    for (int64_t i = threadIdx.x; i < a.N; i += kGatherThreads) {
      const bool active = a.tokens[i] != kNoToken;
      all += active;
      before += active && i < row - wave;
    }
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) {
      before += __shfl_xor(before, o, kWave);
      all += __shfl_xor(all, o, kWave);
    }
    if (lane == 0) s_before[wave] = before, s_all[wave] = all;
    __syncthreads();
    before = all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      before += s_before[w];
      all += s_all[w];
    }
    for (int w = 0; w < wave; ++w) {
      const int64_t other = row - wave + w;
      before += other < a.N && a.tokens[other] != kNoToken;
    }
    count = all;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      *a.active_count = all;
      if constexpr (kGrad) *a.splits = best_split(a, all, hidden_tile(a)).parts;
    }
    if (here && !idle) {
      if (lane == 0) a.active[before] = static_cast<int32_t>(row);
      gather_row<kGrad>(a, before, row, true, lane);
    }
    if (row >= count && row < tiles_of(count, kTile) * kTile) gather_row<kGrad>(a, row, 0, false, lane);
  } else {
    count = *a.active_count;
    if (row < tiles_of(count, kTile) * kTile) gather_row<kGrad>(a, row, row < count ? a.active[row] : 0, row < count, lane);
  }
  if (kGrad && idle) {
    const int64_t bytes = a.H * (a.grad_bf16 ? 2 : 4);
    char* const out = static_cast<char*>(a.d_hidden) + row * bytes;
    const v4u zero = {0u, 0u, 0u, 0u};
    for (int64_t i = lane * 16; i < bytes; i += kWave * 16) *reinterpret_cast<v4u*>(out + i) = zero;
  }
}

// Row `row` of the operands, from `step`, or (not `in`) zeros.
template <bool kGrad>
__device__ __forceinline__ void gather_row(const VocabArgs& a, int64_t row, int64_t step, bool in, int lane) {
  const v4u zero = {0u, 0u, 0u, 0u};
  const uint16_t* const from = a.hidden + step * a.H;
  uint16_t* const out = a.x + row * a.x_pitch;
  for (int64_t i = lane * 8; i < a.x_pitch; i += kWave * 8)
    *reinterpret_cast<v4u*>(out + i) = in && i < a.H ? *reinterpret_cast<const v4u*>(from + i) : zero;
  if (lane != 0) return;
  const int32_t token = in ? a.tokens[step] : kNoToken;
  a.row_tokens[row] = token;
  if constexpr (!kGrad) return;
  float4v scalars = {1e30f, 0.0f, 0.0f, 0.0f};
  if (in) {
    constexpr double kLn2 = 0.6931471805599453;
    float d_lp = a.d_log_probs[step];
    if (token < 0 || token >= a.V) {
      raise_error_flag(a.error_flag);
      d_lp = NAN;
    }
    const double lse = a.in_log_sums[step], exact = lse / kLn2;
    const float l2 = static_cast<float>(exact);
    const double factor = __builtin_isfinite(lse) ? 1.0 + (static_cast<double>(l2) - exact) * kLn2 : 1.0;
    double c0 = -static_cast<double>(d_lp), c1 = 0.0;
    if (a.d_entropy != nullptr) {
      c1 = -static_cast<double>(a.d_entropy[step]);
      c0 += c1 * static_cast<double>(a.in_entropy[step]);
    }
    scalars[0] = l2;
    scalars[1] = static_cast<float>(c0 * factor);
    scalars[2] = static_cast<float>(c1 * factor * kLn2);
    scalars[3] = d_lp;
  }
  a.row_scalars[row] = scalars;
}

// d_hidden of the active steps from the splits' sums.
constexpr int kFinishThreads = 256;
template <typename Out>
__global__ __launch_bounds__(kFinishThreads) void vocab_finish_kernel(VocabArgs a) {
  const int64_t quads = a.H / 4;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kFinishThreads + threadIdx.x;
  const int64_t row = i / quads, h = (i % quads) * 4;
  if (row >= *a.active_count) return;
  f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
  const int splits = *a.splits;
  const int64_t rows = tiles_of(*a.active_count, hidden_tile(a)) * hidden_tile(a);
#pragma unroll 8
  for (int k = 0; k < splits; ++k) x += *reinterpret_cast<const f32x4*>(a.h_partials + (k * rows + row) * a.H + h);
  Out* const out = static_cast<Out*>(a.d_hidden) + static_cast<int64_t>(a.active[row]) * a.H + h;
  if constexpr (sizeof(Out) == 4) {
    *reinterpret_cast<f32x4*>(out) = x;
  } else {
    v2u w;
    w.x = pack_bf16x2(x[0], x[1]);
    w.y = pack_bf16x2(x[2], x[3]);
    *reinterpret_cast<v2u*>(out) = w;
  }
}

// d_bias of one piece: the sums of 64 or 128 steps each, in order.
__global__ __launch_bounds__(kFinishThreads) void vocab_bias_kernel(VocabArgs a, int64_t v_begin) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kFinishThreads + threadIdx.x;
  if (i >= a.g_pitch || v_begin + i >= a.V) return;
  const int64_t blocks = (static_cast<int64_t>(*a.active_count) + kBiasSteps - 1) / kBiasSteps;
  double sum = 0.0;
#pragma unroll 8
  for (int64_t b = 0; b < blocks; ++b) sum += static_cast<double>(a.bias_partials[b * a.g_pitch + i]);
  a.d_bias[v_begin + i] = static_cast<float>(sum);
}

int64_t round_up(int64_t n, int64_t k) { return (n + k - 1) / k * k; }
unsigned blocks_of(int64_t n, int64_t k) { return static_cast<unsigned>((n + k - 1) / k); }

// Pieces of a workspace, each on a 256-byte boundary.
struct Carver {
  uintptr_t base;  // an integer: sizes are asked for without a workspace
  size_t at = kWsDataOffset;
  explicit Carver(void* ws) : base(reinterpret_cast<uintptr_t>(ws)) {}
  template <typename T>
  T* take(int64_t n) {
    T* const p = reinterpret_cast<T*>(base + at);
    at = static_cast<size_t>(round_up(static_cast<int64_t>(at) + n * static_cast<int64_t>(sizeof(T)), 256));
    return p;
  }
};

void header(VocabArgs* a, void* ws) {
  a->error_flag = reinterpret_cast<unsigned int*>(reinterpret_cast<uintptr_t>(ws) + kWsFlagOffset);
  a->active_count = reinterpret_cast<int32_t*>(reinterpret_cast<uintptr_t>(ws) + kWsActiveCountOffset);
}

size_t carve_log_probs(VocabArgs* a, const VocabPlan& p, void* ws) {
  header(a, ws);
  Carver c(ws);
  a->row_pitch = p.row_pitch;
  a->pieces = p.pieces;
  a->tile_tokens = p.tile_tokens;
  a->narrow = p.narrow;
  a->narrow_per_cu = p.narrow_per_cu;
  a->active = c.take<int32_t>(a->N);
  a->part_max = c.take<float>(p.pieces * p.row_pitch);
  a->part_sum = c.take<float>(p.pieces * p.row_pitch);
  a->part_dot = c.take<float>(p.pieces * p.row_pitch);
  a->token_logit = c.take<float>(p.row_pitch);
  if (!p.few) {
    a->small_logits = p.small_logits;
    a->x_pitch = p.x_pitch;
    a->x = c.take<uint16_t>(p.row_pitch * p.x_pitch);
    a->row_tokens = c.take<int32_t>(p.row_pitch);
  }
  return c.at;
}

size_t carve_grad(VocabArgs* a, const VocabPlan& p, void* ws) {
  header(a, ws);
  Carver c(ws);
  a->row_pitch = p.row_pitch;
  a->x_pitch = p.x_pitch;
  a->g_pitch = p.g_pitch;
  a->small_logits = p.small_logits;
  a->small_weight = p.small_weight;
  a->small_hidden = p.small_hidden;
  a->pieces = p.pieces;
  a->splits = reinterpret_cast<int32_t*>(reinterpret_cast<uintptr_t>(ws) + kWsSplitsOffset);
  a->active = c.take<int32_t>(a->N);
  a->row_scalars = c.take<float4v>(p.row_pitch);
  a->row_tokens = c.take<int32_t>(p.row_pitch);
  a->x = c.take<uint16_t>(p.row_pitch * p.x_pitch);
  a->g = c.take<uint16_t>((a->grad_bf16 ? 1 : 2) * p.row_pitch * p.g_pitch);
  a->bias_partials = c.take<float>(p.row_pitch / kBiasSteps * p.g_pitch);
  a->h_partials = c.take<float>(p.split_rows * a->H);
  return c.at;
}

// The kernels for few steps against tiles (H = 4096, V = 131072: 128 steps 249 us, 129 in
// tiles 326; H = 512, V = 8000 19.6, 21.7).
constexpr int64_t kMostFewSteps = 128;
// Between those two.  The narrow kernel keeps more of the layer on its way, if its workgroups
// have tokens enough: 16 steps, H = 4096, V = 32000 46 us against 63 streamed, 1 step, V =
// 100003 156 against 168 (131072: 212, 208); 32 steps, H = 1024, V = 20000 16.4, 20.8; 64 steps,
// H = 256, V = 32768 14.0, 16.9.  The streaming kernel starts faster: 16 steps, H = 512, V =
// 16000 13.2 us narrow, 10.7 streamed; 32 steps, H = 4096, V = 8000 30, 28 and 64 41, 35.
bool narrow_pays(int64_t N, int64_t V, int64_t H) {
  return N > 64 || (V >= 12288 && (N > 32 || V * H > int64_t(1) << 24));
}
// Its workgroups a CU.  Up to 32 steps and few tokens: one, with more of them and more stages
// (1 step, H = 8192, V = 20000 70 us, with two 82; H = 512, V = 50000 18.5, 16.7).  More than 64
// steps: one of eight waves and 256 tokens.
int narrow_per_cu(int64_t N, int64_t V) { return N > 64 || (N <= 32 && V < 24576) ? 1 : 2; }

// G is written and read twice within the 256 MB Infinity Cache: as one piece of the
// vocabulary where it fits, and otherwise in pieces of half of it (or one tile's columns).
// 4096 steps, H = 4096, V = 131072 (1.07 GB, bfloat16): pieces of 128 MB 9.96 ms, of 96
// 10.02, of 256 10.30, of 1024 10.48; 3200 steps, H = 1024, V = 32768 (213 MB): one piece 660
// us, two 685.
constexpr int64_t kOnePieceBytes = int64_t(256) << 20, kPieceBytes = int64_t(128) << 20;

// Whether a product m x n over `steps` steps of 64 k is done in tiles of 128 rather than of
// 256.
bool small_tiles_pay(int64_t m, int64_t n, int64_t steps) {
  auto cost = [&](int size) {
    const int64_t tiles = tiles_of(m, size) * tiles_of(n, size), resident = resident_tiles(size);
    return static_cast<double>((tiles + resident - 1) / resident) * round_cost(size, steps);
  };
  return cost(kSmallTile) < cost(kTile);
}

}  // namespace

VocabPlan plan_vocab_log_probs(int64_t N, int64_t V, int64_t H) {
  VocabPlan p = {};
  p.few = N <= kMostFewSteps;
  if (p.few) {
    p.row_pitch = N;
    p.narrow = narrow_pays(N, V, H);
    if (p.narrow) {
      // As few rounds over the workgroups that fit the GPU as tiles of 128 or 256 tokens
      // allow, all of them even (48 steps, H = 2048, V = 100003: 92 us, with tiles of whole
      // 16 tokens 98).
      p.narrow_per_cu = narrow_per_cu(N, V);
      const int64_t slots = p.narrow_per_cu * kCus, most = N <= 64 ? 128 : 256;
      const int64_t rounds = (V + most * slots - 1) / (most * slots);
      p.tile_tokens = static_cast<int>((V + rounds * slots - 1) / (rounds * slots));
      const int64_t tiles = (V + p.tile_tokens - 1) / p.tile_tokens;
      p.pieces = tiles < slots ? tiles : slots;
    } else {
      // Tokens of a workgroup: as many as leave about a workgroup or two a CU (64 of them with
      // more than 32 steps would not fit the registers).
      p.tile_tokens = V >= 64 * 2 * kCus && N <= 32 ? 64 : V >= 24 * kCus ? 32 : 16;
      const int64_t tiles = (V + p.tile_tokens - 1) / p.tile_tokens;
      p.pieces = tiles < 4 * kCus ? tiles : 4 * kCus;
    }
  } else {
    p.row_pitch = round_up(N, kTile);
    p.x_pitch = round_up(H, kTileK);
    p.small_logits = small_tiles_pay(N, V, p.x_pitch / kTileK);
    p.pieces = 2 * tiles_of(V, p.small_logits ? kSmallTile : kTile);
  }
  VocabArgs a = {};
  a.N = N;
  p.bytes = carve_log_probs(&a, p, nullptr);
  return p;
}

VocabPlan plan_vocab_grad(int64_t N, int64_t V, int64_t H, bool grad_bf16) {
  VocabPlan p = {};
  p.row_pitch = round_up(N, kTile);
  p.x_pitch = round_up(H, kTileK);
  const int64_t all = round_up(V, kTile);
  const int64_t column = p.row_pitch * (grad_bf16 ? 2 : 4);
  const int64_t fit = (column * all <= kOnePieceBytes ? kOnePieceBytes : kPieceBytes) / column / kTile * kTile;
  const int64_t most = fit < kTile ? kTile : fit;
  const int64_t pieces = (all + most - 1) / most;
  p.g_pitch = round_up((all + pieces - 1) / pieces, kTile);
  p.pieces = pieces;
  p.small_logits = small_tiles_pay(N, p.g_pitch, p.x_pitch / kTileK);
  p.small_weight = small_tiles_pay(H, p.g_pitch, tiles_of(N, kTileK) * (grad_bf16 ? 1 : 2));
  // d_hidden's tiles, whatever the number of active steps: those of one part, or as many as
  // it is split into at most.
  VocabArgs a = {};
  a.N = N;
  a.H = H;
  a.g_pitch = p.g_pitch;
  a.pieces = pieces;
  a.grad_bf16 = grad_bf16;
  const int n = static_cast<int>(N);
  p.small_hidden = best_split(a, n, kSmallTile).cost < best_split(a, n, kTile).cost;
  const int size = p.small_hidden ? kSmallTile : kTile;
  const int64_t split_rows = most_split_tiles(size) / tiles_of(H, size) * size;
  p.split_rows = split_rows > p.row_pitch ? split_rows : p.row_pitch;
  p.bytes = carve_grad(&a, p, nullptr);
  return p;
}

void attach_vocab_log_probs(VocabArgs* a, const VocabPlan& p, void* ws) { carve_log_probs(a, p, ws); }
void attach_vocab_grad(VocabArgs* a, const VocabPlan& p, void* ws) { carve_grad(a, p, ws); }

namespace {

template <bool kGrad>
hipError_t launch_gather(const VocabArgs& a, const VocabPlan& p, hipStream_t st) {
  const dim3 grid(blocks_of(p.row_pitch, kGatherThreads / kWave)), block(kGatherThreads);
  if (a.N <= kOwnListMost) {
    hipLaunchKernelGGL((vocab_gather_kernel<kGrad, true>), grid, block, 0, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(vocab_list_kernel<kGrad>, dim3(1), dim3(kListThreads), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((vocab_gather_kernel<kGrad, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_vocab_log_probs(const VocabArgs& a, const VocabPlan& p, hipStream_t st) {
  hipError_t e;
  if (!p.few) {
    if ((e = launch_gather<false>(a, p, st)) != hipSuccess) return e;
  }
  e = p.few ? launch_vocab_few(a, st) : launch_vocab_stats(a, st);
  if (e != hipSuccess) return e;
  const dim3 few(static_cast<unsigned>(a.N)), few_block(kJoinFewThreads);
  const dim3 grid(blocks_of(a.N, kJoinRows)), block(kJoinThreads);
  if (p.few && a.entropy) hipLaunchKernelGGL(vocab_join_few_kernel<true>, few, few_block, 0, st, a);
  else if (p.few) hipLaunchKernelGGL(vocab_join_few_kernel<false>, few, few_block, 0, st, a);
  else if (a.entropy) hipLaunchKernelGGL(vocab_join_kernel<true>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(vocab_join_kernel<false>, grid, block, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_vocab_grad(const VocabArgs& a, const VocabPlan& p, hipStream_t st) {
  hipError_t e;
  if ((e = launch_gather<true>(a, p, st)) != hipSuccess) return e;
  for (int64_t v0 = 0; v0 < a.V; v0 += p.g_pitch) {
    if ((e = launch_vocab_logit_grads(a, v0, st)) != hipSuccess) return e;
    if ((e = launch_vocab_d_weight(a, v0, st)) != hipSuccess) return e;
    if ((e = launch_vocab_d_hidden(a, v0, v0 == 0, st)) != hipSuccess) return e;
    if (a.d_bias != nullptr) {
      hipLaunchKernelGGL(vocab_bias_kernel, dim3(blocks_of(p.g_pitch, kFinishThreads)), dim3(kFinishThreads), 0, st, a,
                         v0);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  const dim3 grid(blocks_of(a.N * (a.H / 4), kFinishThreads)), block(kFinishThreads);
  if (a.grad_bf16) hipLaunchKernelGGL(vocab_finish_kernel<uint16_t>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(vocab_finish_kernel<float>, grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace vtrace
