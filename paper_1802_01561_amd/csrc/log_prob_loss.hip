// V-trace losses and gradients from log-probabilities [T,B] (Sec. 4 with log pi(a_t|x_t)
// and log mu(a_t|x_t) as inputs), for lanes of different lengths and for unrolls far
// longer than an environment's: a language policy's answers.
//
// With x_t = v_t - V(x_t) the recursion is affine, x_t = delta_t + gamma_t c_t x_{t+1},
// and maps compose: (A, B) o (A', B') = (A A', A B' + B).  A workgroup takes up to 16
// consecutive lanes (64 bytes of a time row) and walks backwards over tiles of time: a
// thread has 4 consecutive steps of one lane, composes them, and a suffix scan over the
// workgroup's threads gives each the value behind its steps.
//
// Few lanes with many steps are split along time as well (chunks of whole tiles): a
// first launch forms the chunks' composites, and the second starts each chunk from the
// composite of those behind it.  The inputs are then read twice, the second time mostly
// from the Infinity Cache.
//
// Measured, us a call back to back: T = 100, B = 32 (one launch) 8.4; T = 16384, B = 128 (1.56 M
// steps of 36 bytes, 10 us at 5.5 TB/s) 32, bound by the latency of two walks of two tiles
// each (four waves a SIMD; at three, 41); T = 1000, B = 16384 (590 MB) 181, 3.3 TB/s, bound by
// 16 tiles one after the other, each with its loads, scan and stores in turn.
#include "device_common.hpp"
#include "log_prob_loss.hpp"
#include "tickets.hpp"
#include "wave_ops.hpp"

namespace vtrace {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kSteps = 4;       // consecutive steps of a thread
constexpr int kMostLanes = 16;  // of a workgroup
// Workgroups that an unroll is split up to: four a CU (16384 x 128: 33 us; 2048 of them 40).
constexpr int64_t kWantedGroups = 1024;
constexpr double kLog2e = 1.4426950408889634;

// Raw buffers: loads beyond the end give 0, stores there are dropped.
typedef __amdgpu_buffer_rsrc_t Rsrc;
constexpr int kRawBufferFlags = 0x00020000;
constexpr uint32_t kOutOfRange = 0x80000000u;

struct Map {
  double a, b;  // x -> a x + b
};
// coefficient_product with a branch, of either sign: here, where registers are short, the
// cheaper form (T = 1000, B = 8192 113 us, without a branch 118, unchecked 111).
__device__ __forceinline__ double product(double a, double b) {
  const double p = a * b;
  if (__builtin_isinf(p) && !__builtin_isinf(a) && !__builtin_isinf(b)) return __builtin_copysign(__DBL_MAX__, p);
  return p;
}
__device__ __forceinline__ Map after(Map first, Map then) {  // first o then
  return {product(first.a, then.a), fma(first.a, then.b, first.b)};
}

// Suffix composites over the threads of a lane (later threads hold later steps): of the
// threads behind this one, and of all of them.
template <int kLanes>
struct Scan {
  Map s_wave[kWaves][kLanes];

  __device__ __forceinline__ Map behind(Map mine, Map* all) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    Map upto = mine;
#pragma unroll
    for (int o = kLanes; o < kWave; o <<= 1) {
      const Map m = {__shfl_down(upto.a, o, kWave), __shfl_down(upto.b, o, kWave)};
      if (lane + o < kWave) upto = after(upto, m);
    }
    if (lane < kLanes) s_wave[wave][lane] = upto;
    Map next = {__shfl_down(upto.a, kLanes, kWave), __shfl_down(upto.b, kLanes, kWave)};
    if (lane + kLanes >= kWave) next = {1.0, 0.0};
    __syncthreads();
    Map later = {1.0, 0.0}, total = {1.0, 0.0};
#pragma unroll
    for (int w = kWaves - 1; w >= 0; --w) {
      const Map m = s_wave[w][lane % kLanes];
      if (w > wave) later = after(m, later);
      total = after(m, total);
    }
    __syncthreads();
    *all = total;
    return after(next, later);
  }
};

// The loss totals, by the last workgroup.
__device__ __forceinline__ void add_totals(const StepArgs& a, double* scratch) {
  double s0 = 0.0, s1 = 0.0, s2 = 0.0;
#pragma unroll 4
  for (unsigned i = threadIdx.x; i < gridDim.x; i += kThreads) {
    const double* p = a.partials + 3 * static_cast<size_t>(i);
    s0 += __hip_atomic_load(p + 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s1 += __hip_atomic_load(p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s2 += __hip_atomic_load(p + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  block_sum3<kThreads>(s0, s1, s2, scratch);
  if (threadIdx.x == 0) store_totals(a, s0, s1, s2);
}

template <int kLanes, bool kFinish, bool kEpsilon>
__global__ __launch_bounds__(kThreads, 4) void log_prob_kernel(LogProbArgs args) {
  constexpr int kRows = kThreads / kLanes;        // threads of a lane
  constexpr int64_t kTileSteps = kRows * kSteps;
  __shared__ Scan<kLanes> s_scan;
  __shared__ double s_red[3 * kWaves];
  const StepArgs& a = args.step;
  const int64_t groups = (a.B + kLanes - 1) / kLanes;
  const int64_t id = xcd_tile(blockIdx.x, groups * args.chunks);
  const int64_t chunk = id / groups;
  const int q = threadIdx.x / kLanes;
  const uint32_t l = threadIdx.x % kLanes;
  const int64_t b0 = (id % groups) * kLanes;
  const int64_t b = b0 + l;
  const uint32_t stride = static_cast<uint32_t>(a.B);
  const bool lane_ok = b < a.B;
  int64_t n = 0;  // steps of this lane
  double boot = 0.0;
  if (lane_ok) {
    n = a.T;
    if (args.lengths) {
      const int64_t given = args.lengths[b];
      n = given < 0 ? 0 : given < n ? given : n;
    }
    boot = static_cast<double>(a.bootstrap_value[b]);
  }
  const double lam = a.lambda, rho_bar = a.rho_bar, c_bar = a.c_bar;
  const bool weighted = a.correction == kCorrVtrace, weighted_pg = weighted || a.correction == kCorrOneStepIs;
  // variant_weights with the choices made once.
  auto weights = [&](double ratio) {
    const double rho = clip_above(ratio, rho_bar);
    return StepWeights{weighted ? rho : 1.0, lam * (weighted ? clip_above(ratio, c_bar) : 1.0), weighted_pg ? rho : 1.0};
  };
  auto step_of = [](const StepWeights& w, double diff, float g) {  // x -> delta + gamma c x
    return Map{static_cast<double>(g) * w.c_v, w.rho_v * diff};
  };
  const bool q_baseline = a.q_estimate == kQBaseline;

  double x_end = 0.0;  // x at the first step behind the tile
  if (kFinish && args.chunks > 1) {
    // The chunks behind this one, a contiguous share of them to each thread of the lane.
    const int64_t later = args.chunks - 1 - chunk;
    const int64_t from = chunk + 1 + later * q / kRows, to = chunk + 1 + later * (q + 1) / kRows;
    Map m = {1.0, 0.0};
    if (lane_ok) {
      const Map* const maps = reinterpret_cast<const Map*>(args.composites);
#pragma unroll 4
      for (int64_t k = to - 1; k >= from; --k) m = after(maps[k * a.B + b], m);
    }
    Map all;
    s_scan.behind(m, &all);
    x_end = all.b;
  }

  const int64_t tiles = (a.T + kTileSteps - 1) / kTileSteps;
  const int64_t first_tile = chunk * args.chunk_tiles;
  const int64_t last_tile = first_tile + args.chunk_tiles < tiles ? first_tile + args.chunk_tiles : tiles;
  uint32_t place[kSteps + 1];  // of this thread's steps in a tile
#pragma unroll
  for (int j = 0; j <= kSteps; ++j) place[j] = 4 * ((static_cast<uint32_t>(q * kSteps) + j) * stride + l);
  auto read = [](Rsrc p, uint32_t o) { return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(p, o, 0, 0)); };
  auto write = [](Rsrc p, uint32_t o, float value) {
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, value), p, o, 0, 0);
  };
  Map composite = {1.0, 0.0};
  double sum_pg = 0.0, sum_base = 0.0, sum_ent = 0.0;
  for (int64_t tile = last_tile - 1; tile >= first_tile; --tile) {
    // Of this thread's steps in the tile, how many are the lane's, and how many there are.
    const int64_t t0 = tile * kTileSteps + q * kSteps;
    auto steps_to = [&](int64_t end) { return static_cast<int>(end - t0 < 0 ? 0 : end - t0 > kSteps + 1 ? kSteps + 1 : end - t0); };
    const int mine_n = steps_to(n);
    // The tile's place in the arrays (uniform).  A step that is not the lane's is read out of
    // range, as zeros: log-ratio, reward, discount and value 0 make every quantity below 0.
    const int64_t corner = tile * kTileSteps * a.B + b0;
    const int64_t left = 4 * (a.T * a.B - corner);
    const int records = left >> 31 ? 0x7fffffff : static_cast<int>(left);
    auto array = [&](const void* p) {
      return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(static_cast<const float*>(p) + corner), 0, p ? records : 0,
                                               kRawBufferFlags);
    };
    uint32_t off[kSteps + 1];
#pragma unroll
    for (int j = 0; j <= kSteps; ++j) off[j] = j < mine_n ? place[j] : kOutOfRange;
    float lp[kSteps], lm[kSteps], r[kSteps], gm[kSteps], v[kSteps + 1], entropy[kSteps];
    {
      const Rsrc p_lp = array(args.target), p_lm = array(args.behaviour), p_r = array(a.rewards), p_g = array(a.discounts),
                 p_v = array(a.values);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        lp[j] = read(p_lp, off[j]);
        lm[j] = read(p_lm, off[j]);
        r[j] = read(p_r, off[j]);
        gm[j] = read(p_g, off[j]);
        v[j] = read(p_v, off[j]);
      }
      v[kSteps] = read(p_v, off[kSteps]);
    }
    if constexpr (kFinish) {
      const Rsrc p_h = array(args.entropy);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) entropy[j] = read(p_h, off[j]);
    }
    if (a.reward_transform != 0) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) r[j] = transform_reward(r[j], a.reward_transform);
    }
    // Of each step: the ratio, and the temporal difference before its weight.
    double ratio[kSteps], diff[kSteps];
    Map mine = {1.0, 0.0};
#pragma unroll
    for (int j = kSteps - 1; j >= 0; --j) {
      ratio[j] = exp2_f64((static_cast<double>(lp[j]) - static_cast<double>(lm[j])) * kLog2e);
      const double v_next = j + 1 == mine_n ? boot : v[j + 1];
      diff[j] = fma(static_cast<double>(gm[j]), v_next, static_cast<double>(r[j]) - static_cast<double>(v[j]));
      mine = after(step_of(weights(ratio[j]), diff[j], gm[j]), mine);
    }
    Map all;
    const Map behind = s_scan.behind(mine, &all);
    if constexpr (!kFinish) {
      composite = after(all, composite);
    } else {
      const int here_n = lane_ok ? steps_to(a.T) : 0;
      double x = fma(behind.a, x_end, behind.b);
      float d_lps[kSteps], d_vs[kSteps], advs[kSteps];
#pragma unroll
      for (int j = kSteps - 1; j >= 0; --j) {
        const StepWeights w = weights(ratio[j]);
        const double g = gm[j];
        const double adv = w.rho_pg * (q_baseline ? diff[j] : fma(g, x, diff[j]));
        x = fma(g * w.c_v, x, w.rho_v * diff[j]);
        double d_lp = adv, log_p = lp[j];
        if constexpr (kEpsilon) {
          const double p = exp2_f64(log_p * kLog2e), eps = a.epsilon;
          d_lp *= p / (p + eps);
          log_p = log(p + eps);
        }
        sum_pg = fma(-adv, log_p, sum_pg);
        sum_base = fma(0.5 * x, x, sum_base);
        sum_ent -= static_cast<double>(entropy[j]);
        d_lps[j] = static_cast<float>(-d_lp);
        d_vs[j] = static_cast<float>(-a.baseline_cost * x);
        advs[j] = static_cast<float>(adv);
        if (a.vs) v[j] = static_cast<float>(v[j] + x);
      }
      // Steps behind a lane's last get zeros.
#pragma unroll
      for (int j = 0; j <= kSteps; ++j) off[j] = j < here_n ? place[j] : kOutOfRange;
      const Rsrc o_lp = array(args.d_log_probs), o_v = array(a.d_values);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        write(o_lp, off[j], d_lps[j]);
        write(o_v, off[j], d_vs[j]);
      }
      if (args.d_entropy) {
        const Rsrc o = array(args.d_entropy);
#pragma unroll
        for (int j = 0; j < kSteps; ++j) write(o, off[j], j < mine_n ? -a.entropy_cost : 0.0f);
      }
      if (a.vs) {
        const Rsrc o = array(a.vs);
#pragma unroll
        for (int j = 0; j < kSteps; ++j) write(o, off[j], v[j]);
      }
      if (a.pg_adv) {
        const Rsrc o = array(a.pg_adv);
#pragma unroll
        for (int j = 0; j < kSteps; ++j) write(o, off[j], advs[j]);
      }
      x_end = fma(all.a, x_end, all.b);
    }
  }
  if constexpr (!kFinish) {
    if (q == 0 && lane_ok) {
      double* p = args.composites + 2 * (chunk * a.B + b);
      p[0] = composite.a;
      p[1] = composite.b;
    }
  } else {
    block_sum3<kThreads>(sum_pg, sum_base, sum_ent, s_red);
    if (threadIdx.x == 0) publish_losses(a, sum_pg, a.baseline_cost * sum_base, a.entropy_cost * sum_ent);
    if (gridDim.x > 1 && last_workgroup(a.ticket, args.counters)) add_totals(a, s_red);
  }
}

// Lanes of a workgroup: as many as there are, up to 16; fewer (down to 4) where the unroll
// then fits one tile, so that one launch does.
int lanes_of(int64_t T, int64_t B) {
  int n = 1;
  while (n < kMostLanes && n < B) n *= 2;
  if (B < kMostLanes * kWantedGroups)
    for (int m = n; m >= 4; m /= 2)
      if (T <= kThreads / m * kSteps) return m;
  return n;
}

// Chunks: as many as give kWantedGroups workgroups, none shorter than a tile.
void split_time(int64_t T, int64_t B, int64_t* chunks, int64_t* chunk_tiles, int64_t* groups) {
  const int64_t lanes = lanes_of(T, B), steps = kThreads / lanes * kSteps;
  const int64_t tiles = (T + steps - 1) / steps;
  *groups = (B + lanes - 1) / lanes;
  int64_t want = (kWantedGroups + *groups - 1) / *groups;
  if (want > tiles) want = tiles;
  *chunk_tiles = (tiles + want - 1) / want;
  *chunks = (tiles + *chunk_tiles - 1) / *chunk_tiles;
}

size_t partial_bytes(int64_t groups) { return (static_cast<size_t>(groups) * 3 * sizeof(double) + 255) / 256 * 256; }

template <int kLanes>
hipError_t launch(const LogProbArgs& a, hipStream_t st) {
  const int64_t groups = (a.step.B + kLanes - 1) / kLanes;
  const dim3 grid(static_cast<unsigned>(groups * a.chunks)), block(kThreads);
  if (a.chunks > 1) {
    hipLaunchKernelGGL((log_prob_kernel<kLanes, false, false>), grid, block, 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.step.correction == kCorrEpsilon)
    hipLaunchKernelGGL((log_prob_kernel<kLanes, true, true>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((log_prob_kernel<kLanes, true, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t log_prob_workspace_bytes(int64_t T, int64_t B) {
  int64_t chunks, chunk_tiles, groups;
  split_time(T, B, &chunks, &chunk_tiles, &groups);
  const size_t composites = chunks > 1 ? static_cast<size_t>(chunks * B) * 2 * sizeof(double) : 0;
  return kWsDataOffset + partial_bytes(groups * chunks) + composites;
}

void attach_log_prob_workspace(LogProbArgs* a, void* ws) {
  int64_t groups;
  split_time(a->step.T, a->step.B, &a->chunks, &a->chunk_tiles, &groups);
  char* const base = static_cast<char*>(ws);
  a->step.ticket = reinterpret_cast<unsigned int*>(base + kWsTicketOffset);
  a->counters = reinterpret_cast<unsigned int*>(base + kWsHeaderBytes);
  char* const sums = base + kWsDataOffset;
  a->step.partials = reinterpret_cast<double*>(sums);
  a->composites = reinterpret_cast<double*>(sums + partial_bytes(groups * a->chunks));
}

hipError_t launch_log_prob_loss(const LogProbArgs& a, hipStream_t st) {
  switch (lanes_of(a.step.T, a.step.B)) {
    case 1: return launch<1>(a, st);
    case 2: return launch<2>(a, st);
    case 4: return launch<4>(a, st);
    case 8: return launch<8>(a, st);
    default: return launch<kMostLanes>(a, st);
  }
}

}  // namespace vtrace
