// V-trace losses and gradients from log-probabilities [T,B] (Sec. 4 with log pi(a_t|x_t)
// and log mu(a_t|x_t) as inputs), for lanes of different lengths and for unrolls far
// longer than an environment's: a language policy's answers.
//
// With x_t = v_t - V(x_t) the recursion is affine, x_t = delta_t + gamma_t c_t x_{t+1},
// and maps compose: (A, B) o (A', B') = (A A', A B' + B).  A workgroup takes up to 16
// consecutive lanes (64 bytes of a time row) and walks backwards over tiles of time: a
// thread has 8 consecutive steps of one lane, composes them, and a suffix scan over the
// workgroup's threads gives each the value behind its steps.
//
// Few lanes with many steps are split along time as well (chunks of whole tiles): a
// first launch forms the chunks' composites, and the second starts each chunk from the
// composite of those behind it.  The inputs are then read twice, the second time mostly
// from the Infinity Cache.
#include "device_common.hpp"
#include "log_prob_loss.hpp"
#include "wave_ops.hpp"

namespace vtrace {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kSteps = 8;      // consecutive steps of a thread
constexpr int kMostLanes = 16;  // of a workgroup
constexpr int64_t kWantedGroups = 1024;

struct Map {
  double a, b;  // x -> a x + b
};
__device__ __forceinline__ Map after(Map first, Map then) {  // first o then
  return {first.a * then.a, fma(first.a, then.b, first.b)};
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

template <int kLanes, bool kFinish>
__global__ __launch_bounds__(kThreads) void log_prob_kernel(LogProbArgs args) {
  constexpr int kRows = kThreads / kLanes;        // threads of a lane
  constexpr int64_t kTileSteps = kRows * kSteps;
  __shared__ Scan<kLanes> s_scan;
  __shared__ double s_red[3 * kWaves];
  const StepArgs& a = args.step;
  const int64_t groups = (a.B + kLanes - 1) / kLanes;
  const int64_t id = xcd_tile(blockIdx.x, groups * args.chunks);
  const int64_t chunk = id / groups;
  const int q = threadIdx.x / kLanes;
  const int64_t b = (id % groups) * kLanes + threadIdx.x % kLanes;
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

  double x_end = 0.0;  // x at the first step behind the tile
  if (kFinish && args.chunks > 1) {
    // The chunks behind this one, a contiguous share of them to each thread of the lane.
    const int64_t later = args.chunks - 1 - chunk;
    const int64_t from = chunk + 1 + later * q / kRows, to = chunk + 1 + later * (q + 1) / kRows;
    Map m = {1.0, 0.0};
    if (lane_ok) {
      for (int64_t k = to - 1; k >= from; --k) {
        const double* p = args.composites + 2 * (k * a.B + b);
        m = after({p[0], p[1]}, m);
      }
    }
    Map all;
    s_scan.behind(m, &all);
    x_end = all.b;
  }

  const int64_t tiles = (a.T + kTileSteps - 1) / kTileSteps;
  const int64_t first_tile = chunk * args.chunk_tiles;
  const int64_t last_tile = first_tile + args.chunk_tiles < tiles ? first_tile + args.chunk_tiles : tiles;
  Map composite = {1.0, 0.0};
  double sum_pg = 0.0, sum_base = 0.0, sum_ent = 0.0;
  for (int64_t tile = last_tile - 1; tile >= first_tile; --tile) {
    const int64_t t0 = tile * kTileSteps + static_cast<int64_t>(q) * kSteps;
    const int64_t at = t0 * a.B + b;
    float lp[kSteps], lm[kSteps], r[kSteps], gm[kSteps], v[kSteps + 1];
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const bool in = t0 + j < n;
      const int64_t i = at + j * a.B;
      lp[j] = in ? args.target[i] : 0.0f;
      lm[j] = in ? args.behaviour[i] : 0.0f;
      r[j] = in ? a.rewards[i] : 0.0f;
      gm[j] = in ? a.discounts[i] : 0.0f;
      v[j] = in ? a.values[i] : 0.0f;
    }
    v[kSteps] = t0 + kSteps < n ? a.values[at + kSteps * a.B] : 0.0f;
    double delta[kSteps], decay[kSteps];
    StepWeights w[kSteps];
    Map mine = {1.0, 0.0};
#pragma unroll
    for (int j = kSteps - 1; j >= 0; --j) {
      const bool in = t0 + j < n;
      const double ratio = exp2_f64((static_cast<double>(lp[j]) - static_cast<double>(lm[j])) * 1.4426950408889634);
      w[j] = variant_weights(a.correction, clip_above(ratio, rho_bar), lam * clip_above(ratio, c_bar), lam, true);
      const double v_next = t0 + j + 1 == n ? boot : static_cast<double>(v[j + 1]);
      const double reward = transform_reward(r[j], a.reward_transform), g = gm[j], V = v[j];
      delta[j] = in ? w[j].rho_v * (reward + g * v_next - V) : 0.0;
      decay[j] = in ? g * w[j].c_v : 0.0;
      mine = after({decay[j], delta[j]}, mine);
    }
    Map all;
    const Map behind = s_scan.behind(mine, &all);
    if constexpr (!kFinish) {
      composite = after(all, composite);
    } else {
      double x = fma(behind.a, x_end, behind.b);
#pragma unroll
      for (int j = kSteps - 1; j >= 0; --j) {
        const int64_t t = t0 + j;
        const bool in = t < n;
        const double v_next = t + 1 == n ? boot : static_cast<double>(v[j + 1]);
        const double V = v[j], g = gm[j], reward = transform_reward(r[j], a.reward_transform);
        const double q_next = a.q_estimate == kQBaseline ? v_next : v_next + x;
        const double adv = in ? w[j].rho_pg * (reward + g * q_next - V) : 0.0;
        x = fma(decay[j], x, delta[j]);
        if (t >= a.T || !lane_ok) continue;
        const int64_t i = at + j * a.B;
        double d_lp = -adv, log_p = lp[j];
        if (a.correction == kCorrEpsilon) {
          const double p = exp2_f64(log_p * 1.4426950408889634), eps = a.epsilon;
          d_lp *= p / (p + eps);
          log_p = log(p + eps);
        }
        args.d_log_probs[i] = in ? static_cast<float>(d_lp) : 0.0f;
        a.d_values[i] = in ? static_cast<float>(-a.baseline_cost * x) : 0.0f;
        if (args.d_entropy) args.d_entropy[i] = in ? -a.entropy_cost : 0.0f;
        if (a.vs) a.vs[i] = in ? static_cast<float>(V + x) : 0.0f;
        if (a.pg_adv) a.pg_adv[i] = static_cast<float>(adv);
        if (in) {
          sum_pg -= adv * log_p;
          sum_base += 0.5 * x * x;
          if (args.entropy) sum_ent -= static_cast<double>(args.entropy[i]);
        }
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
    finish_losses<kThreads>(a, sum_pg, a.baseline_cost * sum_base, a.entropy_cost * sum_ent, s_red);
  }
}

int lanes_of(int64_t B) {
  int n = 1;
  while (n < kMostLanes && n < B) n *= 2;
  return n;
}

// Chunks: as many as give kWantedGroups workgroups, none shorter than a tile.
void split_time(int64_t T, int64_t B, int64_t* chunks, int64_t* chunk_tiles, int64_t* groups) {
  const int64_t lanes = lanes_of(B), steps = kThreads / lanes * kSteps;
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
    hipLaunchKernelGGL((log_prob_kernel<kLanes, false>), grid, block, 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((log_prob_kernel<kLanes, true>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t log_prob_workspace_bytes(int64_t T, int64_t B) {
  int64_t chunks, chunk_tiles, groups;
  split_time(T, B, &chunks, &chunk_tiles, &groups);
  const size_t composites = chunks > 1 ? static_cast<size_t>(chunks * B) * 2 * sizeof(double) : 0;
  return kWsHeaderBytes + partial_bytes(groups * chunks) + composites;
}

void attach_log_prob_workspace(LogProbArgs* a, void* ws) {
  int64_t groups;
  split_time(a->step.T, a->step.B, &a->chunks, &a->chunk_tiles, &groups);
  char* const base = static_cast<char*>(ws);
  a->step.ticket = reinterpret_cast<unsigned int*>(base + kWsTicketOffset);
  a->step.partials = reinterpret_cast<double*>(base + kWsHeaderBytes);
  a->composites = reinterpret_cast<double*>(base + kWsHeaderBytes + partial_bytes(groups * a->chunks));
}

hipError_t launch_log_prob_loss(const LogProbArgs& a, hipStream_t st) {
  switch (lanes_of(a.step.B)) {
    case 1: return launch<1>(a, st);
    case 2: return launch<2>(a, st);
    case 4: return launch<4>(a, st);
    case 8: return launch<8>(a, st);
    default: return launch<kMostLanes>(a, st);
  }
}

}  // namespace vtrace
