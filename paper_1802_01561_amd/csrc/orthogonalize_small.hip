// The products of Newton-Schulz steps for matrices too small or too few to fill the chip with
// tiles of 128: a workgroup of four waves for each 64 x 64 or 32 x 32 of the result.
//
// Everything here is latency, so that what counts are bytes in flight: operands are copied
// straight to LDS, kStages steps of 64 k ahead.  (Fragments read from memory into registers, a
// 16-byte piece of 16 rows each, make 64 requests where these make 8: 1024 x 1024 in 16 us a
// product.)  All three products have both operands' k innermost, which for the last one, B X,
// takes X^T, kept beside X.  A launch takes 5 to 8 us for a 256 x 1024 float32 matrix (32 x 32, 4 to 16
// steps of k in three products each), 10 to 13 for 1000 x 1000 bfloat16 (64 x 64, 16 steps), 2 to
// 3 of them before the first step: what bounds a step is the path into one CU's LDS, 65 KB a us.
#include "orthogonalize_few.hpp"
#include "orthogonalize_impl.hpp"

namespace vtrace {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// The compiler's own instruction, whose latency it knows: here accumulators move at the loop's end.
__device__ __forceinline__ void multiply_add(f32x4& c, bf16x8 a, bf16x8 b) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

constexpr int kSmallWaves = 4, kSmallThreads = kSmallWaves * kWave;
// Steps of k in LDS, of two operands in `parts` parts.
__host__ __device__ constexpr int small_stages(int side, int parts) { return side == 64 ? 6 - parts : parts == 1 ? 8 : 5; }

// kOf: a symmetric matrix of X, one or two; kUpdate: X, or of the last step the result.  Wave (wm, wn) has a
// quarter of the tile; a lane of the MFMA layout holds columns j + 16 m + 4 g + 0..3 of row
// i + 16 n + s of that.
constexpr int kUpdate = 3;
// kFew: and the results of the matrices of few rows, by the first workgroups.
template <int kOf, typename Out, bool kLast, int kSide, bool kFew>
__global__ __launch_bounds__(kSmallThreads) void ortho_small_kernel(Table t, int turn, std::conditional_t<kOf == kUpdate, Update, Product> f,
                                                                    std::conditional_t<kFew, FewSteps, int> few) {
  constexpr bool kPair = sizeof(Out) == 4;
  constexpr int kKind = kOf == kOfX ? 0 : kOf == kUpdate ? 2 : 1;
  constexpr int kParts = kPair ? 2 : 1, kN = kSide / 32;
  constexpr int kStages = small_stages(kSide, kParts), kBytes = kSide * kTileK * 2, kStage = 2 * kParts * kBytes;
  __shared__ __align__(1024) char lds[kStages * kStage];
  const int workgroup = kFew ? static_cast<int>(blockIdx.x) - t.few_blocks : blockIdx.x;
  if constexpr (kFew) {
    static_assert(kFewLds <= kStages * kStage && kFewThreads == kSmallThreads);
    if (workgroup < 0) {
      few_apply<Out>(t, few, blockIdx.x, lds);
      return;
    }
  }
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int s = lane % 16, g = lane / 16;
  const Entry& e = t.at[entry_of(t, workgroup, [](const Entry& e) { return e.first_tile[kKind]; })];
  const int id = workgroup - e.first_tile[kKind];
  TileAt at;
  if constexpr (kKind < 2) {
    at = triangle_at(id);
  } else {
    const int rows = e.pr / kSide;
    at = {id % rows, id / rows};
  }
  const Pieces p = pieces_of<kPair>(e, turn);
  const TransposedPieces pt = transposed_of<kPair>(e, turn);
  const int64_t pitch = kKind == 0 ? e.pc : e.pr;
  const int steps = static_cast<int>(pitch / kTileK);

  // A descriptor for each operand, at its tile's rows, and where in it the steps begin; rows
  // behind the last one arrive as zeros.
  typedef Loader<kSide, kSmallWaves> Places;
  Places places[2];
  Rsrc operand[kParts][2], nothing[kParts][2];
#pragma unroll
  for (int o = 0; o < 2; ++o) {
    const int64_t first = static_cast<int64_t>(o == 0 ? at.wide : at.deep) * kSide;
    const int64_t rows = (kKind == 2 && o == 1 ? e.c : e.r) - first;
    places[o].along(pitch, static_cast<int>(rows < kSide ? rows : kSide), wave, lane);
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const uint16_t* array;
      if constexpr (kOf == kOfX) array = p.from[k];
      else if constexpr (kOf == kUpdate) array = o == 0 ? symmetric_of<kPair>(e, p, f.by, k) : pt.from[k];
      else array = symmetric_of<kPair>(e, p, o == 0 ? f.m : f.n, k);
      operand[k][o] = make_rsrc(array + first * pitch, 0x7fffffff);
      nothing[k][o] = make_rsrc(array, 0);
    }
  }
  auto copy = [&](int stage, int step) {
    const bool more = step < steps;
#pragma unroll
    for (int k = 0; k < kParts; ++k)
#pragma unroll
      for (int o = 0; o < 2; ++o) {
        char* const to = lds + stage * kStage + (2 * k + o) * kBytes + wave * 1024;
#pragma unroll
        for (int i = 0; i < Places::kCopies; ++i)
          copy_to_lds(more ? operand[k][o] : nothing[k][o], to + i * Places::kCopyBytes, places[o].off[i],
                      more ? step * (kTileK * 2) : 0);
      }
  };
  constexpr int kCopies = 2 * kParts * Places::kCopies;
  const int wm = (wave % 2) * (kSide / 2), wn = (wave / 2) * (kSide / 2);
  Reader<false, false, kN, kSide> ri, rj;
  ri.start(wn, s, g);
  rj.start(wm, s, g);
  f32x4 acc[kN][kN] = {};  // [m][n]
  f32x4 cross[kN][kN] = {}, total[kN][kN] = {};  // of the low parts; of all
  const int i0 = at.wide * kSide + wn + s, j0 = at.deep * kSide + wm + 4 * g;
  // What the results take beside the products is under way before them.
  constexpr int kMatrices = kOf == kOfTwo ? 2 : 1;
  f32x4 x[kN][kN];
  v2u o[kMatrices][2][kN][kN];  // of M and N, or of X: high and low parts
  float of_row[kN];
  f32x4 of_column[kN];
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    const int i = i0 + 16 * n, i_in = i < e.r ? i : e.r - 1;  // rows behind the last one: nobody stores them
    if constexpr (kOf == kOfOne || kOf == kOfTwo) of_row[n] = diagonal_of(e, p, f.m)[i_in];
    if constexpr (kOf == kUpdate) of_row[n] = diagonal_of(e, p, f.by)[i_in];
#pragma unroll
    for (int m = 0; m < kN; ++m) {
      const int j = j0 + 16 * m;
      if constexpr (kOf == kOfOne || kOf == kOfTwo) {
#pragma unroll
        for (int w = 0; w < kMatrices; ++w)
#pragma unroll
          for (int k = 0; k < kParts; ++k)
            o[w][k][m][n] = *reinterpret_cast<const v2u*>(symmetric_of<kPair>(e, p, w == 0 ? f.m : f.n, k) + static_cast<int64_t>(i_in) * e.pr + j);
      }
      if constexpr (kOf == kUpdate) {
        const int64_t from = static_cast<int64_t>(i_in) * e.pc + j;
        if constexpr (kPair) {
          x[m][n] = *reinterpret_cast<const f32x4*>(p.x + from);
        } else {
          o[0][0][m][n] = *reinterpret_cast<const v2u*>(p.from[0] + from);
          o[0][1][m][n] = *reinterpret_cast<const v2u*>(p.low + from);
        }
      }
    }
  }
  if constexpr (kOf == kOfOne || kOf == kOfTwo) {
#pragma unroll
    for (int m = 0; m < kN; ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j = j0 + 16 * m + q;
        of_column[m][q] = diagonal_of(e, p, f.n)[j < e.r ? j : e.r - 1];
      }
  }
#pragma unroll
  for (int k = 0; k + 1 < kStages; ++k) copy(k, k);
  // A step's fragments are read while the one before it is multiplied: from barrier to barrier there
  // is the longer of the two, not both (one after the other 0.3 us a step).
  struct Fragments {
    bf16x8 i[2][kParts][kN], j[2][kParts][kN];
  };
  int stage = 0, k = 0;
  auto read = [&](Fragments& f) {
    stage_barrier<(kStages - 2) * kCopies>();
    copy(stage == 0 ? kStages - 1 : stage - 1, k + kStages - 1);
    const char* const from = lds + stage * kStage;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int n = 0; n < kN; ++n) {
          f.i[kk][part][n] = ri.read(from + 2 * part * kBytes, n, kk);
          f.j[kk][part][n] = rj.read(from + (2 * part + 1) * kBytes, n, kk);
        }
    stage = stage + 1 == kStages ? 0 : stage + 1;
    ++k;
    __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply = [&](const Fragments& f) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int m = 0; m < kN; ++m)
#pragma unroll
        for (int n = 0; n < kN; ++n) {
          if constexpr (kPair) {
            multiply_add(cross[m][n], f.j[kk][1][m], f.i[kk][0][n]);
            multiply_add(cross[m][n], f.j[kk][0][m], f.i[kk][1][n]);
          }
          multiply_add(acc[m][n], f.j[kk][0][m], f.i[kk][0][n]);
        }
  };
  // Float32 results: sums over 256 k apiece, added up.  The rounding errors of one long sum would
  // be the most of a result's (256 x 2592: 1.6e-6 off, so 9e-7).
  auto add_up = [&](int left) {
    if (!kPair || (steps - left) % 4 != 0) return;
#pragma unroll
    for (int m = 0; m < kN; ++m)
#pragma unroll
      for (int n = 0; n < kN; ++n) {
        total[m][n] += acc[m][n];
        acc[m][n] = f32x4{};
      }
  };
  Fragments even, odd;
  read(even);
  for (int left = steps;;) {
    if (left > 1) read(odd);
    multiply(even);
    if (--left == 0) break;
    add_up(left);
    if (left > 1) read(even);
    multiply(odd);
    if (--left == 0) break;
    add_up(left);
  }
#pragma unroll
  for (int m = 0; m < kN; ++m)
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      if constexpr (kPair) total[m][n] += cross[m][n];
      total[m][n] += acc[m][n];
    }

  // The tile by way of LDS, so that rows and columns of it are stored in whole pieces.
  stage_barrier();
  float(*const s_y)[kSide + 1] = reinterpret_cast<float(*)[kSide + 1]>(lds);
#pragma unroll
  for (int n = 0; n < kN; ++n)
#pragma unroll
    for (int m = 0; m < kN; ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int i = i0 + 16 * n, j = j0 + 16 * m + q;
        const bool in = i < e.r && j < (kKind == 2 ? e.c : e.r);
        const float sum = total[m][n][q];
        float y;
        if constexpr (kOf == kOfX) {
          y = sum * (1.0f / (kScaleX * kScaleX));
          if (in && i == j) diagonal_of(e, p, f.out)[i] = y;
        } else if constexpr (kOf == kUpdate) {
          float before;
          if constexpr (kPair) before = x[m][n][q];
          else before = whole_of(o[0][0][m][n], o[0][1][m][n], q) * (1.0f / kScaleX);
          y = fmaf(f.of_x + of_row[n], before, sum * (1.0f / (kScaleA * kScaleX)));
        } else {
          const float oo = sum * (1.0f / (kScaleA * kScaleA)), di = of_row[n];
          float off[kMatrices];
#pragma unroll
          for (int w = 0; w < kMatrices; ++w) {
            off[w] = high_of(o[w][0][m][n][q / 2], q % 2);
            if constexpr (kPair) off[w] += high_of(o[w][1][m][n][q / 2], q % 2);
            off[w] *= 1.0f / kScaleA;
          }
          y = product_off<kOf>(f, off[0], off[kMatrices - 1], di, of_column[m][q], oo);
          if (in && i == j) diagonal_of(e, p, f.out)[i] = product_diagonal<kOf>(f, di, of_column[m][q], oo);
        }
        s_y[wn + s + 16 * n][wm + 4 * g + 16 * m + q] = in && (kKind == 2 || i != j) ? y : 0.0f;
      }
  __syncthreads();

  constexpr int kQuads = kSide / 4;
  const int r0 = at.wide * kSide, c0 = at.deep * kSide;
  // Four elements of an operand, and what it leaves of them where that is wanted.
  auto store_operand = [&](uint16_t* high_out, uint16_t* low_out, int64_t to, float (&y)[4], float scale) {
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] *= scale;
    const v2u high = high4(y);
    *reinterpret_cast<v2u*>(high_out + to) = high;
    if (low_out != nullptr) *reinterpret_cast<v2u*>(low_out + to) = kPair ? low4(y, high) : left4(y, high);
  };
#pragma unroll
  for (int w = 0; w < kSide * kQuads / kSmallThreads; ++w) {
    const int id = w * kSmallThreads + threadIdx.x, y0 = id / kQuads, x0 = id % kQuads * 4;
    // Along the tile's rows.
    if (r0 + y0 < e.r && !(kLast && e.transposed)) {
      const int i = r0 + y0, j = c0 + x0;
      float y[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) y[q] = s_y[y0][x0 + q];
      if constexpr (kLast) {
        Out* const out = static_cast<Out*>(e.out);
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] *= e.scale;
        store_result(out + static_cast<int64_t>(i) * e.c + j, y, e.c - j,
                     e.c % 4 == 0 && reinterpret_cast<uintptr_t>(out) % (4 * sizeof(Out)) == 0);
      } else if constexpr (kOf == kUpdate) {
        const int64_t to = static_cast<int64_t>(i) * e.pc + j;
        if constexpr (kPair) *reinterpret_cast<f32x4*>(p.x + to) = f32x4{y[0], y[1], y[2], y[3]};
        store_operand(p.to[0], kPair ? p.to[1] : p.low, to, y, kScaleX);
      } else {
        store_operand(symmetric_of<kPair>(e, p, f.out, 0), kPair ? symmetric_of<kPair>(e, p, f.out, 1) : nullptr,
                      static_cast<int64_t>(i) * e.pr + j, y, kScaleA);
      }
    }
    // And along its columns: the other half of a symmetric result, or X^T.
    if ((kKind < 2 && at.wide == at.deep) || c0 + y0 >= (kKind == 2 ? e.c : e.r)) continue;
    const int j = c0 + y0, i = r0 + x0;
    float y[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] = s_y[x0 + q][y0];
    if constexpr (kLast) {
      if (!e.transposed) continue;
      Out* const out = static_cast<Out*>(e.out);
#pragma unroll
      for (int q = 0; q < 4; ++q) y[q] *= e.scale;
      store_result(out + static_cast<int64_t>(j) * e.r + i, y, e.r - i,
                   e.r % 4 == 0 && reinterpret_cast<uintptr_t>(out) % (4 * sizeof(Out)) == 0);
    } else if constexpr (kOf == kUpdate) {
      store_operand(pt.to[0], kPair ? pt.to[1] : nullptr, static_cast<int64_t>(j) * e.pr + i, y, kScaleX);
    } else {
      store_operand(symmetric_of<kPair>(e, p, f.out, 0), kPair ? symmetric_of<kPair>(e, p, f.out, 1) : nullptr,
                    static_cast<int64_t>(j) * e.pr + i, y, kScaleA);
    }
  }
}

template <int kOf, typename Out, bool kLast, typename F>
hipError_t launch_kind(const Table& t, int turn, const F& f, hipStream_t st) {
  constexpr int kKind = kOf == kOfX ? 0 : kOf == kUpdate ? 2 : 1;
  const dim3 grid(t.total_tiles[kKind]), block(kSmallThreads);
  if (t.size[kKind] == 32) hipLaunchKernelGGL((ortho_small_kernel<kOf, Out, kLast, 32, false>), grid, block, 0, st, t, turn, f, 0);
  else hipLaunchKernelGGL((ortho_small_kernel<kOf, Out, kLast, 64, false>), grid, block, 0, st, t, turn, f, 0);
  return hipGetLastError();
}

template <typename Out>
hipError_t launch_symmetric(const Table& t, int of, int turn, const Product& p, const FewSteps* few, hipStream_t st) {
  if (of == kOfX && few != nullptr) {
    const dim3 grid(t.total_tiles[0] + t.few_blocks), block(kSmallThreads);
    if (t.size[0] == 32) hipLaunchKernelGGL((ortho_small_kernel<kOfX, Out, false, 32, true>), grid, block, 0, st, t, turn, p, *few);
    else hipLaunchKernelGGL((ortho_small_kernel<kOfX, Out, false, 64, true>), grid, block, 0, st, t, turn, p, *few);
    return hipGetLastError();
  }
  if (of == kOfX) return launch_kind<kOfX, Out, false>(t, turn, p, st);
  return of == kOfOne ? launch_kind<kOfOne, Out, false>(t, turn, p, st) : launch_kind<kOfTwo, Out, false>(t, turn, p, st);
}

}  // namespace

hipError_t launch_ortho_small_symmetric(const Table& t, int of, bool pair, int turn, const Product& p, const FewSteps* few, hipStream_t st) {
  return pair ? launch_symmetric<float>(t, of, turn, p, few, st) : launch_symmetric<uint16_t>(t, of, turn, p, few, st);
}

hipError_t launch_ortho_small_update(const Table& t, bool pair, int turn, const Update& u, hipStream_t st) {
  if (pair) return u.last ? launch_kind<kUpdate, float, true>(t, turn, u, st) : launch_kind<kUpdate, float, false>(t, turn, u, st);
  return u.last ? launch_kind<kUpdate, uint16_t, true>(t, turn, u, st) : launch_kind<kUpdate, uint16_t, false>(t, turn, u, st);
}

}  // namespace vtrace
