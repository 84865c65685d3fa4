// Newton-Schulz steps of matrices of few rows.
//
// All steps are taken in the small matrices alone, in float64: from A = X X^T, with P = a I + b A + c A A,
// A' = P A P and X' = P X, so that the result is Q X with Q the product of all P.  Two launches that
// other matrices have anyway, that of |G| and that of X or of their first A, and each reads G once.
// With float16 operands 2 x 2 and 4 x 4 bfloat16 matrices were up to 5.1e-3 off (few rows do not
// average rounding errors out), and took as many launches as large ones.
#pragma once

#include "orthogonalize_impl.hpp"

namespace vtrace {
namespace {

constexpr int kFewRows = 32, kFewThreads = 256;
constexpr int kFewTile = 64;                             // columns at a time
constexpr int64_t kFewMostChunks = 32;                   // of A's partial sums
constexpr int64_t kFewMostBlocks = 512;                  // workgroups that form results, where more columns each avoid it

__host__ __device__ inline int64_t few_chunk(int64_t c) {
  return round_up((c + kFewMostChunks - 1) / kFewMostChunks, kFewTile);
}
__host__ __device__ inline int64_t few_chunks(int64_t c) { return (c + few_chunk(c) - 1) / few_chunk(c); }

typedef float FewTile[kFewRows][kFewTile + 1];

// Columns j0 .. j0 + 63 of G, as many as there are: a thread's elements in the order in which they lie
// in memory.  k / r is (k (2^16 / r + 1)) >> 16: k < 2^11 and r <= 2^5 leave less than 1 / r over.
struct FewPlace {
  int row, column;
  int64_t at;  // in the matrix; -1 where there is none
};
__device__ __forceinline__ FewPlace few_place(const Entry& g, int j0, int n) {
  const int columns = g.c - j0 < kFewTile ? g.c - j0 : kFewTile;
  const int k = threadIdx.x + n * kFewThreads;
  if (g.transposed) {
    const int column = (k * (65536 / g.r + 1)) >> 16;
    return {k - column * g.r, column, k < columns * g.r ? static_cast<int64_t>(j0) * g.r + k : -1};
  }
  const int row = k / kFewTile, column = k % kFewTile;
  return {row, column, row < g.r && column < columns ? static_cast<int64_t>(row) * g.c + j0 + column : -1};
}
constexpr int kFewEach = kFewRows * kFewTile / kFewThreads;
template <typename In>
struct FewFetch {
  In x[kFewEach];
  // Element 0 for those that are not there.
  __device__ __forceinline__ void fetch(const Entry& g, int64_t j0) {
#pragma unroll
    for (int n = 0; n < kFewEach; ++n) {
      const FewPlace p = few_place(g, static_cast<int>(j0), n);
      x[n] = static_cast<const In*>(g.in)[p.at < 0 ? 0 : p.at];
    }
  }
  // Zeros around what is there.
  __device__ __forceinline__ void put(const Entry& g, int64_t j0, FewTile& tile) const {
#pragma unroll
    for (int n = 0; n < kFewEach; ++n) {
      const int k = threadIdx.x + n * kFewThreads;
      tile[k / kFewTile][k % kFewTile] = 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kFewEach; ++n) {
      const FewPlace p = few_place(g, static_cast<int>(j0), n);
      if (p.at >= 0) tile[p.row][p.column] = logit_to_float(x[n]);
    }
    __syncthreads();
  }
};

// float64 products on the matrix cores: 16 x 16 of them a wave, a lane's four elements are rows
// lane / 16 + 4 i of column lane % 16.  (Two rows by two columns a thread from local memory,
// without them: a call for one 32 x 32 matrix 29 us, so 17.)
typedef double Four __attribute__((ext_vector_type(4)));
typedef double FewMatrix[kFewRows][kFewRows + 2];

__device__ __forceinline__ Four few_mfma(double x, double y, Four sum) {
  return __builtin_amdgcn_mfma_f64_16x16x4f64(x, y, sum, 0, 0, 0);
}
// The four of a wave's quarter of a matrix.
__device__ __forceinline__ int four_row(int i) { return threadIdx.x / (2 * kWave) * 16 + threadIdx.x % kWave / 16 + 4 * i; }
__device__ __forceinline__ int four_column() { return threadIdx.x / kWave % 2 * 16 + threadIdx.x % 16; }
__device__ __forceinline__ int mfma_k() { return threadIdx.x % kWave / 16; }

template <typename In>
__device__ void few_gram(const Table& t, int id) {
  __shared__ FewTile s_tile;
  const Entry& g = t.at[entry_of(t, id, [](const Entry& e) { return e.first_partial; }, t.count, t.few)];
  const int64_t chunk = id - g.first_partial, from = chunk * few_chunk(g.c);
  const int64_t to = from + few_chunk(g.c) < g.c ? from + few_chunk(g.c) : g.c;
  const int row = threadIdx.x / (2 * kWave) * 16 + threadIdx.x % 16, column = four_column();
  Four sum = {};
  FewFetch<In> tile;
  tile.fetch(g, from);
  for (int64_t j0 = from; j0 < to; j0 += kFewTile) {
    tile.put(g, j0, s_tile);
    if (j0 + kFewTile < to) tile.fetch(g, j0 + kFewTile);
#pragma unroll
    for (int k = 0; k < kFewTile; k += 4) sum = few_mfma(s_tile[row][k + mfma_k()], s_tile[column][k + mfma_k()], sum);
    __syncthreads();
  }
  double* const out = reinterpret_cast<double*>(g.base) + chunk * kFewRows * kFewRows;
#pragma unroll
  for (int i = 0; i < 4; ++i) out[four_row(i) * kFewRows + four_column()] = sum[i];
}

__device__ __forceinline__ void store_four(FewMatrix& m, const Four& f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) m[four_row(i)][four_column()] = f[i];
}
__device__ __forceinline__ Four few_product(const FewMatrix& x, const FewMatrix& y, int r) {
  const int row = threadIdx.x / (2 * kWave) * 16 + threadIdx.x % 16, column = four_column();
  Four f = {};
#pragma unroll
  for (int k = 0; k < kFewRows; k += 4)
    if (k < r) f = few_mfma(x[row][k + mfma_k()], y[k + mfma_k()][column], f);
  return f;
}

// The result's columns from few_block * block on; every workgroup of a matrix forms its Q.
constexpr int kFewLds = 3 * sizeof(FewMatrix) + sizeof(FewTile);
template <typename In>
__device__ void few_apply(const Table& t, const FewSteps& steps, int id, char* lds) {
  FewMatrix* const s_few = reinterpret_cast<FewMatrix*>(lds);
  FewMatrix &s_a = s_few[0], &s_p = s_few[1], &s_q = s_few[2];
  FewTile& s_tile = *reinterpret_cast<FewTile*>(lds + 3 * sizeof(FewMatrix));
  const Entry& g = t.at[entry_of(t, id, [](const Entry& e) { return e.first_block; }, t.count, t.few)];
  const double* const partials = reinterpret_cast<const double*>(g.base);
  const int64_t from = static_cast<int64_t>(id - g.first_block) * t.few_block;
  const int64_t to = from + t.few_block < g.c ? from + t.few_block : g.c;
  FewFetch<In> tile;
  tile.fetch(g, from);
  Four a = {};
#pragma unroll 8
  for (int chunk = 0; chunk < g.partials; ++chunk)
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] += partials[(chunk * kFewRows + four_row(i)) * kFewRows + four_column()];
  store_four(s_a, a);
  __syncthreads();
  double squares = 0.0;
#pragma unroll
  for (int i = 0; i < kFewRows; ++i) squares += s_a[i][i];
  const double norm = sqrt(squares), least = t.epsilon;
  const double factor = 1.0 / (norm < least ? least : norm);  // a NaN norm stays
  __syncthreads();
  a = a * factor * factor;
  store_four(s_a, a);
  __syncthreads();
  for (int k = 0; k < steps.count; ++k) {
    const double pa = steps.at[k].a, pb = steps.at[k].b, pc = steps.at[k].c;
    const Four aa = few_product(s_a, s_a, g.r);
    Four p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = (four_row(i) == four_column() ? pa : 0.0) + pb * a[i] + pc * aa[i];
    store_four(s_p, p);
    __syncthreads();
    const bool last = k + 1 == steps.count;
    const Four q = k == 0 ? p : few_product(s_p, s_q, g.r);
    if (!last) a = few_product(s_p, s_a, g.r);
    __syncthreads();
    store_four(s_q, q);
    store_four(s_a, a);
    __syncthreads();
    if (last) break;
    a = few_product(s_a, s_p, g.r);
    __syncthreads();
    store_four(s_a, a);
    __syncthreads();
  }
  const double scale = factor * g.scale;
  for (int64_t j0 = from; j0 < to; j0 += kFewTile) {
    tile.put(g, j0, s_tile);
    if (j0 + kFewTile < to) tile.fetch(g, j0 + kFewTile);
    // A wave's 16 columns, of all rows.
    const int column = threadIdx.x / kWave * 16 + threadIdx.x % 16;
    Four y[2] = {};
#pragma unroll
    for (int k = 0; k < kFewRows; k += 4) {
      const double x = s_tile[k + mfma_k()][column];
#pragma unroll
      for (int half = 0; half < 2; ++half) y[half] = few_mfma(s_q[16 * half + threadIdx.x % 16][k + mfma_k()], x, y[half]);
    }
    __syncthreads();
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_tile[16 * half + mfma_k() + 4 * i][column] = static_cast<float>(y[half][i] * scale);
    __syncthreads();
    In* const out = static_cast<In*>(g.out);
#pragma unroll
    for (int n = 0; n < kFewEach; ++n) {
      const FewPlace p = few_place(g, static_cast<int>(j0), n);
      if (p.at < 0) continue;
      if constexpr (sizeof(In) == 4) out[p.at] = s_tile[p.row][p.column];
      else out[p.at] = to_bf16(s_tile[p.row][p.column]);
    }
    __syncthreads();
  }
}

}  // namespace
}  // namespace vtrace
