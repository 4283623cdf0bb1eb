// Layer norm over the columns of a matrix, and its gradient.
//
// A row is held in the registers of L lanes, C chunks of E entries each (16 bytes of memory), so that it is read once:
// the mean first, then the sum of squares about it, as exact as two passes over memory.  L is the smallest power of two
// that covers the columns, at least a group of the 8-bit form, up to a wavefront, then a workgroup; longer rows than
// that holds are read once per sum (they fit the L2).  The gradient of the weight is summed by the lanes along the rows
// that they walk, then over the rows of a workgroup, and the workgroups' sums are joined in a fixed order by a second
// kernel: no atomics, the same bits every time.
//
// Bound by memory.  300,007 x 501 in f32: 252 us, 4.8 TB/s; the gradient of 2^20 x 128 in bf16 with another branch's: 203
// us, 5.3 TB/s; 400,003 x 96 in f16 forward and back through 8-bit rows: 95 us, 4.1 TB/s (134 without loading a turn's
// rows during the turn before).  Rows of 15 entries leave half of a wavefront's bytes unused: 1.9 M of them 128 us, 1.9
// TB/s.
#include <algorithm>

#include "gosh_head.h"

namespace gosh {
namespace {

// Sum over the L lanes of a row (L = 256: over the workgroup, whose threads all come here).
template <int L>
__device__ __forceinline__ float row_sum(float v, float *lds) {
#pragma unroll
  for (int s = 1; s < (L < 64 ? L : 64); s *= 2) v += __shfl_xor(v, s);
  if constexpr (L == 256) {
    __syncthreads();  // who still reads the last sum
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = (lds[0] + lds[1]) + (lds[2] + lds[3]);
  }
  return v;
}

struct NormArgs {
  Plane x, y, xhat8, y8;
  const float *gamma, *beta;
  float *mean, *rstd;
  int64_t rows;
  int32_t cols;
  float eps;
};

template <typename T>
struct Chunk {
  static constexpr int E = T::kType == GOSH_F32 ? 4 : 8;
  static constexpr int kGroupLanes = kGroup / E;
};

template <typename T, int L, int C>
__global__ __launch_bounds__(256) void norm_kernel(const NormArgs g) {
  constexpr int E = Chunk<T>::E;
  typedef typename T::Store S;
  __shared__ float lds[4];
  const int lane = threadIdx.x % L;
  // divided by, not multiplied with its inverse: the mean of equal entries is that entry
  const float width = static_cast<float>(g.cols);
  int col[C], count[C];
  float gamma[C][E], beta[C][E];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = (c * L + lane) * E;
    count[c] = g.cols - col[c] < 0 ? 0 : g.cols - col[c] < E ? g.cols - col[c] : E;
#pragma unroll
    for (int e = 0; e < E; ++e) gamma[c][e] = beta[c][e] = 0.f;
    if (count[c] > 0) {
      Entries<F32, E>::load(g.gamma + col[c], count[c], gamma[c]);
      Entries<F32, E>::load(g.beta + col[c], count[c], beta[c]);
    }
  }
  // the rows of a workgroup take turns together, past the last one without memory accesses; a turn's rows are loaded
  // while the turn before is worked on
  typename Entries<T, E>::Vec next[C];
  const auto fetch = [&](int64_t first) {
    const int64_t row = first + threadIdx.x / L;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      next[c] = 0;
      if (row < g.rows && count[c] > 0) next[c] = Entries<T, E>::fetch(static_cast<const S *>(g.x.data) + row * g.x.ld + col[c], count[c]);
    }
  };
  const int64_t step = static_cast<int64_t>(gridDim.x) * (256 / L);
  fetch(static_cast<int64_t>(blockIdx.x) * (256 / L));
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * (256 / L); first < g.rows; first += step) {
    const int64_t row = first + threadIdx.x / L;
    const bool there = row < g.rows;
    float v[C][E];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[c][e] = T::up(next[c][e]);
        sum += v[c][e];
      }
    fetch(first + step);
    const float mean = row_sum<L>(sum, lds) / width;
    float squares = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[c][e] = e < count[c] ? v[c][e] - mean : 0.f;
        squares = fmaf(v[c][e], v[c][e], squares);
      }
    const float rstd = 1.f / sqrtf(row_sum<L>(squares, lds) / width + g.eps);
    if (there && lane == 0) {
      if (g.mean != nullptr) g.mean[row] = mean;
      if (g.rstd != nullptr) g.rstd[row] = rstd;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int here = there ? count[c] : 0;
#pragma unroll
      for (int e = 0; e < E; ++e) v[c][e] *= rstd;
      const bool head = lane % Chunk<T>::kGroupLanes == 0;
      if (g.xhat8.data != nullptr) store_packed<T, E>(g.xhat8, row, col[c], here, v[c], head, Chunk<T>::kGroupLanes);
#pragma unroll
      for (int e = 0; e < E; ++e) v[c][e] = fmaf(v[c][e], gamma[c][e], beta[c][e]);
      if (g.y8.data != nullptr) store_packed<T, E>(g.y8, row, col[c], here, v[c], head, Chunk<T>::kGroupLanes);
      if (here > 0) Entries<T, E>::store(static_cast<S *>(g.y.data) + row * g.y.ld + col[c], here, v[c]);
    }
  }
}

// Rows too long for registers: a workgroup a row, which it reads three times.
template <typename T>
__global__ __launch_bounds__(256) void norm_long_kernel(const NormArgs g) {
  constexpr int E = Chunk<T>::E;
  typedef typename T::Store S;
  __shared__ float lds[4];
  const float width = static_cast<float>(g.cols);
  for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
    const S *const x = static_cast<const S *>(g.x.data) + row * g.x.ld;
    float v[E], sum = 0.f, squares = 0.f;
    for (int col = threadIdx.x * E; col < g.cols; col += 256 * E) {
      Entries<T, E>::load(x + col, g.cols - col, v);
#pragma unroll
      for (int e = 0; e < E; ++e) sum += v[e];
    }
    const float mean = row_sum<256>(sum, lds) / width;
    for (int col = threadIdx.x * E; col < g.cols; col += 256 * E) {
      Entries<T, E>::load(x + col, g.cols - col, v);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = e < g.cols - col ? v[e] - mean : 0.f;
        squares = fmaf(d, d, squares);
      }
    }
    const float rstd = 1.f / sqrtf(row_sum<256>(squares, lds) / width + g.eps);
    if (threadIdx.x == 0) {
      if (g.mean != nullptr) g.mean[row] = mean;
      if (g.rstd != nullptr) g.rstd[row] = rstd;
    }
    // whole groups of lanes stay together for the 8-bit form
    for (int first = 0; first < g.cols; first += 256 * E) {
      const int col = first + threadIdx.x * E;
      const int count = g.cols - col < 0 ? 0 : g.cols - col < E ? g.cols - col : E;
      float gamma[E], beta[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = gamma[e] = beta[e] = 0.f;
      if (count > 0) {
        Entries<T, E>::load(x + col, count, v);
        Entries<F32, E>::load(g.gamma + col, count, gamma);
        Entries<F32, E>::load(g.beta + col, count, beta);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = e < count ? (v[e] - mean) * rstd : 0.f;
      const bool head = threadIdx.x % Chunk<T>::kGroupLanes == 0;
      if (g.xhat8.data != nullptr) store_packed<T, E>(g.xhat8, row, col, count, v, head, Chunk<T>::kGroupLanes);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = fmaf(v[e], gamma[e], beta[e]);
      if (g.y8.data != nullptr) store_packed<T, E>(g.y8, row, col, count, v, head, Chunk<T>::kGroupLanes);
      if (count > 0) Entries<T, E>::store(static_cast<S *>(g.y.data) + row * g.y.ld + col, count, v);
    }
  }
}

struct NormBackArgs {
  Plane dy, x, add, dx;
  const float *gamma, *mean, *rstd;
  float *parts;  // gridDim.x x 2 x cols: dgamma, dbeta; or null
  int64_t rows;
  int32_t cols;
  int32_t packed;
};

// xhat of a chunk: what the 8-bit form stands for, or from x and the row's statistics.
template <typename T, int E>
__device__ __forceinline__ void load_xhat(const NormBackArgs &g, int64_t row, int col, int count, float mean, float rstd, float (&v)[E]) {
  load_entries<T, E>(g.x, g.packed != 0, row, col, count, v);
  if (!g.packed)
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e < count ? (v[e] - mean) * rstd : 0.f;
}

template <typename T, int L, int C>
__global__ __launch_bounds__(256) void norm_back_kernel(const NormBackArgs g) {
  constexpr int E = Chunk<T>::E;
  typedef typename T::Store S;
  __shared__ float sums[4];
  __shared__ float lds[L < 256 ? 256 * E : 1];
  const int lane = threadIdx.x % L;
  const float inv = 1.f / static_cast<float>(g.cols);
  int col[C], count[C];
  float gamma[C][E], dgamma[C][E], dbeta[C][E];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = (c * L + lane) * E;
    count[c] = g.cols - col[c] < 0 ? 0 : g.cols - col[c] < E ? g.cols - col[c] : E;
#pragma unroll
    for (int e = 0; e < E; ++e) gamma[c][e] = dgamma[c][e] = dbeta[c][e] = 0.f;
    if (count[c] > 0) Entries<F32, E>::load(g.gamma + col[c], count[c], gamma[c]);
  }
  // a turn's rows are loaded while the turn before is worked on
  constexpr int kWords = E * sizeof(S) / 4;
  typename Entries<T, E>::Vec next_d[C];
  uint32_t next_x[C][kWords], next_unit[C];
  float next_rstd, next_mean;
  const auto fetch = [&](int64_t first) {
    const int64_t row = first + threadIdx.x / L;
    const bool there = row < g.rows;
    next_rstd = there ? g.rstd[row] : 0.f;
    next_mean = there && !g.packed ? g.mean[row] : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      next_d[c] = 0;
      next_unit[c] = 0;
#pragma unroll
      for (int w = 0; w < kWords; ++w) next_x[c][w] = 0;
      if (!there || count[c] <= 0) continue;
      next_d[c] = Entries<T, E>::fetch(static_cast<const S *>(g.dy.data) + row * g.dy.ld + col[c], count[c]);
      if (g.packed) {
        uint32_t q[E / 4];
        load_bytes<E>(static_cast<const int8_t *>(g.x.data) + row * g.x.ld + col[c], count[c], q);
#pragma unroll
        for (int w = 0; w < E / 4; ++w) next_x[c][w] = q[w];
        next_unit[c] = g.x.exps[row * g.x.ld_exps + col[c] / kGroup];
      } else {
        const auto x = Entries<T, E>::fetch(static_cast<const S *>(g.x.data) + row * g.x.ld + col[c], count[c]);
        const auto u = __builtin_bit_cast(typename Words<kWords>::V, x);
#pragma unroll
        for (int w = 0; w < kWords; ++w) next_x[c][w] = u[w];
      }
    }
  };
  const int64_t step = static_cast<int64_t>(gridDim.x) * (256 / L);
  fetch(static_cast<int64_t>(blockIdx.x) * (256 / L));
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * (256 / L); first < g.rows; first += step) {
    const int64_t row = first + threadIdx.x / L;
    const bool there = row < g.rows;
    const float rstd = next_rstd, mean = next_mean;
    float d[C][E], xhat[C][E];
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (g.packed) {
        uint32_t q[E / 4];
#pragma unroll
        for (int w = 0; w < E / 4; ++w) q[w] = next_x[c][w];
        widen<E>(q, read_unit(next_unit[c]), xhat[c]);
      } else {
        typename Words<kWords>::V u;
#pragma unroll
        for (int w = 0; w < kWords; ++w) u[w] = next_x[c][w];
        const auto x = __builtin_bit_cast(typename Entries<T, E>::Vec, u);
#pragma unroll
        for (int e = 0; e < E; ++e) xhat[c][e] = e < count[c] ? (T::up(x[e]) - mean) * rstd : 0.f;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) d[c][e] = T::up(next_d[c][e]);
    }
    fetch(first + step);
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        dgamma[c][e] = fmaf(d[c][e], xhat[c][e], dgamma[c][e]);
        dbeta[c][e] += d[c][e];
        d[c][e] *= gamma[c][e];
        s0 += d[c][e];
        s1 = fmaf(d[c][e], xhat[c][e], s1);
      }
    }
    if (g.dx.data == nullptr) continue;
    s0 = row_sum<L>(s0, sums) * inv;
    s1 = row_sum<L>(s1, sums) * inv;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!there || count[c] <= 0) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) d[c][e] = rstd * (d[c][e] - s0 - xhat[c][e] * s1);
      if (g.add.data != nullptr) {
        float a[E];
        Entries<T, E>::load(static_cast<const S *>(g.add.data) + row * g.add.ld + col[c], count[c], a);
#pragma unroll
        for (int e = 0; e < E; ++e) d[c][e] += a[e];
      }
      Entries<T, E>::store(static_cast<S *>(g.dx.data) + row * g.dx.ld + col[c], count[c], d[c]);
    }
  }
  if (g.parts == nullptr) return;
  // the sums of the workgroup's rows, dgamma then dbeta, a chunk at a time
  float *const part = g.parts + static_cast<int64_t>(blockIdx.x) * 2 * g.cols;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = which == 0 ? dgamma[c][e] : dbeta[c][e];
      if constexpr (L < 256) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) lds[threadIdx.x * E + e] = v[e];
        __syncthreads();
        if (threadIdx.x < L)
          for (int s = 1; s < 256 / L; ++s)
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] += lds[(s * L + threadIdx.x) * E + e];
      }
      if (threadIdx.x < L && count[c] > 0) Entries<F32, E>::store(part + which * g.cols + col[c], count[c], v);
    }
}

// dx of rows too long for registers.
template <typename T>
__global__ __launch_bounds__(256) void norm_back_long_kernel(const NormBackArgs g) {
  constexpr int E = Chunk<T>::E;
  typedef typename T::Store S;
  __shared__ float lds[4];
  const float inv = 1.f / static_cast<float>(g.cols);
  for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
    const S *const dy = static_cast<const S *>(g.dy.data) + row * g.dy.ld;
    const float rstd = g.rstd[row], mean = g.packed ? 0.f : g.mean[row];
    float s0 = 0.f, s1 = 0.f;
    for (int col = threadIdx.x * E; col < g.cols; col += 256 * E) {
      const int count = g.cols - col;
      float d[E], xhat[E], gamma[E];
      Entries<T, E>::load(dy + col, count, d);
      load_xhat<T, E>(g, row, col, count, mean, rstd, xhat);
      Entries<F32, E>::load(g.gamma + col, count, gamma);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        s0 = fmaf(d[e], gamma[e], s0);
        s1 = fmaf(d[e] * gamma[e], xhat[e], s1);
      }
    }
    s0 = row_sum<256>(s0, lds) * inv;
    s1 = row_sum<256>(s1, lds) * inv;
    for (int col = threadIdx.x * E; col < g.cols; col += 256 * E) {
      const int count = g.cols - col;
      float d[E], xhat[E], gamma[E];
      Entries<T, E>::load(dy + col, count, d);
      load_xhat<T, E>(g, row, col, count, mean, rstd, xhat);
      Entries<F32, E>::load(g.gamma + col, count, gamma);
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = rstd * (d[e] * gamma[e] - s0 - xhat[e] * s1);
      if (g.add.data != nullptr) {
        float a[E];
        Entries<T, E>::load(static_cast<const S *>(g.add.data) + row * g.add.ld + col, count, a);
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] += a[e];
      }
      Entries<T, E>::store(static_cast<S *>(g.dx.data) + row * g.dx.ld + col, count, d);
    }
  }
}

// Their dgamma and dbeta: a thread has a chunk of columns, a workgroup (blockIdx.y) a run of rows.
template <typename T>
__global__ __launch_bounds__(256) void norm_sums_kernel(const NormBackArgs g, int64_t rows_per_block) {
  constexpr int E = Chunk<T>::E;
  typedef typename T::Store S;
  const int col = (blockIdx.x * 256 + threadIdx.x) * E;
  const int count = g.cols - col;
  if (count <= 0) return;
  const int64_t r0 = blockIdx.y * rows_per_block, r1 = r0 + rows_per_block < g.rows ? r0 + rows_per_block : g.rows;
  float dgamma[E], dbeta[E];
#pragma unroll
  for (int e = 0; e < E; ++e) dgamma[e] = dbeta[e] = 0.f;
  for (int64_t row = r0; row < r1; ++row) {
    float d[E], xhat[E];
    Entries<T, E>::load(static_cast<const S *>(g.dy.data) + row * g.dy.ld + col, count, d);
    load_xhat<T, E>(g, row, col, count, g.packed ? 0.f : g.mean[row], g.packed ? 1.f : g.rstd[row], xhat);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      dgamma[e] = fmaf(d[e], xhat[e], dgamma[e]);
      dbeta[e] += d[e];
    }
  }
  float *const part = g.parts + static_cast<int64_t>(blockIdx.y) * 2 * g.cols;
  Entries<F32, E>::store(part + col, count, dgamma);
  Entries<F32, E>::store(part + g.cols + col, count, dbeta);
}

constexpr int kMostParts = 1024;  // workgroups of the gradient, each of which leaves sums of its rows: 16 wavefronts a CU

// Shape of the lanes for one row: L lanes of C chunks of 16 bytes; C = 0 for rows that registers do not hold.
struct RowShape {
  int L, C;
};
RowShape shape_of(int32_t cols, int32_t type) {
  const int chunks = static_cast<int>(ceil_div(cols, type == GOSH_F32 ? 4 : 8)), least = type == GOSH_F32 ? 8 : 4;
  if (chunks <= 64) {
    int L = least;
    while (L < chunks) L *= 2;
    return {L, 1};
  }
  for (int C = 2; C <= 4; C *= 2)
    if (chunks <= 64 * C) return {64, C};
  for (int C = 2; C <= 4; C *= 2)
    if (chunks <= 256 * C) return {256, C};
  return {256, 0};
}

// A few rows get a workgroup each turn of 4 rows (the sums of 4 rows are more bytes than half of what the rows read).
int64_t back_blocks(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(ceil_div(rows, 4), kMostParts)); }

template <typename T, typename F>
int with_shape(RowShape s, F f) {
  constexpr int least = T::kType == GOSH_F32 ? 8 : 4;
  typedef std::integral_constant<int, 1> I1;
  typedef std::integral_constant<int, 2> I2;
  typedef std::integral_constant<int, 4> I4;
  if (s.L == 64) {
    if (s.C == 1) f(std::integral_constant<int, 64>{}, I1{});
    else if (s.C == 2) f(std::integral_constant<int, 64>{}, I2{});
    else f(std::integral_constant<int, 64>{}, I4{});
  } else if (s.L == 256) {
    if (s.C == 2) f(std::integral_constant<int, 256>{}, I2{});
    else f(std::integral_constant<int, 256>{}, I4{});
  } else if (s.L == 32) {
    f(std::integral_constant<int, 32>{}, I1{});
  } else if (s.L == 16) {
    f(std::integral_constant<int, 16>{}, I1{});
  } else if (s.L == 8) {
    f(std::integral_constant<int, 8>{}, I1{});
  } else {
    f(std::integral_constant<int, least>{}, I1{});
  }
  return GOSH_OK;
}

template <typename T>
int norm(const NormArgs &g, hipStream_t st) {
  const RowShape s = shape_of(g.cols, T::kType);
  const int64_t most = 8 * 256;  // workgroups that the device holds
  if (s.C == 0) {
    norm_long_kernel<T><<<dim3(static_cast<unsigned>(std::min(g.rows, most))), dim3(256), 0, st>>>(g);
  } else {
    const unsigned blocks = static_cast<unsigned>(std::min(ceil_div(g.rows, 256 / s.L), most));
    with_shape<T>(s, [&](auto L, auto C) {
      norm_kernel<T, decltype(L)::value, decltype(C)::value><<<dim3(blocks), dim3(256), 0, st>>>(g);
    });
  }
  return check_launch("layer norm");
}

template <typename T>
int norm_back(NormBackArgs g, float *dgamma, float *dbeta, hipStream_t st) {
  const RowShape s = shape_of(g.cols, T::kType);
  int64_t parts = 0;
  if (g.rows > 0) {
    if (s.C == 0) {
      if (g.parts != nullptr) {  // first: dx may be dy
        const int64_t per = ceil_div(g.rows, back_blocks(g.rows));
        parts = ceil_div(g.rows, per);
        const unsigned across = static_cast<unsigned>(ceil_div(g.cols, 256 * Chunk<T>::E));
        norm_sums_kernel<T><<<dim3(across, static_cast<unsigned>(parts)), dim3(256), 0, st>>>(g, per);
        if (int rc = check_launch("gradient of the layer norm")) return rc;
      }
      if (g.dx.data != nullptr)
        norm_back_long_kernel<T><<<dim3(static_cast<unsigned>(std::min<int64_t>(g.rows, 2048))), dim3(256), 0, st>>>(g);
    } else {
      parts = back_blocks(g.rows);
      with_shape<T>(s, [&](auto L, auto C) {
        norm_back_kernel<T, decltype(L)::value, decltype(C)::value><<<dim3(static_cast<unsigned>(parts)), dim3(256), 0, st>>>(g);
      });
    }
    if (int rc = check_launch("gradient of the layer norm")) return rc;
  }
  if (dgamma != nullptr) {
    const int64_t stride = 2 * static_cast<int64_t>(g.cols);
    const int count = static_cast<int>(parts);
    const JoinJob jobs[2] = {{g.parts, stride, g.cols, g.cols, dgamma, count, g.cols, GOSH_F32},
                             {g.parts + g.cols, stride, g.cols, g.cols, dbeta, count, g.cols, GOSH_F32}};
    return join_parts(jobs, 2, st);
  }
  return GOSH_OK;
}

}  // namespace
}  // namespace gosh

extern "C" {

int gosh_layer_norm(const gosh_mat *x, const float *gamma, const float *beta, float eps, const gosh_mat *y, float *mean,
                    float *rstd, const gosh_mat *xhat8, const gosh_mat *y8, void *hip_stream) {
  using namespace gosh;
  if (int rc = check_mat(x, "x")) return rc;
  if (int rc = check_mat(y, "y")) return rc;
  if (int rc = check_mat(xhat8, "xhat8", kOptional | kMustBePacked)) return rc;
  if (int rc = check_mat(y8, "y8", kOptional | kMustBePacked)) return rc;
  if (!(eps >= 0.f)) return fail(GOSH_EINVAL, "eps = %g: must not be negative", eps);
  const struct { const gosh_mat *m; const char *what; } outs[] = {{y, "y"}, {xhat8, "xhat8"}, {y8, "y8"}};
  for (const auto &o : outs) {
    if (int rc = check_shape(o.m, o.what, x->rows, x->cols)) return rc;
    if (int rc = check_type(o.m, o.what, x->type)) return rc;
  }
  if (int rc = check_floats(gamma, x->cols, "gamma", false)) return rc;
  if (int rc = check_floats(beta, x->cols, "beta", false)) return rc;
  if (int rc = check_floats(mean, x->rows, "mean", true)) return rc;
  if (int rc = check_floats(rstd, x->rows, "rstd", true)) return rc;
  if (x->rows == 0) return GOSH_OK;
  const NormArgs g{plane_of(x), plane_of(y), plane_of(xhat8), plane_of(y8), gamma, beta, mean, rstd, x->rows, x->cols, eps};
  hipStream_t st = as_stream(hip_stream);
  if (x->type == GOSH_F32) return norm<F32>(g, st);
  if (x->type == GOSH_BF16) return norm<Bf16>(g, st);
  return norm<F16>(g, st);
}

uint64_t gosh_layer_norm_workspace(int64_t rows, int32_t cols) {
  if (rows < 1 || !gosh::rows_fit(rows) || cols < 1 || cols > GOSH_MAT_MAX_COLS) return 0;
  return static_cast<uint64_t>(gosh::back_blocks(rows)) * 2 * cols * 4;
}

int gosh_layer_norm_backward(const gosh_mat *dy, const gosh_mat *x, const float *gamma, const float *mean,
                             const float *rstd, const gosh_mat *add, const gosh_mat *dx, float *dgamma, float *dbeta,
                             void *workspace, uint64_t workspace_bytes, void *hip_stream) {
  using namespace gosh;
  if (int rc = check_mat(dy, "dy")) return rc;
  if (int rc = check_mat(x, "x", kMayBePacked)) return rc;
  if (int rc = check_mat(add, "add", kOptional)) return rc;
  if (int rc = check_mat(dx, "dx", kOptional)) return rc;
  const struct { const gosh_mat *m; const char *what; } all[] = {{x, "x"}, {add, "add"}, {dx, "dx"}};
  for (const auto &o : all) {
    if (int rc = check_shape(o.m, o.what, dy->rows, dy->cols)) return rc;
    if (int rc = check_type(o.m, o.what, dy->type)) return rc;
  }
  if ((dgamma == nullptr) != (dbeta == nullptr)) return fail(GOSH_EINVAL, "dgamma and dbeta: both or neither may be null");
  if (int rc = check_floats(gamma, dy->cols, "gamma", false)) return rc;
  if (int rc = check_floats(mean, dy->rows, "mean", x->packed != 0)) return rc;
  if (int rc = check_floats(rstd, dy->rows, "rstd", false)) return rc;
  if (int rc = check_floats(dgamma, dy->cols, "dgamma", true)) return rc;
  if (int rc = check_floats(dbeta, dy->cols, "dbeta", true)) return rc;
  if (dgamma != nullptr)
    if (int rc = check_workspace(workspace, workspace_bytes, gosh_layer_norm_workspace(dy->rows, dy->cols))) return rc;
  const NormBackArgs g{plane_of(dy), plane_of(x), plane_of(add), plane_of(dx), gamma, mean, rstd,
                       dgamma != nullptr ? static_cast<float *>(workspace) : nullptr, dy->rows, dy->cols, x->packed};
  hipStream_t st = as_stream(hip_stream);
  if (dy->type == GOSH_F32) return norm_back<F32>(g, dgamma, dbeta, st);
  if (dy->type == GOSH_BF16) return norm_back<Bf16>(g, dgamma, dbeta, st);
  return norm_back<F16>(g, dgamma, dbeta, st);
}

}  // extern "C"
