// Softmax cross-entropy of rows of logits, with its gradient.
//
// A row stays in the registers of the lanes that share it, from 4 lanes of a wavefront to a workgroup of 1,024 (65,536
// entries in 32 bits), so that logits are read once and the gradient is written once: bound by memory.  Each lane subtracts
// the row's maximum (joined over the lanes first), keeps e = exp(x - max), and the lanes join the sum of e:
//   loss = log(sum) + (max - x[target]),  gradient = scale weight (e / sum - [class = target]).
#include <algorithm>

#include "gosh_head.h"

namespace gosh {
namespace {

struct LossArgs {
  Plane x, d;
  const void *targets;
  const float *weight;
  float *loss;
  int64_t rows;
  int32_t cols, targets_are64;
  float scale;
};

__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }  // keeps NaN

// Over `Lanes` lanes of a wavefront, to all of them.
template <int Lanes, typename Op>
__device__ __forceinline__ float over_lanes(float v, Op op) {
#pragma unroll
  for (int s = 1; s < Lanes; s *= 2) v = op(v, __shfl_xor(v, s));
  return v;
}

// The loss and the gradient of a row, Lanes lanes with Count chunks of E entries each: chunk c of lane l is at (c * Lanes
// + l) * E.
template <typename T, int Lanes, int Count>
__global__ __launch_bounds__(Lanes > 256 ? Lanes : 256) void loss_kernel(const LossArgs a) {
  constexpr int E = T::kType == GOSH_F32 ? 4 : 8;
  constexpr int kThreads = Lanes > 256 ? Lanes : 256, kRows = kThreads / Lanes, kWaves = Lanes / 64;
  typedef typename T::Store S;
  __shared__ float lds[kWaves > 1 ? 2 * kThreads / 64 : 1];
  const int lane = threadIdx.x % Lanes;
  const auto join = [&](float v, int which, auto op) {
    v = over_lanes<(Lanes < 64 ? Lanes : 64)>(v, op);
    if constexpr (kWaves > 1) {
      const int wave = threadIdx.x / 64, first = wave / kWaves * kWaves;
      float *const mine = lds + which * (kThreads / 64);
      if (threadIdx.x % 64 == 0) mine[wave] = v;
      __syncthreads();
      v = mine[first];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v = op(v, mine[first + w]);
    }
    return v;
  };
  // every thread of a workgroup takes as many turns: the joins wait for each other
  for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * kRows; row0 < a.rows; row0 += static_cast<int64_t>(gridDim.x) * kRows) {
    const int64_t row = row0 + threadIdx.x / Lanes;
    const bool there = row < a.rows;
    int64_t target = -1;
    float weight = 1.f;
    if (there) {
      target = a.targets_are64 ? static_cast<const int64_t *>(a.targets)[row] : static_cast<const int32_t *>(a.targets)[row];
      if (a.weight != nullptr) weight = a.weight[row];
    }
    const S *const x = static_cast<const S *>(a.x.data) + row * a.x.ld;
    float v[Count][E], most = -INFINITY;
#pragma unroll
    for (int c = 0; c < Count; ++c) {
      const int at = (c * Lanes + lane) * E;
      const int left = there ? a.cols - at : 0;
      Entries<T, E>::load(x + at, left < 0 ? 0 : left, v[c]);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[c][e] = e < left ? v[c][e] : -INFINITY;
        most = larger(most, v[c][e]);
      }
    }
    most = join(most, 0, larger);
    const bool nothing = target < 0 || weight == 0.f || most == -INFINITY;
    const float from = nothing ? 0.f : most;
    float sum = 0.f, hit = -INFINITY;  // hit: the target's logit
#pragma unroll
    for (int c = 0; c < Count; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if ((c * Lanes + lane) * E + e == target) hit = v[c][e];
        v[c][e] = __expf(v[c][e] - from);
        sum += v[c][e];
      }
    sum = join(sum, 1, [](float p, float q) { return p + q; });
    const bool wrong = target >= a.cols;
    if (there) {
      const float nan = __uint_as_float(0x7fc00000u);
      const int holder = static_cast<int>(target / E % Lanes);
      if (nothing || wrong ? lane == 0 : lane == holder)
        a.loss[row] = nothing ? 0.f : wrong ? nan : weight * (logf(sum) + (most - hit));
      if (a.d.data != nullptr) {
        const float share = nothing ? 0.f : a.scale * weight / sum, whole = wrong ? nan : a.scale * weight;
        S *const d = static_cast<S *>(a.d.data) + row * a.d.ld;
#pragma unroll
        for (int c = 0; c < Count; ++c) {
          const int at = (c * Lanes + lane) * E, left = a.cols - at;
          if (left <= 0) continue;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            v[c][e] = nothing ? 0.f : wrong ? nan : v[c][e] * share;
            if (at + e == target) v[c][e] -= nothing ? 0.f : whole;
          }
          Entries<T, E>::store(d + at, left, v[c]);
        }
      }
    }
  }
}

template <typename T, int Lanes, int Count>
int launch_loss(const LossArgs &a, hipStream_t st) {
  constexpr int kThreads = Lanes > 256 ? Lanes : 256, kRows = kThreads / Lanes;
  const unsigned blocks = static_cast<unsigned>(std::min<int64_t>(ceil_div(a.rows, kRows), int64_t{1} << 20));
  loss_kernel<T, Lanes, Count><<<dim3(blocks), dim3(kThreads), 0, st>>>(a);
  return check_launch("softmax loss");
}

template <typename T>
int loss_of(const LossArgs &a, hipStream_t st) {
  constexpr int E = T::kType == GOSH_F32 ? 4 : 8;
  const int64_t chunks = ceil_div(a.cols, E);
  if (chunks <= 4) return launch_loss<T, 4, 1>(a, st);
  if (chunks <= 8) return launch_loss<T, 8, 1>(a, st);
  if (chunks <= 16) return launch_loss<T, 16, 1>(a, st);
  if (chunks <= 32) return launch_loss<T, 16, 2>(a, st);
  if (chunks <= 64) return launch_loss<T, 32, 2>(a, st);
  if (chunks <= 128) return launch_loss<T, 64, 2>(a, st);
  if (chunks <= 256) return launch_loss<T, 64, 4>(a, st);
  if (chunks <= 512) return launch_loss<T, 256, 2>(a, st);
  if (chunks <= 1024) return launch_loss<T, 256, 4>(a, st);
  if (chunks <= 2048) return launch_loss<T, 512, 4>(a, st);
  if (chunks <= 4096) return launch_loss<T, 1024, 4>(a, st);
  if (chunks <= 8192) return launch_loss<T, 1024, 8>(a, st);
  if constexpr (T::kType == GOSH_F32) return launch_loss<T, 1024, 16>(a, st);
  return fail(GOSH_EINVAL, "logits: cols = %d: too many", a.cols);
}

}  // namespace
}  // namespace gosh

extern "C" {

int gosh_softmax_loss(const gosh_mat *logits, const void *targets, int32_t targets_are64, const float *weight, float scale,
                      float *loss, const gosh_mat *dlogits, void *hip_stream) {
  using namespace gosh;
  if (int rc = check_mat(logits, "logits")) return rc;
  if (int rc = check_mat(dlogits, "dlogits", kOptional)) return rc;
  if (int rc = check_shape(dlogits, "dlogits", logits->rows, logits->cols)) return rc;
  if (int rc = check_type(dlogits, "dlogits", logits->type)) return rc;
  if (targets_are64 != 0 && targets_are64 != 1) return fail(GOSH_EINVAL, "targets_are64 = %d: must be 0 or 1", targets_are64);
  const int64_t rows = logits->rows, size = targets_are64 ? 8 : 4;
  if (rows > 0) {
    if (targets == nullptr) return fail(GOSH_EINVAL, "targets is null");
    if (reinterpret_cast<uintptr_t>(targets) % size != 0) return fail(GOSH_EINVAL, "targets must be aligned to its entries");
    if (int rc = check_device_span(targets, static_cast<size_t>(rows * size), "targets")) return rc;
  }
  if (int rc = check_floats(weight, rows, "weight", true)) return rc;
  if (int rc = check_floats(loss, rows, "loss", false)) return rc;
  if (rows == 0) return GOSH_OK;
  LossArgs a{plane_of(logits), plane_of(dlogits), targets, weight, loss, rows, logits->cols, targets_are64, scale};
  hipStream_t st = as_stream(hip_stream);
  if (logits->type == GOSH_F32) return loss_of<F32>(a, st);
  if (logits->type == GOSH_BF16) return loss_of<Bf16>(a, st);
  return loss_of<F16>(a, st);
}

}  // extern "C"
