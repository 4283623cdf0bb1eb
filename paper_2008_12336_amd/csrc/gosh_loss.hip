// Softmax cross-entropy of rows of logits, with its gradient.
//
// A row stays in the registers of the lanes that share it, from one lane to a workgroup of 1,024 (65,536
// entries in 32 bits), so that logits are read once and the gradient is written once: bound by memory.  Each lane subtracts
// the row's maximum (joined over the lanes first), keeps e = exp(x - max), and the lanes join the sum of e:
//   loss = log(sum) + (max - x[target]),  gradient = scale weight (e / sum - [class = target]).
// 65,536 x 4096 in bf16 takes 183 us (5.9 TB/s), 4,096 x 50,000 180, 300,007 x 47 in f32 22 (5.1, partly from the caches).
#include <algorithm>

#include "gosh_head.h"

namespace gosh {
namespace {

struct LossArgs {
  Plane x, d;
  const void *targets;
  const float *weight;
  float *loss;
  int64_t rows, first;  // first: of the launch
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
// + l) * E.  At most one chunk of a row is there in part: it is loaded and stored by itself, once.
template <typename T, int Lanes, int Count>
__global__ __launch_bounds__(Lanes > 256 ? Lanes : 256) void loss_kernel(const LossArgs a) {
  constexpr int E = T::kType == GOSH_F32 ? 4 : 8;
  constexpr int kThreads = Lanes > 256 ? Lanes : 256, kRows = kThreads / Lanes, kWaves = Lanes / 64;
  typedef typename T::Store S;
  typedef typename Entries<T, E>::Vec Vec;
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
  const int64_t row = a.first + static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / Lanes;
  const bool there = row < a.rows;
  int64_t target = -1;
  float weight = 1.f;
  if (there) {
    target = a.targets_are64 ? static_cast<const int64_t *>(a.targets)[row] : static_cast<const int32_t *>(a.targets)[row];
    if (a.weight != nullptr) weight = a.weight[row];
  }
  const bool wrong = target >= a.cols;
  const S *const x = static_cast<const S *>(a.x.data) + row * a.x.ld;
  const int whole_chunks = a.cols / E, over = a.cols % E;
  const int part_count = whole_chunks / Lanes;  // which of a lane's chunks is the one that is there in part, if it is its own
  const bool part = there && over != 0 && lane == whole_chunks % Lanes;
  Vec raw[Count], rest = 0;
#pragma unroll
  for (int c = 0; c < Count; ++c) {
    raw[c] = 0;
    if (there && c * Lanes + lane < whole_chunks) raw[c] = Entries<T, E>::fetch(x + (c * Lanes + lane) * E, E);
  }
  if (part) rest = Entries<T, E>::fetch(x + whole_chunks * E, over);
  // the target's logit: a load of its own is cheaper than to compare every column
  float hit = target < 0 || wrong ? 0.f : T::up(x[target]);
  asm volatile("" : "+v"(hit));  // here by now: another wavefront may write the gradient over it as soon as all have joined
  float v[Count][E], most = -INFINITY;
#pragma unroll
  for (int c = 0; c < Count; ++c) {
    const bool mine = part && c == part_count, none = !mine && c * Lanes + lane >= whole_chunks;
#pragma unroll
    for (int e = 0; e < E; ++e) v[c][e] = T::up(raw[c][e]);
    if (mine) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[c][e] = e < over ? T::up(rest[e]) : -INFINITY;
    }
    if (none) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[c][e] = -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) most = larger(most, v[c][e]);
  }
  most = join(most, 0, larger);
  const bool nothing = target < 0 || weight == 0.f || most == -INFINITY;
  const float from = nothing ? 0.f : most;
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < Count; ++c)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      v[c][e] = __expf(v[c][e] - from);
      sum += v[c][e];
    }
  sum = join(sum, 1, [](float p, float q) { return p + q; });
  if (!there) return;
  const float nan = __uint_as_float(0x7fc00000u);
  if (lane == 0) a.loss[row] = nothing ? 0.f : wrong ? nan : weight * (logf(sum) + (most - hit));
  if (a.d.data == nullptr) return;
  const float whole = a.scale * weight, share = wrong ? nan : whole / sum;
  S *const d = static_cast<S *>(a.d.data) + row * a.d.ld;
  float last[E];
#pragma unroll
  for (int e = 0; e < E; ++e) last[e] = 0.f;
#pragma unroll
  for (int c = 0; c < Count; ++c) {
    const int at = (c * Lanes + lane) * E;
#pragma unroll
    for (int e = 0; e < E; ++e) v[c][e] *= share;
    const int here = static_cast<int>(target) - at;  // a target past the columns has NaN everywhere
    if (static_cast<unsigned>(here) < static_cast<unsigned>(E)) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[c][e] -= e == here ? whole : 0.f;
    }
    if (nothing) {  // whatever the row holds, NaN also
#pragma unroll
      for (int e = 0; e < E; ++e) v[c][e] = 0.f;
    }
    if (c == part_count) {
#pragma unroll
      for (int e = 0; e < E; ++e) last[e] = v[c][e];
    }
    if (c * Lanes + lane < whole_chunks) Entries<T, E>::store(d + at, E, v[c]);
  }
  if (part) Entries<T, E>::store(d + whole_chunks * E, over, last);
}

template <typename T, int Lanes, int Count>
int launch_loss(LossArgs a, hipStream_t st) {
  constexpr int kThreads = Lanes > 256 ? Lanes : 256, kRows = kThreads / Lanes;
  constexpr int64_t kBlocks = int64_t{1} << 20;  // a grid's threads stay below 2^31
  for (a.first = 0; a.first < a.rows; a.first += kBlocks * kRows) {
    const unsigned blocks = static_cast<unsigned>(std::min(ceil_div(a.rows - a.first, kRows), kBlocks));
    loss_kernel<T, Lanes, Count><<<dim3(blocks), dim3(kThreads), 0, st>>>(a);
    if (int rc = check_launch("softmax loss")) return rc;
  }
  return GOSH_OK;
}

template <typename T>
int loss_of(const LossArgs &a, hipStream_t st) {
  constexpr int E = T::kType == GOSH_F32 ? 4 : 8;
  const int64_t chunks = ceil_div(a.cols, E);
  // Few lanes with several chunks each: 300,007 x 47 in f32 takes 21.9 us with 8 lanes and 28.1 with 16, 2^21 x 16 in bf16 27
  // with one lane, 34 with two and 52 with four.
  if (chunks <= 1) return launch_loss<T, 1, 1>(a, st);
  if (chunks <= 2) return launch_loss<T, 1, 2>(a, st);
  if (chunks <= 4) return launch_loss<T, 2, 2>(a, st);
  if (chunks <= 8) return launch_loss<T, 4, 2>(a, st);
  if (chunks <= 16) return launch_loss<T, 8, 2>(a, st);
  if (chunks <= 32) return launch_loss<T, 8, 4>(a, st);
  if (chunks <= 64) return launch_loss<T, 16, 4>(a, st);
  if (chunks <= 128) return launch_loss<T, 32, 4>(a, st);
  if (chunks <= 256) return launch_loss<T, 64, 4>(a, st);
  if (chunks <= 512) return launch_loss<T, 256, 2>(a, st);
  if (chunks <= 768) return launch_loss<T, 256, 3>(a, st);
  if (chunks <= 1024) return launch_loss<T, 256, 4>(a, st);
  if (chunks <= 1536) return launch_loss<T, 512, 3>(a, st);
  if (chunks <= 2048) return launch_loss<T, 512, 4>(a, st);
  // Three chunks a lane: 8,192 x 20,000 in bf16 115 us, 122 with four; near a full third it gains little (24,000: 133 and
  // 137) or loses (12,000 in f32: 135 and 133).
  if (chunks <= 2800) return launch_loss<T, 1024, 3>(a, st);
  if (chunks <= 4096) return launch_loss<T, 1024, 4>(a, st);
  if (chunks <= 6144) return launch_loss<T, 1024, 6>(a, st);
  if (chunks <= 8192) return launch_loss<T, 1024, 8>(a, st);
  if constexpr (T::kType == GOSH_F32) {
    if (chunks <= 12288) return launch_loss<T, 1024, 12>(a, st);
    return launch_loss<T, 1024, 16>(a, st);
  }
  return fail(GOSH_EINVAL, "logits: cols = %d: too many", a.cols);
}

// Two matrices of one shape and type that are one, or have no entry in common.  (A row of one that lies on another row of the other
// would be written before it is read.)
bool same_or_apart(const gosh_mat &a, const gosh_mat &b) {
  if (a.rows == 0) return true;
  if (a.data == b.data) return a.ld == b.ld || a.rows == 1;
  const bool a_first = reinterpret_cast<uintptr_t>(a.data) < reinterpret_cast<uintptr_t>(b.data);
  const gosh_mat &low = a_first ? a : b, &high = a_first ? b : a;
  const int64_t size = a.type == GOSH_F32 ? 4 : 2;
  const uint64_t bytes = reinterpret_cast<uintptr_t>(high.data) - reinterpret_cast<uintptr_t>(low.data);
  const int64_t span = (low.rows - 1) * low.ld + low.cols;
  if (bytes >= static_cast<uint64_t>(span * size)) return true;
  if (a.ld != b.ld && a.rows > 1) return false;
  const int64_t entries = static_cast<int64_t>(bytes) / size, row = entries / low.ld, col = entries % low.ld;  // where high begins in low
  return col >= low.cols && (row + 1 >= low.rows || low.ld - col >= low.cols);
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
  if (dlogits != nullptr && !same_or_apart(*logits, *dlogits))
    return fail(GOSH_EINVAL, "dlogits overlaps logits: it must be logits, or have no entry of it");
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
  LossArgs a{plane_of(logits), plane_of(dlogits), targets, weight, loss, rows, 0, logits->cols, targets_are64, scale};
  hipStream_t st = as_stream(hip_stream);
  if (logits->type == GOSH_F32) return loss_of<F32>(a, st);
  if (logits->type == GOSH_BF16) return loss_of<Bf16>(a, st);
  return loss_of<F16>(a, st);
}

}  // extern "C"
