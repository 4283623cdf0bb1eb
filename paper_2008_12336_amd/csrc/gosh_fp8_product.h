// Matrix products in 8-bit floating point on the matrix cores: C (M x N) = sum over k of A(m, k) B(n, k), both with k along
// their rows.  One unit per type of the results.
#pragma once

#include "gosh_fp8.h"

namespace gosh {

// ---- a few tiles: four wavefronts share the blocks of k of 32 x 32 results ----------------------------

// The rows of a tile that a lane reads; rows past the end read the last one's, for results that nobody stores.
struct Fp8Lane {
  const uint8_t *q, *e;
  __device__ __forceinline__ Fp8Lane(const Fp8Plane &p, int64_t row, int64_t rows) {
    const int64_t r = row < rows ? row : rows - 1;
    q = p.data + r * p.ld + (threadIdx.x >> 5 & 1) * 32;
    e = p.exps + (r >> p.shift) * p.ld_exps;
  }
};

template <typename T, ProductOut Out>
__global__ __launch_bounds__(256) void fp8_small_kernel(const Fp8Args a) {
  __shared__ __attribute__((aligned(16))) float lds[3][16][64];
  __shared__ __attribute__((aligned(16))) float slab[Slab<32>::kFloats];
  const ProductArgs &g = a.g;
  const Place at = place_of(g, static_cast<int>(blockIdx.x), 32, 32);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const Fp8Lane x(a.x, at.m0 + (lane & 31), g.M), w(a.w, at.n0 + (lane & 31), g.N);
  F16x acc[1][1];
  float bias[1] = {0.f};
  if (wave == 0) load_bias<1, Out>(g, at.n0, bias);
  start<1, 1>(bias, acc);
  for (int64_t k = at.k0 + wave; k < at.k1; k += 4) {
    U4 qa[2][2], qb[2][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t off = k * kFp8Block + i / 2 * 64 + i % 2 * 16;
      qa[i / 2][i % 2] = *reinterpret_cast<const U4 *>(x.q + off);
      qb[i / 2][i % 2] = *reinterpret_cast<const U4 *>(w.q + off);
    }
    const uint32_t ua = x.e[k], ub = w.e[k];
#pragma unroll
    for (int h = 0; h < 2; ++h) acc[0][0] = fp8_mma<T::kType == GOSH_F32>(qa[h], qb[h], ua, ub, acc[0][0]);
  }
  if (wave != 0) {
#pragma unroll
    for (int i = 0; i < 16; ++i) lds[wave - 1][i][lane] = acc[0][0][i];
  }
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int s = 0; s < 3; ++s)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[0][0][i] += lds[s][i][lane];
  finish<T, 1, 1, Out>(g, acc, slab, at.m0, at.n0, at.split);
}

template <typename T, ProductOut Out>
int launch_fp8_out(const Fp8Args &a, hipStream_t st) {
  const unsigned blocks = static_cast<unsigned>(a.g.tiles_m) * a.g.tiles_n * a.g.splits;
  fp8_small_kernel<T, Out><<<dim3(blocks), dim3(256), 0, st>>>(a);
  return check_launch("product in 8-bit floating point");
}

template <typename T>
int launch_fp8_any(ProductOut out, const Fp8Args &a, hipStream_t st) {
  if (out == kForward) return launch_fp8_out<T, kForward>(a, st);
  if (out == kStore) return launch_fp8_out<T, kStore>(a, st);
  if constexpr (T::kType != GOSH_F16) return launch_fp8_out<T, kParts>(a, st);
  return fail(GOSH_EINVAL, "parts are of F32 or Bf16");
}

}  // namespace gosh
