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

template <typename T, bool Exact, ProductOut Out>
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
    for (int h = 0; h < 2; ++h) acc[0][0] = fp8_mma<Exact>(qa[h], qb[h], ua, ub, acc[0][0]);
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

// ---- many tiles: straight to LDS ------------------------------------------------------------------------

// The exponents of a step: a lane of the wavefront that has 64 rows of an operand loads four blocks' bytes of its row
// straight to LDS, of which a step takes one.  64 rows of A for each of the first wavefronts, then of B; those that are left
// over load what the first ones do, so that all have as many loads under way.
template <int BM, int BN, int Waves>
struct Fp8Units {
  static constexpr int kSlots = (BM + BN) / 64, kBytes = Waves * 256;
  static_assert(kSlots <= Waves, "a wavefront has one slot");
  uint64_t base;
  int64_t bytes, left;   // of the matrix's exponents from base on; blocks of k up to the row's end
  uint32_t off;
  int block;             // of k, the next to load

  __device__ __forceinline__ void begin(const Fp8Args &a, int64_t m0, int64_t n0, int64_t k0) {
    const int slot = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) % kSlots;
    const bool of_a = slot < BM / 64;
    const Fp8Plane &p = of_a ? a.x : a.w;
    const int64_t rows = of_a ? a.g.M : a.g.N, row0 = of_a ? m0 + 64 * slot : n0 + 64 * (slot - BM / 64);
    const int64_t first = row0 >> p.shift, last = (rows - 1) >> p.shift;
    base = reinterpret_cast<uint64_t>(p.exps) + first * p.ld_exps;
    bytes = (last - first) * p.ld_exps + (a.g.K + 3) / 4 * 4;
    off = static_cast<uint32_t>((((row0 + (threadIdx.x & 63)) >> p.shift) - first) * p.ld_exps);
    block = static_cast<int>(k0);
  }
  __device__ __forceinline__ void fetch(uint32_t lds) {
    const U4 range{static_cast<uint32_t>(base), static_cast<uint32_t>(base >> 32) & 0xffffu,
                   static_cast<uint32_t>(bytes <= 0 ? 0 : bytes > 0x7fffffff ? 0x7fffffff : bytes), 0x00020000u};
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t o = off + (block & ~3);
    // as the loads of the tiles
    asm volatile("s_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" :: "v"(o), "s"(range), "{m0}"(lds + wave * 256) : "memory");
    ++block;
  }
};

// A ring of two tiles of 128 k, as the products in 16 bits have it: rows of 128 bytes lie in LDS as theirs of 64 entries do.
// A wavefront multiplies 32 rows by 64 k at a time, while the next such rows of A (and, before the second half of a step, B's) are
// read from LDS.
template <typename T, int BM, int BN, bool Exact, ProductOut Out>
__global__ __launch_bounds__(64 * direct_waves(BN), 8 / direct_waves(BN)) void fp8_product_kernel(const Fp8Args args) {
  constexpr int kWaves = direct_waves(BN), kAcross = kWaves / 2;
  constexpr int kHalf = kFp8Block / 2;  // k of a step in the 16-bit units of the tiles
  typedef DirectTile<BM, kHalf, true, kWaves> TA;
  typedef DirectTile<BN, kHalf, true, kWaves> TB;
  typedef Fp8Units<BM, BN, kWaves> Units;
  constexpr int WM = BM / 2, WN = BN / kAcross, RM = WM / 32, RN = WN / 32, kRing = 2;
  constexpr int kStep = TA::kBytes + TB::kBytes + Units::kBytes;
  __shared__ __attribute__((aligned(1024))) uint16_t lds[kRing * kStep / 2];
  __shared__ __attribute__((aligned(16))) float slabs[kWaves * Slab<WN>::kFloats];

  const ProductArgs &g = args.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wm = wave / kAcross * WM, wn = wave % kAcross * WN;
  const Turns turns = turns_of(g.tiles_m * g.tiles_n * g.splits);
  if (turns.id >= turns.end) return;
  const Plane pa{const_cast<uint8_t *>(args.x.data), nullptr, args.x.ld / 2, 0}, pb{const_cast<uint8_t *>(args.w.data), nullptr, args.w.ld / 2, 0};

  const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint16_t *)lds));
  TA a;
  TB b;
  Units units;
  a.init(pa);
  b.init(pb);
  // The loads run ahead of the computation, over tiles; after the last tile they load nothing.
  uint32_t into = base;
  int turn = turns.id;
  int to_go;
  const auto begin = [&]() {
    const Place from = place_of(g, turn, BM, BN);
    a.begin(pa, from.m0, g.M, from.k0 * kHalf, from.k1 * kHalf);
    b.begin(pb, from.n0, g.N, from.k0 * kHalf, from.k1 * kHalf);
    units.begin(args, from.m0, from.n0, from.k0);
    to_go = static_cast<int>(from.k1 - from.k0);
  };
  const auto fetch = [&]() {
    a.fetch(pa, into);
    b.fetch(pb, into + TA::kBytes);
    units.fetch(into + TA::kBytes + TB::kBytes);
    into = into == base ? base + kStep : base;
    if (--to_go <= 0 && turn + turns.step < turns.end) {
      turn += turns.step;
      begin();
    }
  };
  begin();
  fetch();

  const uint16_t *now = lds;
  U4 fa[2][2], fb[2][RN][2];  // 32 rows by 64 k: the ones in work and the next
  uint32_t ea[RM], eb[RN];
  const auto take_a = [&](int to, int i, int half) {
#pragma unroll
    for (int c = 0; c < 2; ++c) fa[to][c] = __builtin_bit_cast(U4, Spread<BM, kHalf>::template take<true>(now, wm + 32 * i, 2 * half + c));
  };
  const auto take_b = [&](int half) {
#pragma unroll
    for (int j = 0; j < RN; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        fb[half][j][c] = __builtin_bit_cast(U4, Spread<BN, kHalf>::template take<true>(now + TA::kBytes / 2, wn + 32 * j, 2 * half + c));
  };
  const auto take_units = [&](int block) {
    const uint32_t *const e = reinterpret_cast<const uint32_t *>(now + (TA::kBytes + TB::kBytes) / 2);
    const int shift = (block & 3) * 8;
#pragma unroll
    for (int i = 0; i < RM; ++i) ea[i] = e[wm + 32 * i + (lane & 31)] >> shift & 255u;
#pragma unroll
    for (int j = 0; j < RN; ++j) eb[j] = e[BM + wn + 32 * j + (lane & 31)] >> shift & 255u;
  };
  float bias[RN];
  load_bias<RN, Out>(g, place_of(g, turns.id, BM, BN).n0 + wn, bias);
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  take_b(0);
  take_a(0, 0, 0);
  for (int id = turns.id; id < turns.end; id += turns.step) {
    const Place at = place_of(g, id, BM, BN);
    const int steps = static_cast<int>(at.k1 - at.k0);
    F16x acc[RM][RN];
    start<RM, RN>(bias, acc);
    if (is_forward(Out) && id + turns.step < turns.end)
      load_bias<RN, Out>(g, place_of(g, id + turns.step, BM, BN).n0 + wn, bias);
    const auto multiply = [&](int from, int i, int half) {
#pragma unroll
      for (int j = 0; j < RN; ++j) acc[i][j] = fp8_mma<Exact>(fa[from], fb[half][j], ea[i], eb[j], acc[i][j]);
    };
    for (int s = 0; s < steps; ++s) {
      // Before the products, since there is a branch in it: the compiler would move the products behind it.
      fetch();
      take_units(static_cast<int>(at.k0) + s);
      constexpr int kTurns = 2 * RM;  // 32 rows by 64 k each
#pragma unroll
      for (int t = 0; t + 1 < kTurns; ++t) {
        if (t + 1 == RM) take_b(1);
        take_a((t + 1) & 1, (t + 1) % RM, (t + 1) / RM);
        __builtin_amdgcn_sched_barrier(0);
        multiply(t & 1, t % RM, t / RM);
        __builtin_amdgcn_sched_barrier(0);
      }
      // The next step's tile is there, every wavefront's part of it, and every wavefront is done with this step's.
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      now = now == lds ? lds + kStep / 2 : lds;
      take_b(0);
      take_a(0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      multiply((kTurns - 1) & 1, RM - 1, 1);
    }
    // the next tile's bias is waited for here, before the stores: after them it would wait for those too
#pragma unroll
    for (int j = 0; j < RN; ++j) asm volatile("" : "+v"(bias[j]));
    finish<T, RM, RN, Out>(g, acc, slabs + wave * Slab<WN>::kFloats, at.m0 + wm, at.n0 + wn, at.split);
  }
  // no load may land in LDS that is another workgroup's by then
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <typename T, TileSize Size, bool Exact, ProductOut Out>
int launch_fp8_tiles(const Fp8Args &a, hipStream_t st) {
  constexpr int kTile = tile_m(Size), kWaves = direct_waves(kTile);
  const unsigned blocks = static_cast<unsigned>(a.g.tiles_m) * a.g.tiles_n * a.g.splits;
  const unsigned held = static_cast<unsigned>(resident_waves()) / 4 / kWaves;  // eight wavefronts a CU
  fp8_product_kernel<T, kTile, kTile, Exact, Out><<<dim3(blocks < held ? blocks : held), dim3(64 * kWaves), 0, st>>>(a);
  return check_launch("product in 8-bit floating point");
}

template <typename T, bool Exact, ProductOut Out>
int launch_fp8_out(const Fp8Args &a, hipStream_t st) {
  switch (a.tile) {
    case 256: return launch_fp8_tiles<T, kLarge, Exact, Out>(a, st);
    case 128: return launch_fp8_tiles<T, kMiddle, Exact, Out>(a, st);
    case 64: return launch_fp8_tiles<T, kSmall, Exact, Out>(a, st);
    default: break;
  }
  const unsigned blocks = static_cast<unsigned>(a.g.tiles_m) * a.g.tiles_n * a.g.splits;
  fp8_small_kernel<T, Exact, Out><<<dim3(blocks), dim3(256), 0, st>>>(a);
  return check_launch("product in 8-bit floating point");
}

template <typename T>
int launch_fp8_any(ProductOut out, const Fp8Args &a, hipStream_t st) {
  constexpr bool exact = T::kType != GOSH_BF16;
  if (out == kForward) return a.exact ? launch_fp8_out<T, true, kForward>(a, st) : launch_fp8_out<T, exact, kForward>(a, st);
  if (out == kStore) return launch_fp8_out<T, exact, kStore>(a, st);
  if constexpr (T::kType != GOSH_F16) return launch_fp8_out<T, exact, kParts>(a, st);
  return fail(GOSH_EINVAL, "parts are of F32 or Bf16");
}

}  // namespace gosh
