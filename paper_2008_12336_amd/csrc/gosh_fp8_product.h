// Matrix products in 8-bit floating point on the matrix cores: C (M x N) = sum over k of A(m, k) B(n, k), both with k along
// their rows.  One unit per type of the results.
#pragma once

#include <algorithm>

#include "gosh_fp8.h"

namespace gosh {

// ---- few results: the wavefronts of a workgroup share the blocks of k of 32 x 32 of them -----------------

// The rows of a tile that a lane reads; rows past the end read the last one's, for results that nobody stores.
struct Fp8Lane {
  const uint8_t *q, *e;
  int64_t step;
  __device__ __forceinline__ Fp8Lane(const Fp8Plane &p, int64_t row, int64_t rows) : step(p.step) {
    const int64_t r = row < rows ? row : rows - 1;
    q = p.data + r * p.ld + (threadIdx.x >> 5 & 1) * 32;
    e = p.exps + (r >> p.shift) * p.ld_exps;
  }
  // Block k: 32 bytes of each half.
  __device__ __forceinline__ uint32_t load(int64_t k, U4 (&v)[2][2]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i / 2][i % 2] = *reinterpret_cast<const U4 *>(q + k * step + i / 2 * 64 + i % 2 * 16);
    return e[k];
  }
};

// The same of a row that is put into 8 bits on the way, and stored if `keep`: block k's 128 entries are two lanes'.
template <typename X>
__device__ __forceinline__ uint32_t pack_block(const Fp8Args &a, int64_t row, int64_t k, bool keep, U4 (&v)[2][2]) {
  typedef typename X::Store S;
  const int64_t r = row < a.g.M ? row : a.g.M - 1;
  const int first = static_cast<int>(k) * kFp8Block + (threadIdx.x >> 5 & 1) * 32;  // column
  const S *const x = static_cast<const S *>(a.pack.data) + r * a.pack.ld + first;
  float f[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int left = a.pack_cols - first - (i / 4 * 64 + i % 4 * 8);
    Entries<X, 8>::load(x + i / 4 * 64 + i % 4 * 8, left < 0 ? 0 : left, f[i]);
  }
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[i][e] = __builtin_fabsf(f[i][e]) == INFINITY ? __uint_as_float(0x7fc00000u) : f[i][e];
      most = fmaxf(most, __builtin_fabsf(f[i][e]));
    }
  most = fmaxf(most, __shfl_xor(most, 32));
  const uint32_t byte = fp8_byte(__float_as_uint(most));
  const float inv = inverse_unit(byte);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i / 4][i / 2 % 2][i % 2 * 2] = to_e4m3(f[i][0], f[i][1], f[i][2], f[i][3], inv);
    v[i / 4][i / 2 % 2][i % 2 * 2 + 1] = to_e4m3(f[i][4], f[i][5], f[i][6], f[i][7], inv);
  }
  if (keep && row < a.g.M) {
    uint8_t *const to = const_cast<uint8_t *>(a.x.data) + row * a.x.ld + first;
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<U4 *>(to + i / 2 * 64 + i % 2 * 16) = v[i / 2][i % 2];
    if ((threadIdx.x & 32) == 0) const_cast<uint8_t *>(a.x.exps)[row * a.x.ld_exps + k] = static_cast<uint8_t>(byte);
  }
  return byte;
}

// A product of few results has few tiles, whose blocks of k one after the other are a chain of waits for memory: here four or 16
// wavefronts have a block each at a time, loaded by themselves.  (A training step of 512 x 256 -> 1024, products in tiles of 64 x
// 64: forward 7.8 us, dx 6.8, dw 5.4.)
// Products are exact whatever the type of the results: they are not what this waits for (1 x 512 -> 2048 in bf16 4.5 us and 4.6 with exact
// products, 64 x 4096 -> 4096 14.1 and 14.1, 512 x 256 -> 1024 5.3 and 5.4, its gradient 13.7 and 13.8).
// X: the type of the x, up to 32 rows, that is put into 8 bits on the way; or void.
template <int Waves>
struct FewLds {
  float parts[Waves - 1][16][64];
  float slab[Slab<32>::kFloats];
};
template <typename T, typename X, int Waves, ProductOut Out>
__device__ __forceinline__ void few_results(const Fp8Args &a, int64_t m0, int64_t n0, FewLds<Waves> &lds) {
  const ProductArgs &g = a.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const Fp8Lane x(a.x, m0 + (lane & 31), g.M), w(a.w, n0 + (lane & 31), g.N);
  F16x acc[1][1];
  float bias[1] = {0.f};
  if (wave == 0) load_bias<1, Out>(g, n0, bias);
  start<1, 1>(bias, acc);
  for (int64_t k = wave; k < g.K; k += Waves) {
    U4 qa[2][2], qb[2][2];
    const uint32_t ub = w.load(k, qb);
    uint32_t ua;
    if constexpr (std::is_void<X>::value) ua = x.load(k, qa);
    else ua = pack_block<X>(a, lane & 31, k, n0 == 0, qa);
#pragma unroll
    for (int h = 0; h < 2; ++h) acc[0][0] = fp8_mma<true>(qa[h], qb[h], ua, ub, acc[0][0]);
  }
  if (wave != 0) {
#pragma unroll
    for (int i = 0; i < 16; ++i) lds.parts[wave - 1][i][lane] = acc[0][0][i];
  }
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int s = 0; s < Waves - 1; ++s)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[0][0][i] += lds.parts[s][i][lane];
  finish<T, 1, 1, Out>(g, acc, lds.slab, m0, n0, 0);
}
template <typename T, typename X, int Waves, ProductOut Out>
__global__ __launch_bounds__(64 * Waves) void fp8_few_kernel(const Fp8Args a) {
  __shared__ __attribute__((aligned(16))) FewLds<Waves> lds;
  few_results<T, X, Waves, Out>(a, static_cast<int64_t>(blockIdx.y) * 32, static_cast<int64_t>(blockIdx.x) * 32, lds);
}

// dx, dw and the sums of db's parts of a small layer in one launch: the workgroups of each after the others'.  (A training step of
// 512 x 256 -> 1024 takes 55 us with a launch for each of the three, most of it the caller's.)
template <typename T, typename W, int Waves>
__global__ __launch_bounds__(64 * Waves) void fp8_few_gradients_kernel(const Fp8Args x, const Fp8Args w, const JoinJob db) {
  __shared__ __attribute__((aligned(16))) FewLds<Waves> lds;
  unsigned id = blockIdx.x;
  const unsigned of_x = static_cast<unsigned>(x.g.tiles_m) * x.g.tiles_n, of_w = static_cast<unsigned>(w.g.tiles_m) * w.g.tiles_n;
  if (id < of_x) {
    few_results<T, void, Waves, kStore>(x, id / x.g.tiles_n * int64_t{32}, id % x.g.tiles_n * int64_t{32}, lds);
    return;
  }
  id -= of_x;
  if (id < of_w) {
    few_results<W, void, Waves, kStore>(w, id / w.g.tiles_n * int64_t{32}, id % w.g.tiles_n * int64_t{32}, lds);
    return;
  }
  const int64_t i = (id - of_w) * int64_t{64 * Waves} + threadIdx.x;
  if (i >= db.n) return;
  float sum = 0.f;
#pragma unroll 8
  for (int s = 0; s < db.count; ++s) sum += db.parts[s * db.stride + i];
  static_cast<float *>(db.out)[i] = sum;
}
template <typename T, typename W>
int launch_fp8_few_gradients(const Fp8Args &x, const Fp8Args &w, const JoinJob &db, hipStream_t st) {
  const int waves = std::max(x.g.tiles_m > 0 ? few_waves(x.g.K) : 0, few_waves(w.g.K));
  const unsigned blocks = static_cast<unsigned>(x.g.tiles_m) * x.g.tiles_n + static_cast<unsigned>(w.g.tiles_m) * w.g.tiles_n +
                          static_cast<unsigned>(ceil_div(db.n, 64 * waves));
  if (waves == 4) fp8_few_gradients_kernel<T, W, 4><<<dim3(blocks), dim3(256), 0, st>>>(x, w, db);
  else fp8_few_gradients_kernel<T, W, 16><<<dim3(blocks), dim3(1024), 0, st>>>(x, w, db);
  return check_launch("gradients of a small layer in 8-bit floating point");
}

template <typename T, typename X, ProductOut Out>
int launch_fp8_few(const Fp8Args &a, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(ceil_div(a.g.N, 32)), static_cast<unsigned>(ceil_div(a.g.M, 32)));
  if (few_waves(a.g.K) == 4) fp8_few_kernel<T, X, 4, Out><<<grid, dim3(256), 0, st>>>(a);
  else fp8_few_kernel<T, X, 16, Out><<<grid, dim3(1024), 0, st>>>(a);
  return check_launch("product of few results in 8-bit floating point");
}
template <typename T, ProductOut Out>
int launch_fp8_few(const Fp8Args &a, hipStream_t st) {
  if constexpr (Out == kForward) {
    if (a.pack.data != nullptr && a.pack_type == GOSH_F32) return launch_fp8_few<T, F32, Out>(a, st);
    if (a.pack.data != nullptr && a.pack_type == GOSH_BF16) return launch_fp8_few<T, Bf16, Out>(a, st);
    if (a.pack.data != nullptr) return launch_fp8_few<T, F16, Out>(a, st);
  }
  return launch_fp8_few<T, void, Out>(a, st);
}

// ---- many tiles: straight to LDS ------------------------------------------------------------------------

// The range of memory that a wavefront's loads may touch, in scalar registers; the loads move along it.
struct Fp8Range {
  uint64_t base;
  uint32_t bytes;
  __device__ __forceinline__ U4 words() const {
    return U4{static_cast<uint32_t>(base), static_cast<uint32_t>(base >> 32) & 0xffffu, bytes, 0x00020000u};
  }
};
// m0, which the compiler sets, holds where the first lane's bytes land.  The compiler does not count the wait states of an
// instruction that it cannot see: s_nop 4 are the five that the load needs behind a vector instruction that wrote its range.
template <bool Dword>
__device__ __forceinline__ void load_to_lds(uint32_t off, const Fp8Range &r, uint32_t lds) {
  if constexpr (Dword)
    asm volatile("s_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" :: "v"(off), "s"(r.words()), "{m0}"(lds) : "memory");
  else
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" :: "v"(off), "s"(r.words()), "{m0}"(lds) : "memory");
}

// BX rows of an operand by 128 k, which the memory system writes to LDS by itself, 1 KB an instruction of a wavefront: the lanes
// ask for the chunks of 16 bytes that belong where theirs land.  Rows past the end read as zero.
template <int BX, int Waves>
struct Fp8Tile {
  static constexpr int kBytes = BX * kFp8Block, kLoads = kBytes / 1024 / Waves;
  Fp8Range range;
  uint32_t off[kLoads];
  __device__ __forceinline__ void init(const Fp8Plane &p) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = (static_cast<int>(threadIdx.x / 64) * kLoads + i) * 64 + (threadIdx.x & 63), row = at / 8, slot = at % 8;
      // the shifts are their own inverse
      off[i] = static_cast<uint32_t>(row) * static_cast<uint32_t>(p.ld) + Spread<BX, 64>::k_major(row, slot) / 8 % 8 * 16;
    }
  }
  // A block of the tile's rows: at most 256 rows of 2^23 bytes, 2^31.
  __device__ __forceinline__ void begin(const Fp8Plane &p, int64_t x, int64_t rows, int64_t k0) {
    range.base = reinterpret_cast<uint64_t>(p.data) + x * p.ld + k0 * p.step;
    const int64_t here = rows - x < BX ? rows - x : BX;
    range.bytes = static_cast<uint32_t>((here - 1) * p.ld + kFp8Block);
  }
  __device__ __forceinline__ void load(int i, uint32_t lds) const {
    load_to_lds<false>(off[i], range, lds + (__builtin_amdgcn_readfirstlane(threadIdx.x / 64) * kLoads + i) * 1024);
  }
};

// The exponents: a lane of the wavefront that has 64 rows of an operand loads four blocks' bytes of its row, which
// last for up to four steps.  64 rows of A for each of the first wavefronts, then of B; those that are left over load what the
// first ones do.
template <int BM, int BN, int Waves>
struct Fp8Units {
  static constexpr int kSlots = (BM + BN) / 64, kBytes = Waves * 256;
  static_assert(kSlots <= Waves, "a wavefront has one slot");
  Fp8Range range;
  uint32_t off;
  int block;  // of k

  __device__ __forceinline__ void begin(const Fp8Args &a, int64_t m0, int64_t n0, int64_t k0) {
    const int slot = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) % kSlots;
    const bool of_a = slot < BM / 64;
    const uint8_t *const exps = of_a ? a.x.exps : a.w.exps;
    const int64_t ld = of_a ? a.x.ld_exps : a.w.ld_exps, rows = of_a ? a.g.M : a.g.N;
    const int shift = of_a ? a.x.shift : a.w.shift;
    const int64_t row0 = of_a ? m0 + 64 * slot : n0 + 64 * (slot - BM / 64);
    const int64_t first = row0 >> shift, end = rows < row0 + 64 ? rows : row0 + 64;
    range.base = reinterpret_cast<uint64_t>(exps) + first * ld;
    range.bytes = end <= row0 ? 0 : static_cast<uint32_t>((((end - 1) >> shift) - first) * ld + (a.g.K + 3) / 4 * 4);
    off = static_cast<uint32_t>(((row0 + (threadIdx.x & 63)) >> shift) - first) * static_cast<uint32_t>(ld);
    block = static_cast<int>(k0);
  }
  __device__ __forceinline__ void load(uint32_t lds) const {
    load_to_lds<true>(off + (block & ~3), range, lds + __builtin_amdgcn_readfirstlane(threadIdx.x / 64) * 256);
  }
};

// n / d, and what is left, by d's reciprocal from the host: ceil(2^32 / d), or 2^32 - 1.  n < 2^31.
__device__ __forceinline__ int divided(int n, int d, uint32_t reciprocal, int *rest) {
  int q = static_cast<int>(__umulhi(static_cast<uint32_t>(n), reciprocal));  // right, or 1 too much; for d = 1 also 1 less
  int r = n - q * d;
  if (r < 0) --q, r += d;
  if (r >= d) ++q, r -= d;
  *rest = r;
  return q;
}

// The id-th tile: of eight rows of tiles those of one column after each other, then the next column's, so that the 32 CUs
// of an XCD, which work on 32 tiles in a row, share eight tiles of A and four of B: of 131,072 x 1024 -> 4096 those of B alone, 4
// MB, fill an L2, and with row after row they were fetched again and again (727 -> 697 us).
__device__ __forceinline__ Place fp8_place(const Fp8Args &a, int id, int bm, int bn) {
  const ProductArgs &g = a.g;
  const int all = g.tiles_m * g.tiles_n;
  int rest = id, split = 0, in;
  if (g.splits > 1) split = divided(id, all, a.by_all, &rest);
  const int first = divided(rest, kTileGroup * g.tiles_n, a.by_group, &in) * kTileGroup;
  const int tall = g.tiles_m - first < kTileGroup ? g.tiles_m - first : kTileGroup;
  const int tn = tall == kTileGroup ? in / kTileGroup : in / tall, tm = first + in - tn * tall;
  const int64_t k0 = split * g.k_per_split;
  return {static_cast<int64_t>(tm) * bm, static_cast<int64_t>(tn) * bn, k0, k0 + g.k_per_split < g.K ? k0 + g.k_per_split : g.K, split};
}

// Two tiles in LDS: while a step is multiplied the next one's loads are under way, also across the end of a tile: a workgroup
// goes from tile to tile.  Rows of 128 bytes lie as those of 64 entries of 16 bits do.  A wavefront multiplies 32 rows by 64
// k at a time, while the next such rows of A (and, before the second half of a step, B's) are read from LDS.
//
// 16,384 x 8192 -> 4096 takes 437 us, 2.5 PFLOP/s (the matrix cores are busy 63 % of it; the vendor's product with a single
// scale 416), and 427 without the results' way to memory.  131,072 x 1024 -> 4096 takes 540 to 605 (52 %; 519), of which 495 are left
// without that: 1.07 GB of results need 155 at the rate of a fill, and the next tile's second step waits behind them.
template <typename T, int BM, int BN, bool Exact, ProductOut Out>
__global__ __launch_bounds__(64 * direct_waves(BN), 8 / direct_waves(BN)) void fp8_product_kernel(const Fp8Args args) {
  constexpr int kWaves = direct_waves(BN), kAcross = kWaves / 2;
  typedef Fp8Tile<BM, kWaves> TA;
  typedef Fp8Tile<BN, kWaves> TB;
  typedef Fp8Units<BM, BN, kWaves> Units;
  constexpr int WM = BM / 2, WN = BN / kAcross, RM = WM / 32, RN = WN / 32;
  constexpr int kStep = TA::kBytes + TB::kBytes, kLoads = TA::kLoads + TB::kLoads;
  __shared__ __attribute__((aligned(1024))) uint16_t lds[(2 * kStep + 2 * Units::kBytes) / 2];
  __shared__ __attribute__((aligned(16))) float slabs[kWaves * Slab<WN>::kFloats];

  const ProductArgs &g = args.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wm = wave / kAcross * WM, wn = wave % kAcross * WN;
  const Turns turns = turns_of(g.tiles_m * g.tiles_n * g.splits);
  if (turns.id >= turns.end) return;

  const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint16_t *)lds));
  TA a;
  TB b;
  Units units;
  a.init(args.x);
  b.init(args.w);
  uint32_t into = base;
  // exponents go to their two places in turns: a place is written again only a whole step after it was read last
  uint32_t units_into = base + 2 * kStep, units_from = units_into;
  int turn = turns.id, to_go;
  Place from;  // of the tile that is being loaded
  bool units_next;  // the step that is loaded next needs other exponents
  const auto begin = [&]() {
    from = fp8_place(args, turn, BM, BN);
    a.begin(args.x, from.m0, g.M, from.k0);
    b.begin(args.w, from.n0, g.N, from.k0);
    units.begin(args, from.m0, from.n0, from.k0);
    to_go = static_cast<int>(from.k1 - from.k0);
    units_next = true;
  };
  // On to the step after: the next of the tile, or the first of the next tile, or none, whose loads read nothing.
  const auto advance = [&]() {
    into = into == base ? base + kStep : base;
    a.range.base += args.x.step;
    b.range.base += args.w.step;
    units_next = (++units.block & 3) == 0;
    if (--to_go > 0) return;
    turn += turns.step;
    if (turn < turns.end) begin();
    else a.range.bytes = b.range.bytes = units.range.bytes = 0, to_go = 0x7fffffff;
  };
  const auto load = [&]() {
#pragma unroll
    for (int i = 0; i < TA::kLoads; ++i) a.load(i, into);
#pragma unroll
    for (int i = 0; i < TB::kLoads; ++i) b.load(i, into + TA::kBytes);
    if (units_next) {
      units.load(units_into);
      units_from = units_into;
      units_into = units_into == base + 2 * kStep ? units_into + Units::kBytes : base + 2 * kStep;
    }
  };
  begin();
  load();
  const uint32_t units_first = units_from;
  float bias[RN];
  load_bias<RN, Out>(g, from.n0 + wn, bias);
  bool ahead = to_go > 1;  // two steps are under way before the first
  if (ahead) {
    advance();
    load();
  }

  const uint16_t *now = lds;
  U4 fa[2][2], fb[2][RN][2];  // 32 rows by 64 k: the ones in work and the next
  uint32_t ea[2][RM], eb[2][RN];
  const auto take_a = [&](int to, int i, int half) {
#pragma unroll
    for (int c = 0; c < 2; ++c) fa[to][c] = __builtin_bit_cast(U4, Spread<BM, 64>::template take<true>(now, wm + 32 * i, 2 * half + c));
  };
  const auto take_b = [&](int half) {
#pragma unroll
    for (int j = 0; j < RN; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        fb[half][j][c] = __builtin_bit_cast(U4, Spread<BN, 64>::template take<true>(now + TA::kBytes / 2, wn + 32 * j, 2 * half + c));
  };
  const auto take_units = [&](uint32_t where, uint32_t (&x)[RM], uint32_t (&w)[RN]) {
    const uint32_t *const e = reinterpret_cast<const uint32_t *>(lds + (where - base) / 2);
#pragma unroll
    for (int i = 0; i < RM; ++i) x[i] = e[wm + 32 * i + (lane & 31)];
#pragma unroll
    for (int j = 0; j < RN; ++j) w[j] = e[BM + wn + 32 * j + (lane & 31)];
  };
  // all but the loads of the second step, of which there are kLoads or, with its exponents, one more
  if (ahead) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(kLoads) : "memory");
  else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  take_units(units_first, ea[0], eb[0]);
  take_b(0);
  take_a(0, 0, 0);
  for (int id = turns.id; id < turns.end; id += turns.step) {
    const Place at = from;
    const int steps = static_cast<int>(at.k1 - at.k0);
    F16x acc[RM][RN];
    start<RM, RN>(bias, acc);
    for (int s = 0; s < steps; ++s) {
      // before the products: the compiler would move them behind the branches
      if (!ahead) {
        advance();
        if (is_forward(Out) && s + 1 == steps) load_bias<RN, Out>(g, from.n0 + wn, bias);  // the next tile's, or this one's again
        load();
      }
      ahead = false;
      const int shift = (static_cast<int>(at.k0) + s & 3) * 8;
#pragma unroll
      for (int i = 0; i < RM; ++i) ea[1][i] = ea[0][i] >> shift & 255u;
#pragma unroll
      for (int j = 0; j < RN; ++j) eb[1][j] = eb[0][j] >> shift & 255u;
      const auto multiply = [&](int from, int i, int half) {
#pragma unroll
        for (int j = 0; j < RN; ++j) acc[i][j] = fp8_mma<Exact>(fa[from], fb[half][j], ea[1][i], eb[1][j], acc[i][j]);
      };
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
      take_units(units_from, ea[0], eb[0]);
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
  if constexpr (Size == kLarge && Out == kForward)
    if (a.g.forward.past)
      return a.g.forward.z.data == nullptr ? launch_fp8_tiles<T, Size, Exact, kPast>(a, st) : launch_fp8_tiles<T, Size, Exact, kPastZ>(a, st);
  const unsigned blocks = static_cast<unsigned>(a.g.tiles_m) * a.g.tiles_n * a.g.splits;
  const unsigned held = static_cast<unsigned>(resident_waves()) / 4 / kWaves;  // eight wavefronts a CU
  fp8_product_kernel<T, kTile, kTile, Exact, Out><<<dim3(blocks < held ? blocks : held), dim3(64 * kWaves), 0, st>>>(a);
  return check_launch("product in 8-bit floating point");
}

template <typename T, bool Exact, ProductOut Out>
int launch_fp8_out(const Fp8Args &a, hipStream_t st) {
  if constexpr (!Exact || Out != kForward) {  // see fp8_time
    if (a.tile == 256) return launch_fp8_tiles<T, kLarge, Exact, Out>(a, st);
  } else if (a.tile == 256) {
    return fail(GOSH_EINVAL, "no exact forward products in tiles of 256");
  }
  if (a.tile == 128) return launch_fp8_tiles<T, kMiddle, Exact, Out>(a, st);
  if constexpr (Out != kParts)
    if (a.tile == 32) return launch_fp8_few<T, Out>(a, st);
  return launch_fp8_tiles<T, kSmall, Exact, Out>(a, st);
}

template <typename T>
int launch_fp8_any(ProductOut out, const Fp8Args &a, hipStream_t st) {
  constexpr bool exact = T::kType != GOSH_BF16;
  if (out == kForward) return a.exact ? launch_fp8_out<T, true, kForward>(a, st) : launch_fp8_out<T, exact, kForward>(a, st);
  if (out == kStore) return a.exact ? launch_fp8_out<T, true, kStore>(a, st) : launch_fp8_out<T, exact, kStore>(a, st);
  if constexpr (T::kType != GOSH_F16) return launch_fp8_out<T, exact, kParts>(a, st);
  return fail(GOSH_EINVAL, "parts are of F32 or Bf16");
}

}  // namespace gosh
