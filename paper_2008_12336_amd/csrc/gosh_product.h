// Tiled matrix products of the linear layer on the matrix cores, one unit per element type.
//
// C (M x N) = sum over k of A(m, k) B(n, k).  An operand lies in memory either with k along its rows ("k-major": x and w
// of the forward pass, dz of dx) or with k across them ("m-major": w of dx, dz and x of dw, where k counts rows of the
// batch).  Both are staged through LDS in 16-bit entries: k-major tiles are read 8 k at a time, m-major ones through the
// transposing read (16 lanes fetch 4 rows of 16 entries and get 4 entries of one column each), so that no operand is
// transposed in memory.
//
// Three ways, all ending in the same epilogue.  Aligned 16-bit rows go straight to LDS, in tiles of 256 x 256 by eight
// wavefronts where there are enough: 65,536 x 512 x 2048 takes 137 to 150 us (0.9 to 1.0 PFLOP/s; a large product of the
// vendor's library reaches 1.33; the matrix cores are busy 48 % of it in dx, 55 % in dw), and with K = 512, where the
// epilogue counts, 262,144 x 512 -> 2048 625 to 652 us without and 700 to 740 with GELU (38 %).  There, by the times for K
// from 64 to 512, each tile costs 14 to 15 us of products and then, since the eight wavefronts go through it together, 4 to
// 6 of epilogue, 7 to 9 with GELU; its stores alone need 4.9 at the rate of a fill.  One instruction in six less,
// workgroups that start at different times, rows of 256 bytes and rows fetched from LDS ahead of the stores changed
// nothing; tiles of 128 x 128, two workgroups to a CU, which do overlap both, lose more to fetching (914 us).  Other
// tiles pass through registers on their way to LDS (32-bit entries, odd strides): 65,536 x 1024 -> 1024 in f32 takes
// 735 us, 187 TFLOP/s (that library: 144 to 152), and the matrix cores are busy 68 % of it; 131,072 x 513 -> 1024 in bf16
// takes 393 where 512 columns take 181.  A packed x of dw is widened in registers beside direct tiles of dz: 188 us for
// 131,072 x 512 and 1024 (33 %), against 143 unpacked, also where the widening lies between the products; that kernel
// spills 159 registers, none of them in the loop over k, but where it goes from one tile to the next.
//
// 32-bit entries are taken apart into three bf16 parts, x = h + m + l, each the nearest to what the ones before leave
// (|m| <= 2^-9 |x|, |l| <= 2^-18 |x|, nothing is left from |x| = 2^-110 on; of smaller ones up to 2^-134, half of the least
// bf16 number, which the matrix cores take as it is), and their products summed as hh + hm + mh + hl + mm + lh in the 32-bit
// accumulators: what is left out is 2^-26 of a product, less than 32 bits round it by.  Six bf16 products of the matrix
// cores take three eighths of the time of one in 32 bits.  What an infinity leaves is NaN.
#pragma once

#include <type_traits>

#include "gosh_head.h"

namespace gosh {

// kPast: kForward of y alone, in tiles of kLarge, y stored past the caches.  (A kernel of its own: as a branch at each store it
// cost the other calls 2 to 20 %, in registers.  kForward, with every optional output, has 112 scalar registers in lanes of
// vector ones there, kPast 18: 131,072 x 512 -> 1024 with SiLU takes 180 us, 214 with z and 226 with a packed z.)
// kPastZ: kPast with z beside y, a z that is not packed past the caches too.
enum ProductOut : int { kForward, kStore, kParts, kPast, kPastZ };
constexpr bool is_forward(ProductOut out) { return out == kForward || out == kPast || out == kPastZ; }

struct ForwardOut {
  const float *bias;
  Plane residual, y, z, y8;
  int32_t act, z_packed;
  int32_t past;  // y alone, and too large for the caches
};

struct ProductArgs {
  Plane a, b;
  int64_t M, N, K;        // M, N < 2^31; K also
  int64_t k_per_split;    // a multiple of the tile's depth
  int32_t tiles_m, tiles_n, splits;
  int32_t direct;         // 16-bit operands of aligned rows: see can_be_direct
  ForwardOut forward;     // kForward, kPast
  Plane out;              // kStore
  float *parts;           // kParts: splits x M x N; dx in small tiles may have them too
};

// The products of a layer: which operands are k-major, whether B is packed.
enum ProductKind : int { kProductForward, kProductDx, kProductDw, kProductDwPacked };

enum TileSize : int { kSmall, kMiddle, kLarge };  // kLarge: only straight to LDS, others leave too few registers
constexpr int tile_m(TileSize s) { return s == kLarge ? 256 : s == kMiddle ? 128 : 64; }
constexpr int tile_n(TileSize s) { return tile_m(s); }

// Launches for entries of one type; defined in gosh_product_{f32,bf16,f16}.hip.
template <typename T>
int launch_product(ProductKind kind, TileSize size, const ProductArgs &args, hipStream_t st);
template <>
int launch_product<F32>(ProductKind, TileSize, const ProductArgs &, hipStream_t);
template <>
int launch_product<Bf16>(ProductKind, TileSize, const ProductArgs &, hipStream_t);
template <>
int launch_product<F16>(ProductKind, TileSize, const ProductArgs &, hipStream_t);

// dx and dw, both in tiles of kSmall, in one launch; `packed`: x is.
template <typename T>
int launch_both(bool packed, const ProductArgs &dx, const ProductArgs &dw, hipStream_t st);
template <>
int launch_both<F32>(bool, const ProductArgs &, const ProductArgs &, hipStream_t);
template <>
int launch_both<Bf16>(bool, const ProductArgs &, const ProductArgs &, hipStream_t);
template <>
int launch_both<F16>(bool, const ProductArgs &, const ProductArgs &, hipStream_t);

template <typename T>
struct ProductDepth {  // k of a tile that passes through registers: 128 and 64 bytes of LDS a row and part
  static constexpr int value(bool small) { return T::kType == GOSH_F32 ? (small ? 32 : 16) : 64; }
};

// Whether an operand can go straight to LDS: 16-byte aligned rows, of whole chunks along memory.
inline bool can_be_direct(const Plane &p, int64_t along) {
  return reinterpret_cast<uintptr_t>(p.data) % 16 == 0 && p.ld % 8 == 0 && along % 8 == 0;
}
// k of a tile, and tiles in LDS.  Rows of 64 k are lines of 128 bytes: with 32 k and a ring of 3 or 4 the address unit was
// busy 71 % of the time and the matrix cores 48 %, and 65,536 x 2048 -> 512 took 151 instead of 137 us.
constexpr int kDirectDepth = 64, kDirectRing = 2;
constexpr int direct_waves(int bn) { return bn == 256 ? 8 : 4; }

typedef float F16x __attribute__((ext_vector_type(16)));
typedef short S4 __attribute__((ext_vector_type(4)));
typedef short S8 __attribute__((ext_vector_type(8)));

template <typename T>
struct Cores {  // bf16, also the parts of 32-bit entries
  typedef __bf16 V8 __attribute__((ext_vector_type(8)));
  static constexpr int kParts = T::kType == GOSH_F32 ? 3 : 1;
  static __device__ __forceinline__ F16x mma(S8 a, S8 b, F16x c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
  }
};
template <>
struct Cores<F16> {
  typedef _Float16 V8 __attribute__((ext_vector_type(8)));
  static constexpr int kParts = 1;
  static __device__ __forceinline__ F16x mma(S8 a, S8 b, F16x c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
  }
};

// A range of memory whose bounds the hardware checks: what lies past `bytes` reads as zero.
typedef __amdgpu_buffer_rsrc_t Range;
__device__ __forceinline__ Range range_of(const void *p, int64_t bytes) {
  const int n = bytes <= 0 ? 0 : bytes > 0x7fffffff ? 0x7fffffff : static_cast<int>(bytes);
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, n, 0x00020000);
}
constexpr uint32_t kNowhere = 0x80000000u;  // an offset past every range, also with what is added to it

// Where an operand's 16-byte chunks lie in LDS, in entries.  16 lanes of a wavefront are served at a time, from 64 banks
// of 4 bytes: rows are shifted against each other so that the 16 chunks (or half chunks) that they ask for together lie
// in different banks.  Unshifted rows of 128 bytes were read at half the rate (124 instead of 240 bytes a cycle and CU).
template <int BX, int BK>
struct Spread {
  static constexpr int kAlongK = BK / 8, kRowsK = 128 / BK;  // chunks of a k-major row, rows that span the banks
  static __device__ __forceinline__ int k_major(int row, int chunk) {  // row = m
    return row * BK + ((chunk ^ ((row / kRowsK) & (kAlongK - 1))) * 8);
  }
  static __device__ __forceinline__ int shift(int k) { return BX >= 128 ? 2 * (k & 3) : 2 * ((k >> 1) & 1); }
  static __device__ __forceinline__ int m_major(int row, int chunk) {  // row = k
    return row * BX + (((chunk >> 1) ^ shift(row)) * 16) + (chunk & 1) * 8;
  }
  // 8 k (16 kk + 8 (lane / 32) + 0..7) of m = base + lane % 32, as the matrix cores take them.
  template <bool KMajor>
  static __device__ __forceinline__ S8 take(const uint16_t *lds, int base, int kk) {
    const int lane = threadIdx.x & 63;
    if constexpr (KMajor) {
      return *reinterpret_cast<const S8 *>(lds + k_major(base + (lane & 31), kk * 2 + (lane >> 5)));
    } else {
      typedef __attribute__((address_space(3))) S4 Shared;
      const int k = kk * 16 + 8 * (lane >> 5) + (lane & 15) / 4;
      const int pair = base / 16 + ((lane >> 4) & 1);
      const uint16_t *const from = lds + k * BX + ((pair ^ shift(k)) * 16) + (lane & 3) * 4;
      const S4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Shared *)(from));
      const S4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Shared *)(from + 4 * BX));
      return S8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    }
  }
};

// One operand's tile: BX entries of m by BK of k.
template <typename T, int BX, int BK, bool KMajor, bool Packed, int Threads = 256>
struct Tile {
  static_assert(!(KMajor && Packed), "only x of dw is packed");
  // a packed entry is a whole number of 8 bits times a power of two: one part holds it
  static constexpr int kParts = Packed ? 1 : Cores<T>::kParts;
  static constexpr int kBytes = kParts * BX * BK * 2;  // of LDS
  static constexpr int kSize = Packed ? 1 : T::kType == GOSH_F32 ? 4 : 2;
  static constexpr int kChunks = BX * BK / 8;               // of 8 entries along memory
  static constexpr int kPerThread = kChunks / Threads;
  static constexpr int kAlong = (KMajor ? BK : BX) / 8;     // chunks in a row of the tile
  static constexpr int kWords = Packed ? 2 : T::kType == GOSH_F32 ? 8 : 4;
  static constexpr int kLoads = 0;  // straight to LDS
  static_assert(kChunks % Threads == 0 && Threads % kAlong == 0, "");

  uint32_t raw[kPerThread][kWords];
  uint32_t unit[Packed ? kPerThread : 1];

  // x: first m of the tile, of `mx`; k: first k, up to `kx`.  `ragged`: the step may hold chunks of which some entries
  // are there.
  __device__ __forceinline__ void fetch(const Plane &p, int64_t x, int64_t mx, int64_t k, int64_t kx, bool ragged) {
    const int t = threadIdx.x;
    const int at = t % kAlong * 8;  // first entry of a chunk along memory
    const int64_t row0 = KMajor ? x : k, col0 = KMajor ? k : x;
    const int64_t rows = (KMajor ? mx : kx) - row0, cols = (KMajor ? kx : mx) - col0;
    const int64_t bytes = ((rows - 1) * p.ld + cols) * kSize;
    const Range r = range_of(static_cast<const char *>(p.data) + (row0 * p.ld + col0) * kSize, bytes);
    const int ld = static_cast<int>(p.ld) * kSize;
    Range re;
    if constexpr (Packed)
      re = range_of(p.exps + row0 * p.ld_exps + col0 / kGroup, (rows - 1) * p.ld_exps + (cols + kGroup - 1) / kGroup);
    const int there = static_cast<int>(cols < BX + BK ? cols : BX + BK) - at;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      const int row = t / kAlong + i * (Threads / kAlong);
      const uint32_t off = static_cast<uint32_t>(row * ld + at * kSize);
      if constexpr (Packed)
        unit[i] = __builtin_amdgcn_raw_buffer_load_b8(re, row * static_cast<int>(p.ld_exps) + at / kGroup, 0, 0);
      if (!ragged) {
        // along k, entries past the end of a row are another row's and must count as zero; along m they are
        // columns of the result that nobody stores
        const uint32_t o = KMajor && there <= 0 ? kNowhere : off;
        if constexpr (kWords == 2) {
          const U2 v = __builtin_amdgcn_raw_buffer_load_b64(r, o, 0, 0);
          raw[i][0] = v[0], raw[i][1] = v[1];
        } else {
#pragma unroll
          for (int w = 0; w < kWords; w += 4) {
            const U4 v = __builtin_amdgcn_raw_buffer_load_b128(r, o + 4 * w, 0, 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) raw[i][w + j] = v[j];
          }
        }
      } else {
#pragma unroll
        for (int w = 0; w < kWords; ++w) raw[i][w] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t o = e < there ? off + e * kSize : kNowhere;
          if constexpr (kSize == 4) raw[i][e] = __builtin_amdgcn_raw_buffer_load_b32(r, o, 0, 0);
          if constexpr (kSize == 2) {
            const uint32_t v = static_cast<uint16_t>(__builtin_amdgcn_raw_buffer_load_b16(r, o, 0, 0));
            raw[i][e / 2] |= v << (16 * (e % 2));
          }
          if constexpr (kSize == 1) {
            const uint32_t v = static_cast<uint8_t>(__builtin_amdgcn_raw_buffer_load_b8(r, o, 0, 0));
            raw[i][e / 4] |= v << (8 * (e % 4));
          }
        }
      }
    }
  }

  __device__ __forceinline__ void put(uint16_t *lds) const {
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      const int row = t / kAlong + i * (Threads / kAlong), c = t % kAlong;
      uint16_t *const to = lds + (KMajor ? Spread<BX, BK>::k_major(row, c) : Spread<BX, BK>::m_major(row, c));
      if constexpr (Packed) {
        const uint32_t q[2] = {raw[i][0], raw[i][1]};
        float v[8];
        widen<8>(q, read_unit(unit[i] & 255u), v);
        typedef typename std::conditional<T::kType == GOSH_F16, F16, Bf16>::type E;
        typename E::Store e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = E::down(v[j]);
        U4 w;
        __builtin_memcpy(&w, e, 16);
        *reinterpret_cast<U4 *>(to) = w;
      } else if constexpr (kParts == 1) {
        *reinterpret_cast<U4 *>(to) = U4{raw[i][0], raw[i][1], raw[i][2], raw[i][3]};
      } else {
        uint32_t part[3][4];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          float x[2] = {__uint_as_float(raw[i][j]), __uint_as_float(raw[i][j + 1])};
#pragma unroll
          for (int p = 0; p < 3; ++p) {
            typedef float Two __attribute__((ext_vector_type(2)));
            typedef __bf16 Near __attribute__((ext_vector_type(2)));
            const uint32_t two = __builtin_bit_cast(uint32_t, __builtin_convertvector((Two{x[0], x[1]}), Near));
            part[p][j / 2] = two;
            if (p == 2) break;
            const float near[2] = {__uint_as_float(two << 16), __uint_as_float(two & 0xffff0000u)};
#pragma unroll
            for (int s = 0; s < 2; ++s) x[s] -= near[s];  // exact
          }
        }
#pragma unroll
        for (int p = 0; p < 3; ++p)
          *reinterpret_cast<U4 *>(to + p * BX * BK) = U4{part[p][0], part[p][1], part[p][2], part[p][3]};
      }
    }
  }
};

// Where a lane's entries lie in a matrix: a row and column that are the same for the wavefront, in scalar registers, and
// the lane's place from there, 32 bits.
struct Spot {
  int64_t row, col;
  int down, right;
  template <typename S>
  __device__ __forceinline__ S *in(const Plane &p) const {
    const uint32_t lane = static_cast<uint32_t>(down * static_cast<int>(p.ld) + right) * static_cast<uint32_t>(sizeof(S));
    return reinterpret_cast<S *>(static_cast<char *>(p.data) + (row * p.ld + col) * static_cast<int64_t>(sizeof(S)) + lane);
  }
  __device__ __forceinline__ uint8_t *exponent_in(const Plane &p) const {
    return p.exps + (row * p.ld_exps + col / kGroup) + static_cast<uint32_t>(down * static_cast<int>(p.ld_exps) + right / kGroup);
  }
};

// E entries of a row of z become entries of y; r: the residual's.  Full: all of them are there.  Past, More: see kPast; More:
// z and y8 may be asked for.
template <typename T, int E, bool Full, bool Past, bool More>
__device__ __forceinline__ void put_forward(const ForwardOut &f, const Spot &at, int there, float (&v)[E],
                                            const typename Entries<T, E>::Vec &r) {
  typedef typename T::Store S;
  constexpr int kLanes = kGroup / E;  // of a group of the 8-bit form
  const bool head = threadIdx.x % kLanes == 0;
  const int count = Full ? E : there;
  if (!Full) {
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = i < count ? v[i] : 0.f;  // entries that are not there count in no group
  }
  if (More && f.z.data != nullptr) {
    if (f.z_packed) store_packed<T, E>(at.in<int8_t>(f.z), at.exponent_in(f.z), count, v, head, kLanes);
    else if (Full || count > 0) Entries<T, E>::template store<Past>(at.in<S>(f.z), count, v);
  }
  with_activation(f.act, [&](auto a) {
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = decltype(a)::value(v[i]);
  });
  if (f.residual.data != nullptr) {
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] += T::up(r[i]);
  }
  if (More && f.y8.data != nullptr) {
    if (!Full) {
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = i < count ? v[i] : 0.f;
    }
    store_packed<T, E>(at.in<int8_t>(f.y8), at.exponent_in(f.y8), count, v, head, kLanes);
  }
  if (Full || count > 0) Entries<T, E>::template store<Past>(at.in<S>(f.y), count, v);
}

// The id-th tile.
struct Place {
  int64_t m0, n0, k0, k1;
  int split;
};
__device__ __forceinline__ Place place_of(const ProductArgs &g, int id, int bm, int bn) {
  const int tn = id % g.tiles_n, tm = id / g.tiles_n % g.tiles_m, split = id / g.tiles_n / g.tiles_m;
  const int64_t k0 = split * g.k_per_split;
  return {static_cast<int64_t>(tm) * bm, static_cast<int64_t>(tn) * bn, k0,
          k0 + g.k_per_split < g.K ? k0 + g.k_per_split : g.K, split};
}

// Workgroups go round the 8 XCDs: each XCD gets a contiguous run of tiles, those of the same rows next to each other, so
// that they share its L2, and its workgroups take turns along the run.
struct Turns {
  int id, end, step;
};
__device__ __forceinline__ Turns turns_of(int total) {
  const int blocks = gridDim.x, b = blockIdx.x;
  if (blocks % 8 != 0) return {b, total, blocks};
  const int xcd = b % 8, per = total / 8, more = total % 8;
  const int first = xcd * per + (xcd < more ? xcd : more);
  return {first + b / 8, first + per + (xcd < more), blocks / 8};
}

// What the accumulators start from: the bias of a lane's columns.
template <int RN, ProductOut Out>
__device__ __forceinline__ void load_bias(const ProductArgs &g, int64_t n, float (&bias)[RN]) {
#pragma unroll
  for (int j = 0; j < RN; ++j) {
    const int64_t col = n + 32 * j + (threadIdx.x & 31);
    bias[j] = is_forward(Out) && g.forward.bias != nullptr && col < g.N ? g.forward.bias[col] : 0.f;
  }
}
template <int RM, int RN>
__device__ __forceinline__ void start(const float (&bias)[RN], F16x (&acc)[RM][RN]) {
#pragma unroll
  for (int j = 0; j < RN; ++j)
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = bias[j];
}

// A wavefront's 8 rows of W results on their way from columns to rows: where entry (row, col) lies.  Written by lanes of
// which half are 4 rows on, read 8 columns of a lane in two steps: the shifts keep both off each other's banks.
template <int W>
struct Slab {
  static constexpr int kFloats = 8 * W;
  static __device__ __forceinline__ int at(int row, int col) {
    return W == 64 ? row * W + (col ^ (row & 4) * 8 ^ (row & 1) * 4) : row * W + (col ^ (row & 2) * 2);
  }
};

// The accumulators of a wavefront, at m, n, to where they go, 8 rows at a time through its slab: a lane of the
// accumulators holds entries of one column.
template <typename T, int RM, int RN, ProductOut Out, bool Full>
__device__ __forceinline__ void finish(const ProductArgs &g, const F16x (&acc)[RM][RN], float *slab, int64_t m, int64_t n, int split) {
  constexpr int W = 32 * RN;
  constexpr int E = Out == kParts || T::kType == GOSH_F32 ? 4 : 8;  // 16 bytes of a row to a lane
  constexpr int kLanes = W / E, kRows = 64 / kLanes < 8 ? 64 / kLanes : 8;  // lanes of a row, rows at a time
  constexpr bool kFull = Full && kLanes * kRows == 64;
  typedef typename T::Store S;
  const int lane = threadIdx.x & 63;
  const int r = lane / kLanes, c = lane % kLanes * E;
  const int across = static_cast<int>(g.N - n) - c, down = static_cast<int>(g.M - m < 32 * RM ? g.M - m : 32 * RM) - r;
  const auto count_of = [&](int turn) {
    const int left = r < kRows && kRows * turn < down ? across : 0;
    return kFull ? E : left < 0 ? 0 : left > E ? E : left;
  };
  const auto spot_of = [&](int turn) { return Spot{m + kRows * turn, n, r, c}; };
  // the residual of some rows is loaded kAhead turns before: by itself each load would be waited for, behind the stores
  // before it
  constexpr int kAhead = 2, kTurns = 32 / kRows * RM;
  typename Entries<T, E>::Vec residual[kAhead + 1];
  const auto load_residual = [&](int turn) {
    if (!is_forward(Out) || g.forward.residual.data == nullptr) return;
    residual[turn % (kAhead + 1)] = Entries<T, E>::fetch(spot_of(turn).template in<S>(g.forward.residual), count_of(turn));
  };
#pragma unroll
  for (int turn = 0; turn < kAhead; ++turn) load_residual(turn);
#pragma unroll
  for (int i = 0; i < RM; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int j = 0; j < RN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) slab[Slab<W>::at(4 * (lane >> 5) + e, 32 * j + (lane & 31))] = acc[i][j][4 * q + e];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int h = 0; h < 8 / kRows; ++h) {
        const int turn = (4 * i + q) * (8 / kRows) + h;
        if (turn + kAhead < kTurns) load_residual(turn + kAhead);
        const int count = count_of(turn);
        float v[E];
#pragma unroll
        for (int w = 0; w < E; w += 4) {
          const F4 x = *reinterpret_cast<const F4 *>(slab + Slab<W>::at((kRows * h + r) & 7, c + w));
#pragma unroll
          for (int e = 0; e < 4; ++e) v[w + e] = x[e];
        }
        if constexpr (is_forward(Out)) {
          put_forward<T, E, kFull, Out == kPast || Out == kPastZ, Out != kPast>(g.forward, spot_of(turn), count, v, residual[turn % (kAhead + 1)]);
        } else if constexpr (Out == kStore) {
          if (count > 0) Entries<T, E>::store(spot_of(turn).template in<S>(g.out), count, v);
        } else {
          const Plane parts{g.parts + split * g.M * g.N, nullptr, g.N, 0};
          if (count > 0) Entries<F32, E>::store(spot_of(turn).template in<float>(parts), count, v);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
}

template <typename T, int RM, int RN, ProductOut Out>
__device__ __forceinline__ void finish(const ProductArgs &g, const F16x (&acc)[RM][RN], float *slab, int64_t m, int64_t n, int split) {
  if (m + 32 * RM <= g.M && n + 32 * RN <= g.N) finish<T, RM, RN, Out, true>(g, acc, slab, m, n, split);
  else finish<T, RM, RN, Out, false>(g, acc, slab, m, n, split);
}

// Tiles that pass through registers on their way to LDS: 32-bit entries, packed ones, and matrices whose rows are not
// 16-byte aligned.
template <typename T, int BX, ProductKind Kind>
struct Staged {
  static constexpr int BK = ProductDepth<T>::value(BX == 64);
  static constexpr bool a_k = Kind == kProductForward || Kind == kProductDx, b_k = Kind == kProductForward;
  typedef Tile<T, BX, BK, a_k, false> TA;
  typedef Tile<T, BX, BK, b_k, Kind == kProductDwPacked> TB;
  static constexpr int kBuffer = (TA::kBytes + TB::kBytes) / 2;
  static constexpr int kSlabs = 4 * Slab<BX / 2>::kFloats * 4;
  static constexpr int kLds = 2 * kBuffer * 2 > kSlabs ? 2 * kBuffer * 2 : kSlabs;
};

// The id-th tile.
template <typename T, int BX, ProductKind Kind, ProductOut Out>
__device__ __forceinline__ void staged_product(const ProductArgs &g, int id, uint16_t *lds) {
  typedef Staged<T, BX, Kind> P;
  typedef typename P::TA TA;
  typedef typename P::TB TB;
  constexpr int BK = P::BK, kBuffer = P::kBuffer;
  constexpr bool a_k = P::a_k, b_k = P::b_k;
  constexpr int W = BX / 2, R = W / 32;          // a wavefront's square of the tile, and its 32 x 32 blocks a side

  const Place at = place_of(g, id, BX, BX);
  const int64_t m0 = at.m0, n0 = at.n0, k0 = at.k0, k1 = at.k1;
  const int steps = static_cast<int>((k1 - k0 + BK - 1) / BK);

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wm = wave / 2 * W, wn = wave % 2 * W;
  F16x acc[R][R];
  float bias[R];
  load_bias<R, Out>(g, n0 + wn, bias);
  start<R, R>(bias, acc);

  // The last step's chunks may be short: along k where K is no multiple of 8; along m the very last row of memory ends
  // inside its last chunk, of which the hardware's bounds check drops a dword that is only partly there.  Along m a row of an
  // earlier step has at least one row after it, whose bytes complete its last dword: up to 2 of them are missing in 16-bit
  // rows, none in 32-bit ones, and 3 in packed ones, which rows less than 3 bytes apart do not have.
  const bool ragged_a = a_k ? k1 % 8 != 0 : g.M % 8 != 0, ragged_b = b_k ? k1 % 8 != 0 : g.N % 8 != 0;
  const bool always_b = Kind == kProductDwPacked && g.b.ld < 3;
  TA a;
  TB b;
  if (steps > 0) {
    a.fetch(g.a, m0, g.M, k0, k1, steps == 1 && ragged_a);
    b.fetch(g.b, n0, g.N, k0, k1, always_b || (steps == 1 && ragged_b));
    a.put(lds);
    b.put(lds + TA::kBytes / 2);
  }
  for (int s = 0; s < steps; ++s) {
    __syncthreads();
    uint16_t *const now = lds + (s & 1) * kBuffer, *const next = lds + (~s & 1) * kBuffer;
    const bool more = s + 1 < steps;
    if (more) {
      const int64_t k = k0 + static_cast<int64_t>(s + 1) * BK;
      const bool last = s + 2 == steps;
      a.fetch(g.a, m0, g.M, k, k1, last && ragged_a);
      b.fetch(g.b, n0, g.N, k, k1, always_b || (last && ragged_b));
    }
#pragma unroll
    for (int kk = 0; kk < BK / 16; ++kk) {
      S8 fa[TA::kParts][R], fb[TB::kParts][R];
#pragma unroll
      for (int p = 0; p < TA::kParts; ++p)
#pragma unroll
        for (int i = 0; i < R; ++i) fa[p][i] = Spread<BX, BK>::template take<a_k>(now + p * BX * BK, wm + 32 * i, kk);
#pragma unroll
      for (int p = 0; p < TB::kParts; ++p)
#pragma unroll
        for (int i = 0; i < R; ++i) fb[p][i] = Spread<BX, BK>::template take<b_k>(now + TA::kBytes / 2 + p * BX * BK, wn + 32 * i, kk);
#pragma unroll
      for (int order = TA::kParts + TB::kParts - 2; order >= 0; --order)  // the smallest products first
#pragma unroll
        for (int p = 0; p <= order; ++p) {
          if (order > 2 || p >= TA::kParts || order - p >= TB::kParts) continue;
#pragma unroll
          for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < R; ++j) acc[i][j] = Cores<T>::mma(fa[p][i], fb[order - p][j], acc[i][j]);
        }
    }
    if (more) {
      a.put(next);
      b.put(next + TA::kBytes / 2);
    }
  }
  __syncthreads();

  finish<T, R, R, Out>(g, acc, reinterpret_cast<float *>(lds) + wave * Slab<W>::kFloats, m0 + wm, n0 + wn, at.split);
}

template <typename T, int BX, ProductKind Kind, ProductOut Out>
__global__ __launch_bounds__(256, 2) void product_kernel(const ProductArgs g) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[Staged<T, BX, Kind>::kLds / 2];
  staged_product<T, BX, Kind, Out>(g, turns_of(g.tiles_m * g.tiles_n * g.splits).id, lds);
}

// Both products of a gradient that is small: one launch, and neither waits for the other.  (Measured where it is chosen.)
template <typename T, ProductKind Dw, ProductOut DxOut>
__global__ __launch_bounds__(256, 2) void both_products_kernel(const ProductArgs dx, const ProductArgs dw) {
  constexpr int a = Staged<T, 64, kProductDx>::kLds, b = Staged<T, 64, Dw>::kLds;
  __shared__ __attribute__((aligned(16))) uint16_t lds[(a > b ? a : b) / 2];
  const int first = dx.tiles_m * dx.tiles_n * dx.splits, id = blockIdx.x;
  if (id < first) staged_product<T, 64, kProductDx, DxOut>(dx, id, lds);
  else staged_product<T, 64, Dw, kParts>(dw, id - first, lds);
}

// ---- 16-bit tiles that go straight to LDS -------------------------------------------------------

// A tile that the memory system writes to LDS by itself, 1 KB an instruction of a wavefront: lane i's 16 bytes land at
// 16 i, so that the lanes ask for the chunks that belong there.  Rows are 16-byte aligned and whole numbers of chunks.
template <int BX, int BK, bool KMajor, int Waves>
struct DirectTile {
  static constexpr int kBytes = BX * BK * 2;
  static constexpr int kLoads = kBytes / 1024 / Waves;        // of a wavefront
  static_assert(kBytes % (1024 * Waves) == 0, "");
  static constexpr int kAlong = (KMajor ? BK : BX) / 8;       // chunks in a row of the tile
  uint32_t off[kLoads];
  int along[kLoads];  // first k of the lane's chunks (k-major)

  __device__ __forceinline__ void init(const Plane &p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = (wave * kLoads + i) * 64 + lane;
      const int row = at / kAlong, slot = at % kAlong;
      // the chunk that the shifts put at this slot: they are their own inverse
      const int chunk = KMajor ? Spread<BX, BK>::k_major(row, slot) / 8 % kAlong : Spread<BX, BK>::m_major(row, slot) / 8 % kAlong;
      off[i] = static_cast<uint32_t>(row * static_cast<int>(p.ld) + chunk * 8) * 2;
      along[i] = chunk * 8;
    }
  }
  // The tile of m from x, of mx, and of k from k, up to kx: uniform, in scalar registers.
  uint64_t base;
  int64_t bytes;
  int left;  // k
  __device__ __forceinline__ void begin(const Plane &p, int64_t x, int64_t mx, int64_t k, int64_t kx) {
    const int64_t row0 = KMajor ? x : k, col0 = KMajor ? k : x;
    const int64_t rows = (KMajor ? mx : kx) - row0, cols = (KMajor ? kx : mx) - col0;
    base = reinterpret_cast<uint64_t>(p.data) + (row0 * p.ld + col0) * 2;
    bytes = ((rows - 1) * p.ld + cols) * 2;
    left = static_cast<int>(kx - k);
  }
  // Starts the loads of the next step into the tile at byte `lds` of LDS.  What is past the range reads as zero; so are
  // chunks past the last k made to.
  __device__ __forceinline__ void fetch(const Plane &p, uint32_t lds) {
    const U4 range{static_cast<uint32_t>(base), static_cast<uint32_t>(base >> 32) & 0xffffu,
                   static_cast<uint32_t>(bytes <= 0 ? 0 : bytes > 0x7fffffff ? 0x7fffffff : bytes), 0x00020000u};
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      uint32_t o = off[i];
      if (KMajor) o = along[i] < left ? o : kNowhere;
      // m0, which the compiler sets, holds where the first lane's bytes land; the load has no destination register.  The
      // compiler does not count the wait states of an instruction that it cannot see: s_nop 4 are the five that the load
      // needs behind a vector instruction that wrote its range (a spilled register read back), more than behind m0's move.
      // With the builtin for this load the compiler waits for all under way before a step's transposing reads: 482 instead of
      // 455 us for the gradient of 65,536 x 512 -> 2048.
      asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                   :: "v"(o), "s"(range), "{m0}"(lds + (wave * kLoads + i) * 1024) : "memory");
    }
    const int64_t move = KMajor ? BK * 2 : static_cast<int64_t>(p.ld) * (BK * 2);
    base += move;
    bytes -= move;
    left -= BK;
  }
};

// The same product with a ring of kDirectRing tiles: while a step is computed the loads of the next ones are under way,
// also across the end of a tile: a workgroup goes from tile to tile, and the next one's loads run while the results of
// the last are written.  A packed operand goes through registers, two steps ahead, where its entries get their width.
template <typename T, int BM, int BN, ProductKind Kind, ProductOut Out>
__global__ __launch_bounds__(64 * direct_waves(BN), 8 / direct_waves(BN)) void direct_product_kernel(const ProductArgs g) {
  constexpr int BK = kDirectDepth;
  constexpr bool a_k = Kind == kProductForward || Kind == kProductDx, b_k = Kind == kProductForward;
  constexpr int kWaves = direct_waves(BN), kAcross = kWaves / 2;
  typedef DirectTile<BM, BK, a_k, kWaves> TA;
  constexpr bool packed = Kind == kProductDwPacked;
  typedef typename std::conditional<packed, Tile<T, BN, BK, b_k, packed, 64 * kWaves>, DirectTile<BN, BK, b_k, kWaves>>::type TB;
  constexpr int WM = BM / 2, WN = BN / kAcross, RM = WM / 32, RN = WN / 32, kRing = kDirectRing;
  constexpr int kStep = TA::kBytes + TB::kBytes, kLoads = packed ? 0 : TA::kLoads + TB::kLoads;
  constexpr int kStores = RM * 4;  // of a wavefront for a whole tile, at least
  static_assert(BK / 16 % 2 == 0, "the entries read ahead are in turns");
  __shared__ __attribute__((aligned(1024))) uint16_t lds[kRing * kStep / 2];
  __shared__ __attribute__((aligned(16))) float slabs[kWaves * Slab<WN>::kFloats];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wm = wave / kAcross * WM, wn = wave % kAcross * WN;
  const Turns turns = turns_of(g.tiles_m * g.tiles_n * g.splits);
  if (turns.id >= turns.end) return;
  const auto steps_of = [](const Place &p) { return static_cast<int>((p.k1 - p.k0 + BK - 1) / BK); };

  const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint16_t *)lds));
  TA a;
  TB b;
  a.init(g.a);
  if constexpr (!packed) b.init(g.b);
  // The loads run ahead of the computation, over tiles.  After the last tile they load nothing, so that the count of
  // loads under way stays the same.
  uint32_t into = base;
  int turn = turns.id;
  int to_go;
  Place from;
  const auto begin = [&]() {
    from = place_of(g, turn, BM, BN);
    a.begin(g.a, from.m0, g.M, from.k0, from.k1);
    if constexpr (!packed) b.begin(g.b, from.n0, g.N, from.k0, from.k1);
    to_go = steps_of(from);
  };
  const auto fetch = [&]() {
    if constexpr (packed) {
      b.fetch(g.b, from.n0, g.N, from.k0, from.k1, false);
      from.k0 += BK;
      a.fetch(g.a, into);
    } else {
      a.fetch(g.a, into);
      b.fetch(g.b, into + TA::kBytes);
    }
    into = into == base + (kRing - 1) * kStep ? base : into + kStep;
    if (--to_go <= 0 && turn + turns.step < turns.end) {
      turn += turns.step;
      begin();
    }
  };
  begin();
#pragma unroll
  for (int s = 0; s < kRing; ++s) {
    fetch();
    if constexpr (packed)
      if (s == 0) b.put(lds + TA::kBytes / 2);
  }
  const uint16_t *now = lds;
  S8 fa[2][RM], fb[2][RN];
  const auto take = [&](int part) {
#pragma unroll
    for (int j = 0; j < RN; ++j) fb[part & 1][j] = Spread<BN, BK>::template take<b_k>(now + TA::kBytes / 2, wn + 32 * j, part);
#pragma unroll
    for (int i = 0; i < RM; ++i) fa[part & 1][i] = Spread<BM, BK>::template take<a_k>(now, wm + 32 * i, part);
  };
  float bias[RN];
  load_bias<RN, Out>(g, place_of(g, turns.id, BM, BN).n0 + wn, bias);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"((kRing - 1) * kLoads) : "memory");
  take(0);
  bool stored = false;  // the wavefront has written a whole tile just before
  for (int id = turns.id; id < turns.end; id += turns.step) {
    const Place at = place_of(g, id, BM, BN);
    const int steps = steps_of(at);
    F16x acc[RM][RN];
    start<RM, RN>(bias, acc);
    if (is_forward(Out) && id + turns.step < turns.end)
      load_bias<RN, Out>(g, place_of(g, id + turns.step, BM, BN).n0 + wn, bias);
    const auto multiply = [&](int part) {
#pragma unroll
      for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int j = 0; j < RN; ++j) acc[i][j] = Cores<T>::mma(fa[part & 1][i], fb[part & 1][j], acc[i][j]);
    };
    for (int s = 0; s < steps; ++s) {
      // Each 16 k of a step are read from LDS while those before are multiplied.
      constexpr int kParts = BK / 16;
#pragma unroll
      for (int part = 0; part < kParts - 1; ++part) {
        take(part + 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(part);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (packed) {
        static_assert(kRing == 2, "the other tile is the next step's");
        b.put(lds + (now == lds ? kStep / 2 : 0) + TA::kBytes / 2);
      }
      // Loads and stores end in order.  The next step's loads are followed by those of kRing - 2 steps and, in the first
      // steps after a tile, its stores, which need not be waited for.  Then every wavefront's part is there, and every
      // wavefront is done with this step's tile, which the next loads replace.
      if (!packed && stored && s < kRing - 1)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"((kRing - 2) * kLoads + kStores) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"((kRing - 2) * kLoads) : "memory");
      now = now == lds + (kRing - 1) * (kStep / 2) ? lds : now + kStep / 2;
      take(0);
      fetch();
      __builtin_amdgcn_sched_barrier(0);
      multiply(kParts - 1);
    }
    // the next tile's bias is waited for here, before the stores: after them it would wait for those too
#pragma unroll
    for (int j = 0; j < RN; ++j) asm volatile("" : "+v"(bias[j]));
    finish<T, RM, RN, Out>(g, acc, slabs + wave * Slab<WN>::kFloats, at.m0 + wm, at.n0 + wn, at.split);
    stored = WN == 64 && at.m0 + wm + WM <= g.M && at.n0 + wn + WN <= g.N;
  }
  // no load may land in LDS that is another workgroup's by then
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <typename T, TileSize Size, ProductKind Kind, ProductOut Out>
int launch_one(const ProductArgs &g, hipStream_t st) {
  const unsigned blocks = static_cast<unsigned>(g.tiles_m) * g.tiles_n * g.splits;
  if constexpr (T::kType != GOSH_F32) {
    if (g.direct) {
      const unsigned held = static_cast<unsigned>(resident_waves()) / 4 / direct_waves(tile_n(Size));  // eight wavefronts a CU
      direct_product_kernel<T, tile_m(Size), tile_n(Size), Kind, Out><<<dim3(blocks < held ? blocks : held), dim3(64 * direct_waves(tile_n(Size))), 0, st>>>(g);
      return check_launch("matrix product");
    }
  }
  if constexpr (Size == kLarge) {
    return fail(GOSH_EINVAL, "tiles of 256 x 256 are for aligned rows of 16-bit entries");
  } else {
    product_kernel<T, tile_m(Size), Kind, Out><<<dim3(blocks), dim3(256), 0, st>>>(g);
    return check_launch("matrix product");
  }
}

template <typename T, TileSize Size>
int launch_sized(ProductKind kind, const ProductArgs &g, hipStream_t st) {
  switch (kind) {
    case kProductForward:
      if constexpr (Size == kLarge && T::kType != GOSH_F32)
        if (g.forward.past && g.direct) return launch_one<T, Size, kProductForward, kPast>(g, st);
      return launch_one<T, Size, kProductForward, kForward>(g, st);
    case kProductDx:
      if constexpr (Size == kSmall)
        if (g.parts != nullptr) return launch_one<T, Size, kProductDx, kParts>(g, st);
      return launch_one<T, Size, kProductDx, kStore>(g, st);
    case kProductDw: return launch_one<T, Size, kProductDw, kParts>(g, st);
    default: return launch_one<T, Size, kProductDwPacked, kParts>(g, st);
  }
}

template <typename T>
int launch_any(ProductKind kind, TileSize size, const ProductArgs &g, hipStream_t st) {
  if (size == kLarge) return launch_sized<T, kLarge>(kind, g, st);
  if (size == kMiddle) return launch_sized<T, kMiddle>(kind, g, st);
  return launch_sized<T, kSmall>(kind, g, st);
}

template <typename T>
int launch_both_any(bool packed, const ProductArgs &dx, const ProductArgs &dw, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(dx.tiles_m * dx.tiles_n * dx.splits + dw.tiles_m * dw.tiles_n * dw.splits)), block(256);
  if (packed && dx.parts != nullptr) both_products_kernel<T, kProductDwPacked, kParts><<<grid, block, 0, st>>>(dx, dw);
  else if (packed) both_products_kernel<T, kProductDwPacked, kStore><<<grid, block, 0, st>>>(dx, dw);
  else if (dx.parts != nullptr) both_products_kernel<T, kProductDw, kParts><<<grid, block, 0, st>>>(dx, dw);
  else both_products_kernel<T, kProductDw, kStore><<<grid, block, 0, st>>>(dx, dw);
  return check_launch("matrix products of the gradient");
}

}  // namespace gosh
