// Tiled matrix products of the linear layer on the matrix cores, one unit per element type.
//
// C (M x N) = sum over k of A(m, k) B(n, k).  An operand lies in memory either with k along its rows ("k-major": x and w
// of the forward pass, dz of dx) or with k across them ("m-major": w of dx, dz and x of dw, where k counts rows of the
// batch).  Both are staged through LDS in 16-bit entries: k-major tiles are read 8 k at a time, m-major ones through the
// transposing read (16 lanes fetch 4 rows of 16 entries and get 4 entries of one column each), so that no operand is
// transposed in memory.
//
// 32-bit entries are taken apart into three bf16 parts, x = h + m + l, each the nearest to what the ones before leave
// (|m| <= 2^-9 |x|, |l| <= 2^-18 |x|, nothing is left), and their products summed as hh + hm + mh + hl + mm + lh in the
// 32-bit accumulators: what is left out is 2^-26 of a product, less than 32 bits round it by.  Six bf16 products of the
// matrix cores take three eighths of the time of one in 32 bits.  An infinity has no parts but itself, and meets zeros
// among the other factor's: it gives NaN.
#pragma once

#include <type_traits>

#include "gosh_head.h"

namespace gosh {

enum ProductOut : int { kForward, kStore, kParts };

struct ForwardOut {
  const float *bias;
  Plane residual, y, z, y8;
  int32_t act, z_packed;
};

struct ProductArgs {
  Plane a, b;
  int64_t M, N, K;        // M, N < 2^31; K also
  int64_t k_per_split;    // a multiple of the tile's depth
  int32_t tiles_m, tiles_n, splits;
  ForwardOut forward;     // kForward
  Plane out;              // kStore
  float *parts;           // kParts: splits x M x N
};

// The products of a layer: which operands are k-major, whether B is packed.
enum ProductKind : int { kProductForward, kProductDx, kProductDw, kProductDwPacked };

// Launches for rows of one type; defined in gosh_product_{f32,bf16,f16}.hip.  `small`: 64 x 64 tiles.
template <typename T>
int launch_product(ProductKind kind, bool small, const ProductArgs &args, hipStream_t st);
template <>
int launch_product<F32>(ProductKind, bool, const ProductArgs &, hipStream_t);
template <>
int launch_product<Bf16>(ProductKind, bool, const ProductArgs &, hipStream_t);
template <>
int launch_product<F16>(ProductKind, bool, const ProductArgs &, hipStream_t);

template <typename T>
struct ProductDepth {  // k of a tile: 128 and 64 bytes of LDS a row and part
  static constexpr int value(bool small) { return T::kType == GOSH_F32 ? (small ? 32 : 16) : 64; }
};
inline int product_depth(int32_t type, bool small) {
  return type == GOSH_F32 ? ProductDepth<F32>::value(small) : ProductDepth<Bf16>::value(small);
}

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

// One operand's tile: BX entries of m by BK of k.
template <typename T, int BX, int BK, bool KMajor, bool Packed>
struct Tile {
  static_assert(!(KMajor && Packed), "only x of dw is packed");
  // a packed entry is a whole number of 8 bits times a power of two: one part holds it
  static constexpr int kParts = Packed ? 1 : Cores<T>::kParts;
  static constexpr int kBytes = kParts * BX * BK * 2;
  static constexpr int kSize = Packed ? 1 : T::kType == GOSH_F32 ? 4 : 2;
  static constexpr int kChunks = BX * BK / 8;               // of 8 entries along memory
  static constexpr int kPerThread = kChunks / 256;
  static constexpr int kAlong = (KMajor ? BK : BX) / 8;     // chunks in a row of the tile
  static constexpr int kWords = Packed ? 2 : T::kType == GOSH_F32 ? 8 : 4;
  static_assert(kChunks % 256 == 0 && 256 % kAlong == 0, "");

  uint32_t raw[kPerThread][kWords];
  uint32_t unit[Packed ? kPerThread : 1];

  // Reading 8 lanes' chunks of one column takes in all banks if rows of 128 bytes are shifted against each other.
  static __device__ __forceinline__ int shift_k(int row) {
    constexpr int per = BK / 8;
    return per >= 8 ? row & 7 : (row / (8 / per)) & (per - 1);
  }
  // The transposing reads of a wavefront take in rows k = 0..3 and 8..11 (+ 4 j + 16 i) of two neighbouring 16 columns.
  static __device__ __forceinline__ int shift_m(int k) { return ((k & 3) | ((k >> 1) & 4)) & (BX / 16 - 1); }

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
      const int row = t / kAlong + i * (256 / kAlong);
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
      const int row = t / kAlong + i * (256 / kAlong), c = t % kAlong;
      uint16_t *const to =
          lds + (KMajor ? row * BK + ((c ^ shift_k(row)) * 8) : row * BX + (((c >> 1) ^ shift_m(row)) * 16) + (c & 1) * 8);
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
            const uint32_t two = static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(x[0]))) |
                                 static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(x[1]))) << 16;
            part[p][j / 2] = two;
            if (p == 2) break;
            const float near[2] = {__uint_as_float(two << 16), __uint_as_float(two & 0xffff0000u)};
#pragma unroll
            for (int s = 0; s < 2; ++s) x[s] = __builtin_isinf(near[s]) ? 0.f : x[s] - near[s];  // exact
          }
        }
#pragma unroll
        for (int p = 0; p < 3; ++p)
          *reinterpret_cast<U4 *>(to + p * BX * BK) = U4{part[p][0], part[p][1], part[p][2], part[p][3]};
      }
    }
  }

  // 8 k (16 kk + 8 (lane / 32) + 0..7) of m = base + lane % 32.
  static __device__ __forceinline__ S8 take(const uint16_t *lds, int part, int base, int kk) {
    const int lane = threadIdx.x & 63;
    lds += part * BX * BK;
    if constexpr (KMajor) {
      const int row = base + (lane & 31);
      return *reinterpret_cast<const S8 *>(lds + row * BK + (((kk * 2 + (lane >> 5)) ^ shift_k(row)) * 8));
    } else {
      typedef __attribute__((address_space(3))) S4 Shared;
      const int k = kk * 16 + 8 * (lane >> 5) + (lane & 15) / 4;
      const int pair = base / 16 + ((lane >> 4) & 1);
      const uint16_t *const from = lds + k * BX + ((pair ^ shift_m(k)) * 16) + (lane & 3) * 4;
      const S4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Shared *)(from));
      const S4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Shared *)(from + 4 * BX));
      return S8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    }
  }
};

// Where the entries of the result go, 8 along a row at a time.
template <typename T>
__device__ __forceinline__ void put_forward(const ForwardOut &f, int64_t row, int col, int count, float (&v)[8], bool head) {
  if (f.bias != nullptr && count > 0) {
    float b[8];
    Entries<F32, 8>::load(f.bias + col, count, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += b[i];
  }
  if (f.z.data != nullptr) {
    if (f.z_packed) store_packed<T, 8>(f.z, row, col, count, v, head, 4);
    else if (count > 0) Entries<T, 8>::store(static_cast<typename T::Store *>(f.z.data) + row * f.z.ld + col, count, v);
  }
  with_activation(f.act, [&](auto a) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = decltype(a)::value(v[i]);
  });
  if (f.residual.data != nullptr && count > 0) {
    float r[8];
    Entries<T, 8>::load(static_cast<const typename T::Store *>(f.residual.data) + row * f.residual.ld + col, count, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += r[i];
  }
  if (f.y8.data != nullptr) {  // entries past the last column are not part of their group
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < count ? v[i] : 0.f;
    store_packed<T, 8>(f.y8, row, col, count, v, head, 4);
  }
  if (count > 0) Entries<T, 8>::store(static_cast<typename T::Store *>(f.y.data) + row * f.y.ld + col, count, v);
}

template <typename T, int BX, ProductKind Kind, ProductOut Out>
__global__ __launch_bounds__(256, 2) void product_kernel(const ProductArgs g) {
  constexpr int BK = ProductDepth<T>::value(BX == 64);
  constexpr bool a_k = Kind == kProductForward || Kind == kProductDx, b_k = Kind == kProductForward;
  typedef Tile<T, BX, BK, a_k, false> TA;
  typedef Tile<T, BX, BK, b_k, Kind == kProductDwPacked> TB;
  constexpr int W = BX / 2, R = W / 32;          // a wavefront's square of the tile, and its 32 x 32 blocks a side
  constexpr int kBuffer = (TA::kBytes + TB::kBytes) / 2;
  constexpr int kPitch = W + 8;                  // floats in a row of a wavefront's slab of the result
  constexpr int kSlab = 32 * kPitch;
  constexpr int kLds = 2 * kBuffer * 2 > 4 * kSlab * 4 ? 2 * kBuffer * 2 : 4 * kSlab * 4;
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLds / 2];

  // Workgroups go round the 8 XCDs: each XCD gets a contiguous run of tiles, those of the same rows next to each other,
  // so that they share its L2.
  const int total = g.tiles_m * g.tiles_n * g.splits;
  int id = blockIdx.x;
  if (id < total / 8 * 8) id = id % 8 * (total / 8) + id / 8;
  const int tn = id % g.tiles_n, tm = id / g.tiles_n % g.tiles_m, split = id / g.tiles_n / g.tiles_m;
  const int64_t m0 = static_cast<int64_t>(tm) * BX, n0 = static_cast<int64_t>(tn) * BX;
  const int64_t k0 = split * g.k_per_split, k1 = k0 + g.k_per_split < g.K ? k0 + g.k_per_split : g.K;
  const int steps = static_cast<int>((k1 - k0 + BK - 1) / BK);

  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
  const int wm = wave / 2 * W, wn = wave % 2 * W;
  F16x acc[R][R];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < R; ++j) acc[i][j] = F16x{};

  // The last step's chunks may be short: along k where K is no multiple of 8; along m the very last row of memory ends
  // inside its last chunk, of which the hardware's bounds check drops a dword that is only half there.
  const bool ragged_a = a_k ? k1 % 8 != 0 : g.M % 8 != 0, ragged_b = b_k ? k1 % 8 != 0 : g.N % 8 != 0;
  TA a;
  TB b;
  if (steps > 0) {
    a.fetch(g.a, m0, g.M, k0, k1, steps == 1 && ragged_a);
    b.fetch(g.b, n0, g.N, k0, k1, steps == 1 && ragged_b);
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
      b.fetch(g.b, n0, g.N, k, k1, last && ragged_b);
    }
#pragma unroll
    for (int kk = 0; kk < BK / 16; ++kk) {
      S8 fa[TA::kParts][R], fb[TB::kParts][R];
#pragma unroll
      for (int p = 0; p < TA::kParts; ++p)
#pragma unroll
        for (int i = 0; i < R; ++i) fa[p][i] = TA::take(now, p, wm + 32 * i, kk);
#pragma unroll
      for (int p = 0; p < TB::kParts; ++p)
#pragma unroll
        for (int i = 0; i < R; ++i) fb[p][i] = TB::take(now + TA::kBytes / 2, p, wn + 32 * i, kk);
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

  // Through LDS into rows: a lane of the accumulators holds entries of one column.
  float *const slab = reinterpret_cast<float *>(lds) + wave * kSlab;
  constexpr int kLanes = W / 8;  // lanes of a row
#pragma unroll
  for (int i = 0; i < R; ++i) {
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        slab[(8 * (r / 4) + 4 * (lane >> 5) + r % 4) * kPitch + 32 * j + (lane & 31)] = acc[i][j][r];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int pass = 0; pass < 32 * kLanes / 64; ++pass) {
      const int r = pass * (64 / kLanes) + lane / kLanes, c = lane % kLanes * 8;
      const int64_t row = m0 + wm + 32 * i + r;
      const int64_t col = n0 + wn + c;
      const int64_t left = row < g.M ? g.N - col : 0;
      const int count = static_cast<int>(left < 0 ? 0 : left > 8 ? 8 : left);
      float v[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const F4 x = *reinterpret_cast<const F4 *>(slab + r * kPitch + c + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = x[e];
      }
      if constexpr (Out == kForward) {
        // entries that are not there count in no group
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < count ? v[e] : 0.f;
        put_forward<T>(g.forward, row, static_cast<int>(col), count, v, (lane & 3) == 0);
      } else if constexpr (Out == kStore) {
        if (count > 0)
          Entries<T, 8>::store(static_cast<typename T::Store *>(g.out.data) + row * g.out.ld + col, count, v);
      } else {
        if (count > 0) Entries<F32, 8>::store(g.parts + (split * g.M + row) * g.N + col, count, v);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename T, int BX, ProductKind Kind, ProductOut Out>
int launch_one(const ProductArgs &g, hipStream_t st) {
  const unsigned blocks = static_cast<unsigned>(g.tiles_m) * g.tiles_n * g.splits;
  product_kernel<T, BX, Kind, Out><<<dim3(blocks), dim3(256), 0, st>>>(g);
  return check_launch("matrix product");
}

template <typename T, int BX>
int launch_sized(ProductKind kind, const ProductArgs &g, hipStream_t st) {
  switch (kind) {
    case kProductForward: return launch_one<T, BX, kProductForward, kForward>(g, st);
    case kProductDx: return launch_one<T, BX, kProductDx, kStore>(g, st);
    case kProductDw: return launch_one<T, BX, kProductDw, kParts>(g, st);
    default: return launch_one<T, BX, kProductDwPacked, kParts>(g, st);
  }
}

}  // namespace gosh
