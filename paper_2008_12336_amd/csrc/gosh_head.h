// Shared by the units of the head (layer norm, linear layers, 8-bit activations): views of matrices, their checks,
// the element types and the 8-bit form.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "gosh_common.h"

namespace gosh {

// ---- host: arguments --------------------------------------------------------------------

enum MatUse : int { kMayBePacked = 1, kMustBePacked = 2, kOptional = 4 };

inline bool rows_fit(int64_t rows) { return rows >= 0 && rows < 2147483647LL; }
// A matrix argument: its fields, and that its memory is there.  GOSH_OK also for an optional one that is null.
int check_mat(const gosh_mat *m, const char *what, int use = 0);
// Two matrices of one shape, or GOSH_EINVAL.
int check_shape(const gosh_mat *m, const char *what, int64_t rows, int32_t cols);
int check_type(const gosh_mat *m, const char *what, int32_t type);
int check_floats(const float *p, int64_t count, const char *what, bool optional);
int check_workspace(const void *p, uint64_t have, uint64_t need);
// Up to three sums of partial results in one launch.  A job sums `count` arrays of n floats, each `stride` floats after the
// one before, in an order that depends on these numbers alone (the same bits every time), into out: rows of `cols`
// entries of `type`, ld apart.
struct JoinJob {
  const float *parts;
  int64_t stride, n, ld;
  void *out;
  int32_t count, cols, type;
};
int join_parts(const JoinJob *jobs, int how_many, hipStream_t st);

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- device: element types --------------------------------------------------------------

typedef float F4 __attribute__((ext_vector_type(4)));
typedef uint32_t U4 __attribute__((ext_vector_type(4)));
typedef uint32_t U2 __attribute__((ext_vector_type(2)));

struct F32 {
  typedef float Store;
  static constexpr int32_t kType = GOSH_F32;
  static __device__ __forceinline__ float up(float v) { return v; }
  static __device__ __forceinline__ float down(float v) { return v; }
};
struct Bf16 {
  typedef __bf16 Store;
  static constexpr int32_t kType = GOSH_BF16;
  static __device__ __forceinline__ float up(__bf16 v) { return static_cast<float>(v); }
  static __device__ __forceinline__ __bf16 down(float v) { return static_cast<__bf16>(v); }
};
struct F16 {
  typedef _Float16 Store;
  static constexpr int32_t kType = GOSH_F16;
  static __device__ __forceinline__ float up(_Float16 v) { return static_cast<float>(v); }
  static __device__ __forceinline__ _Float16 down(float v) { return static_cast<_Float16>(v); }
};

// Memory that need not be aligned to what is read from it: the hardware takes accesses of up to 128 bits at any multiple
// of an entry's size, so there is no second path for odd strides.
template <typename U, int Align>
struct Loosely {
  typedef U At __attribute__((aligned(Align)));
};
template <int N>
struct Words {
  typedef uint32_t V __attribute__((ext_vector_type(N)));
};
template <>
struct Words<1> {
  typedef uint32_t V;
};

// `Bytes` bytes at p (aligned to Align) of which the first `there` are loaded, in pieces of powers of two (never past
// them); the others are zero.  Likewise the store.
template <int Bytes, int Align>
struct Span {
  static constexpr int kWords = Bytes / 4;
  typedef typename Words<kWords>::V V;
  typedef typename Loosely<uint16_t, Align>::At Half;
  typedef typename Loosely<uint32_t, Align>::At One;
  typedef typename Loosely<typename Words<2>::V, Align>::At Two;
  typedef typename Loosely<typename Words<4>::V, Align>::At Four;

  static __device__ __forceinline__ V load(const void *p, int there) {
    const char *const c = static_cast<const char *>(p);
    if (there >= Bytes) {
      if constexpr (kWords <= 4) {
        return *reinterpret_cast<const typename Loosely<V, Align>::At *>(p);
      } else {
        const Four lo = *reinterpret_cast<const Four *>(p), hi = *reinterpret_cast<const Four *>(c + 16);
        return V{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      }
    }
    there = there < 0 ? 0 : there;
    // all loads first
    typename Words<4>::V w4 = 0;
    typename Words<2>::V w2 = 0;
    uint32_t w1 = 0, half = 0, low = 0;
    if constexpr (kWords > 4)
      if (there & 16) w4 = *reinterpret_cast<const Four *>(c);
    if constexpr (kWords > 2)
      if (there & 8) w2 = *reinterpret_cast<const Two *>(c + (there & ~15));
    if constexpr (kWords > 1)
      if (there & 4) w1 = *reinterpret_cast<const One *>(c + (there & ~7));
    if constexpr (Align <= 2)
      if (there & 2) half = *reinterpret_cast<const Half *>(c + (there & ~3));
    if constexpr (Align <= 1)
      if (there & 1) low = static_cast<uint8_t>(c[there & ~1]);
    const uint32_t last = Align <= 2 && (there & 2) ? half | low << 16 : low;
    if constexpr (kWords == 1) {
      return last;
    } else if constexpr (kWords == 2) {
      return (there & 4) ? V{w1, last} : V{last, 0};
    } else {
      const uint32_t a = (there & 4) ? w1 : last, b = (there & 4) ? last : 0;
      if constexpr (kWords == 4) {
        return (there & 8) ? V{w2[0], w2[1], a, b} : V{a, b, 0, 0};
      } else {
        const uint32_t d = (there & 8) ? w2[0] : a, e = (there & 8) ? w2[1] : b;
        const uint32_t f = (there & 8) ? a : 0, g = (there & 8) ? b : 0;
        return (there & 16) ? V{w4[0], w4[1], w4[2], w4[3], d, e, f, g} : V{d, e, f, g, 0, 0, 0, 0};
      }
    }
  }
  // Past: of what the caches need not keep.
  template <bool Past = false>
  static __device__ __forceinline__ void store(void *p, int there, V u) {
    char *c = static_cast<char *>(p);
    if (there >= Bytes) {
      if constexpr (kWords <= 4) {
        typedef typename Loosely<V, Align>::At At;
        if constexpr (Past) __builtin_nontemporal_store(u, static_cast<At *>(p));
        else *static_cast<At *>(p) = u;
      } else {
        *reinterpret_cast<Four *>(p) = Four{u[0], u[1], u[2], u[3]};
        *reinterpret_cast<Four *>(c + 16) = Four{u[4], u[5], u[6], u[7]};
      }
      return;
    }
    there = there < 0 ? 0 : there;
    uint32_t a, b = 0;  // the words of which a part is there, as pieces are taken off
    if constexpr (kWords == 1) {
      a = u;
    } else {
      a = u[0], b = u[1];
      uint32_t d = 0, e = 0;
      if constexpr (kWords >= 4) d = u[2], e = u[3];
      if constexpr (kWords > 4) {
        if (there & 16) *reinterpret_cast<Four *>(c) = Four{u[0], u[1], u[2], u[3]};
        if (there & 16) a = u[4], b = u[5], d = u[6], e = u[7];
      }
      if constexpr (kWords > 2) {
        if (there & 8) *reinterpret_cast<Two *>(c + (there & ~15)) = Two{a, b};
        if (there & 8) a = d, b = e;
      }
      if (there & 4) *reinterpret_cast<One *>(c + (there & ~7)) = a;
      if (there & 4) a = b;
    }
    if constexpr (Align <= 2) {
      if (there & 2) *reinterpret_cast<Half *>(c + (there & ~3)) = static_cast<uint16_t>(a);
      if (there & 2) a >>= 16;
    }
    if constexpr (Align <= 1)
      if (there & 1) c[there & ~1] = static_cast<char>(a);
  }
};

// N entries in a row of memory.
template <typename T, int N>
struct Entries {
  typedef typename T::Store S;
  typedef S Vec __attribute__((ext_vector_type(N)));
  typedef Span<N * sizeof(S), sizeof(S)> Memory;
  // The first `count` of N; the others are zero.
  static __device__ __forceinline__ Vec fetch(const S *p, int count) {
    return __builtin_bit_cast(Vec, Memory::load(p, count * static_cast<int>(sizeof(S))));
  }
  static __device__ __forceinline__ void load(const S *p, int count, float (&v)[N]) {
    const Vec x = fetch(p, count);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = T::up(x[i]);
  }
  template <bool Past = false>
  static __device__ __forceinline__ void store(S *p, int count, const float (&v)[N]) {
    Vec x;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = T::down(v[i]);
    Memory::template store<Past>(p, count * static_cast<int>(sizeof(S)), __builtin_bit_cast(typename Memory::V, x));
  }
};

// ---- device: the 8-bit form -------------------------------------------------------------

constexpr int kGroup = 32;          // columns that share an exponent
constexpr uint32_t kNotFinite = 255;

// The exponent byte of a group whose largest magnitude has the bits `most`: with that magnitude = f * 2^E, f in [1, 2),
// the smallest e with 64 f <= 127 * 2^(e + 6 - E) is E - 6, or E - 5 from f > 127/64 on, which the carry decides.
template <typename T>
__device__ __forceinline__ uint32_t exponent_byte(uint32_t most) {
  // what rounds to infinity in T, and infinities and NaN themselves
  constexpr uint32_t too_big = T::kType == GOSH_F32 ? 0x7f800000u : T::kType == GOSH_BF16 ? 0x7f7f8000u : 0x477ff000u;
  constexpr uint32_t low = T::kType == GOSH_F16 ? 127 - 24 : 1;
  if (most >= too_big) return kNotFinite;
  const uint32_t e = (most + 0x1ffffu) >> 23;
  return e < low + 6 ? low : e - 6;
}

// 2^(byte - 127); byte 1 to 254.
__device__ __forceinline__ float unit_of(uint32_t byte) { return __uint_as_float(byte << 23); }
// What an entry of a group is multiplied by: NaN for one that stands for NaN.
__device__ __forceinline__ float read_unit(uint32_t byte) {
  return byte == kNotFinite ? __uint_as_float(0x7fc00000u) : unit_of(byte);
}
// 2^(127 - byte).
__device__ __forceinline__ float inverse_unit(uint32_t byte) {
  return byte <= 253 ? __uint_as_float((254 - byte) << 23) : 0.f;
}
// The unit at which 64 of them leave T.
template <typename T>
__device__ __forceinline__ float top_of(uint32_t byte) {
  constexpr uint32_t top = T::kType == GOSH_F16 ? 137 : 249;
  return byte >= top ? 63.f : 127.f;
}

// N entries' q as bytes of words, from entries in 32 bits.  top = top_of.  v / unit is exact, and its sum with 1.5 * 2^23
// rounds it once, to the nearest whole number (ties to even), whose low byte is the sum's.
template <int N>
__device__ __forceinline__ void quantise(const float (&v)[N], uint32_t byte, float top, uint32_t (&q)[N / 4]) {
  constexpr float kWhole = 12582912.f;
  const float inv = inverse_unit(byte);
  const uint32_t finite = byte == kNotFinite ? 0 : ~0u;
#pragma unroll
  for (int w = 0; w < N / 4; ++w) {
    uint32_t n[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      n[i] = __float_as_uint(__builtin_amdgcn_fmed3f(__builtin_fmaf(v[4 * w + i], inv, kWhole), kWhole - top, kWhole + top));
    const uint32_t lo = __builtin_amdgcn_perm(n[1], n[0], 0x0c0c0400), hi = __builtin_amdgcn_perm(n[3], n[2], 0x04000c0c);
    q[w] = (lo | hi) & finite;
  }
}

// The largest magnitude, as bits, of N entries and of those of the other lanes of a group of `lanes` (1, 2, 4 or 8).
// Bits order as magnitudes do, with infinity and then NaN on top.
template <int Swap>
__device__ __forceinline__ uint32_t larger_of_lanes(uint32_t x) {
  return max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), Swap, 0xf, 0xf, true)));
}
template <int N>
__device__ __forceinline__ uint32_t most_bits(const float (&v)[N], int lanes) {
  float largest = 0.f;  // or a NaN, which this maximum keeps
#pragma unroll
  for (int i = 0; i < N; ++i) largest = __builtin_elementwise_maximum(largest, __builtin_fabsf(v[i]));
  uint32_t most = __float_as_uint(largest) & 0x7fffffffu;
  if (lanes > 1) most = larger_of_lanes<0xb1>(most);   // the other lane of two
  if (lanes > 2) most = larger_of_lanes<0x4e>(most);   // the other two of four
  if (lanes > 4) most = larger_of_lanes<0x141>(most);  // one of the other four of eight: the half row mirrored
  return most;
}

// count of N bytes at p (any alignment).
template <int N>
__device__ __forceinline__ void store_bytes(int8_t *p, int count, const uint32_t (&q)[N / 4]) {
  if constexpr (N == 4) Span<4, 1>::store(p, count, q[0]);
  else Span<8, 1>::store(p, count, U2{q[0], q[1]});
}
template <int N>
__device__ __forceinline__ void load_bytes(const int8_t *p, int count, uint32_t (&q)[N / 4]) {
  if constexpr (N == 4) {
    q[0] = Span<4, 1>::load(p, count);
  } else {
    const U2 w = Span<8, 1>::load(p, count);
    q[0] = w[0], q[1] = w[1];
  }
}
template <int N>
__device__ __forceinline__ void widen(const uint32_t (&q)[N / 4], float unit, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
    v[i] = static_cast<float>(static_cast<int32_t>(q[i / 4] << (24 - 8 * (i % 4))) >> 24) * unit;
}

// A matrix as a kernel sees it.
struct Plane {
  void *data;
  uint8_t *exps;
  int64_t ld, ld_exps;
};
inline Plane plane_of(const gosh_mat *m) {
  return m == nullptr ? Plane{nullptr, nullptr, 0, 0} : Plane{m->data, m->exps, m->ld, m->ld_exps};
}
inline Plane rows_from(Plane p, int64_t row, int32_t type, bool packed) {
  if (p.data == nullptr) return p;
  p.data = static_cast<char *>(p.data) + row * p.ld * (packed ? 1 : type == GOSH_F32 ? 4 : 2);
  if (packed) p.exps += row * p.ld_exps;
  return p;
}

// N entries at (row, col), of which `count` are there, from a matrix that may be packed.
template <typename T, int N>
__device__ __forceinline__ void load_entries(const Plane &m, bool packed, int64_t row, int col, int count, float (&v)[N]) {
  if (packed) {
    uint32_t q[N / 4];
    load_bytes<N>(static_cast<const int8_t *>(m.data) + row * m.ld + col, count, q);
    widen<N>(q, count > 0 ? read_unit(m.exps[row * m.ld_exps + col / kGroup]) : 0.f, v);
  } else {
    Entries<T, N>::load(static_cast<const typename T::Store *>(m.data) + row * m.ld + col, count, v);
  }
}

// N entries into a packed matrix, at p and the exponent at e, by the lanes of a group together: kGroup / N of them, or
// fewer where `lanes` says so, hold a group's columns.  Entries past `count` are zero.  Every lane of the group calls it.
template <typename T, int N>
__device__ __forceinline__ void store_packed(int8_t *p, uint8_t *e, int count, const float (&v)[N], bool first_of_group, int lanes) {
  const uint32_t byte = exponent_byte<T>(most_bits<N>(v, lanes));
  if (count <= 0) return;
  uint32_t q[N / 4];
  quantise<N>(v, byte, top_of<T>(byte), q);
  store_bytes<N>(p, count, q);
  if (first_of_group) *e = static_cast<uint8_t>(byte);
}
// The same at (row, col).
template <typename T, int N>
__device__ __forceinline__ void store_packed(const Plane &m, int64_t row, int col, int count, const float (&v)[N],
                                             bool first_of_group, int lanes) {
  store_packed<T, N>(static_cast<int8_t *>(m.data) + row * m.ld + col, m.exps + row * m.ld_exps + col / kGroup, count, v,
                     first_of_group, lanes);
}

// ---- device: activations ----------------------------------------------------------------

template <int Act>
struct Activation;

constexpr float kLog2E = 1.4426950408889634f;
// The logistic function of -x / kLog2E.
__device__ __forceinline__ float logistic2(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x)); }
__device__ __forceinline__ float logistic(float x) { return logistic2(-kLog2E * x); }

template <>
struct Activation<GOSH_ACT_NONE> {
  static __device__ __forceinline__ float value(float z) { return z; }
  static __device__ __forceinline__ float slope(float) { return 1.f; }
};
template <>
struct Activation<GOSH_ACT_RELU> {  // a NaN stays one
  static __device__ __forceinline__ float value(float z) { return z <= 0.f ? 0.f : z; }
  static __device__ __forceinline__ float slope(float z) { return z <= 0.f ? 0.f : z != z ? z : 1.f; }
};
template <>
struct Activation<GOSH_ACT_SILU> {
  static __device__ __forceinline__ float value(float z) { return z * logistic(z); }
  // beyond +-88 the slope is 1 or 0 to the last bit, and an infinity times the zero of s (1 - s) would be NaN
  static __device__ __forceinline__ float slope(float z) {
    z = z > 88.f ? 88.f : z < -88.f ? -88.f : z;
    const float s = logistic(z);
    return s + z * s * (1.f - s);
  }
};
template <>
struct Activation<GOSH_ACT_GELU> {
  static constexpr float kC = 1.5957691216057308f;             // 2 sqrt(2/pi)
  static constexpr float kD = 1.5957691216057308f * 0.044715f;
  static __device__ __forceinline__ float value(float z) { return z * logistic2(z * (-kLog2E * kC + -kLog2E * kD * (z * z))); }
  static __device__ __forceinline__ float slope(float z) {
    z = z > 12.f ? 12.f : z < -12.f ? -12.f : z;  // as above
    const float s = logistic(z * (kC + kD * z * z));
    return s + z * s * (1.f - s) * (kC + 3.f * kD * z * z);
  }
};

// Calls f with the activation as a type: the branch is taken once, outside the loops.
template <typename F>
__device__ __forceinline__ void with_activation(int act, F f) {
  switch (act) {
    case GOSH_ACT_RELU: f(Activation<GOSH_ACT_RELU>{}); break;
    case GOSH_ACT_GELU: f(Activation<GOSH_ACT_GELU>{}); break;
    case GOSH_ACT_SILU: f(Activation<GOSH_ACT_SILU>{}); break;
    default: f(Activation<GOSH_ACT_NONE>{}); break;
  }
}

}  // namespace gosh
