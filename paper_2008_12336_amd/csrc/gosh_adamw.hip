// AdamW over many tensors at once, moments in 8 or 32 bits.
//
// Tensors are cut into chunks of 2,048 entries, a workgroup each, found by a table in device memory that the optimiser was
// made with: one launch, however many tensors.  A thread has 8 entries, 16 threads a block of 128 that shares an exponent:
// its largest magnitude is joined by lane exchanges in registers, so that each array is read once and written once.  Bound by
// memory: 2^27 entries with 32-bit gradients and 8-bit moments (16 bytes each) 392 us, 5.5 TB/s; 50,000,017 with 16-bit gradients
// and copies and 32-bit moments (28 bytes) 260 us, 5.4 TB/s; 192 tensors of 3,000,000 entries in all 11.8.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <memory>
#include <new>
#include <vector>

#include "gosh_head.h"

namespace gosh {
namespace {

constexpr int kBlock = 128;   // entries that share an exponent
// Entries of a workgroup, eight a thread.  2^27 entries in 8 bits: 391 us, 411 with chunks of 4,096 and 425 of 8,192; 192
// tensors of 3,000,000 in all: 11.8, 15.4 and 16.9.
constexpr int kChunk = 2048;
constexpr int kThreads = 256;
constexpr int64_t kMostEntries = int64_t{1} << 40;

int64_t padded(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Where the parts of a state begin, in bytes.
struct StateLayout {
  int64_t v, m_exps, v_exps, bytes;
};
StateLayout layout_of(int64_t n, int32_t bits) {
  StateLayout l{};
  if (bits == 32) {
    l.v = padded(4 * n, 16);
    l.bytes = l.v + 4 * n;
    return l;
  }
  const int64_t blocks = ceil_div(n, kBlock);
  l.v = padded(n, 16);
  l.m_exps = 2 * l.v;
  l.v_exps = l.m_exps + padded(blocks, 16);
  l.bytes = l.v_exps + blocks;
  return l;
}

struct Tensor {
  float *p;
  const void *g;
  char *state;
  void *copy;
  int64_t n, flat;  // flat: where it begins in flat arrays
  int64_t v, m_exps, v_exps;
  int32_t g_type, copy_type, bits;
  float decay;
};
struct Chunk {
  int32_t tensor, index;  // of the tensor's chunks
};

struct Optimiser {
  int device = 0;
  Tensor *tensors = nullptr;  // device
  Chunk *chunks = nullptr;    // device
  int64_t count = 0;          // of chunks
  int64_t entries = 0;        // of a flat array
};

// ---- 8-bit moments ------------------------------------------------------------------------------

constexpr uint32_t kLowestByte = 32;  // 2^-95: the least number of v, 2^-33 of it, is still one in 32 bits

// The exponent byte of a block whose largest magnitude has the bits `most`: f * 2^E, f in [1, 2), takes E, or E + 1 from
// f > 1.875 on, which the carry decides.
__device__ __forceinline__ uint32_t moment_byte(uint32_t most) {
  const uint32_t e = (most + 0x0fffffu) >> 23;
  return e > 253 ? kNotFinite : e < kLowestByte ? kLowestByte : e;
}
// What puts the least number with a leading one (2^-14 or 2^-30) at 2^-126, so that the bits of a float from the third of its
// mantissa up are the code, also below where both have no leading one.
template <bool Second>
struct Moment {
  static constexpr float kDown = Second ? 0x1p-96f : 0x1p-112f, kUp = Second ? 0x1p96f : 0x1p112f;
  static __device__ __forceinline__ float read(uint32_t code, float unit) {
    const uint32_t number = Second ? code : code & 127u;
    const float x = (__uint_as_float(number << 20) * kUp) * unit;
    return Second ? x : __uint_as_float(__float_as_uint(x) | (code & 128u) << 24);
  }
  // add: 20 bits.
  static __device__ __forceinline__ uint32_t write(float x, float inverse, uint32_t add) {
    const uint32_t number = (__float_as_uint(__builtin_fabsf(x) * inverse * kDown) + add) >> 20;
    // a second moment over 0 stays so: as 0 it would let the next update grow to the root of 1 / (1 - beta2) of the rate
    return Second ? (x > 0.f && number == 0 ? 1u : number) : number | (__float_as_uint(x) >> 24 & 128u);
  }
};

// Multiples of the golden ratio over the entries and of the root of 2 over the steps: both spread evenly, along either.
__device__ __forceinline__ uint32_t spread(int64_t i, uint32_t t) {
  return static_cast<uint32_t>(i) * 2654435769u + t * 1779033703u;
}

// The largest magnitude of 16 lanes' entries, as bits.
template <int N>
__device__ __forceinline__ uint32_t most_of_block(const float (&v)[N]) {
  uint32_t most = most_bits<N>(v, 8);
  return larger_of_lanes<0x140>(most);  // one of the other eight of 16: the row mirrored
}

// ---- the step -------------------------------------------------------------------------------------

struct StepArgs {
  float beta1, rest1, beta2, rest2, eps, lr, log1, log2;
  float rate, root;  // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  int64_t t;
  const float *lr_dev, *scale;
  const int64_t *steps;
};

// The 8 entries of a lane.
struct Step {
  float rate, root, eps, keep;  // keep: 1 - lr * decay
};

constexpr int kEach = 8;

// Rounded operation by operation, so that the state is what the formulas give in 32 bits.
__device__ __forceinline__ float moment1(const StepArgs &a, float m, float g) {
#pragma clang fp contract(off)
  return a.beta1 * m + a.rest1 * g;
}
__device__ __forceinline__ float moment2(const StepArgs &a, float v, float g) {
#pragma clang fp contract(off)
  return a.beta2 * v + (a.rest2 * g) * g;
}

template <typename G>
__device__ __forceinline__ void load_gradients(const Tensor &t, int64_t i, int count, float scale, float (&g)[kEach]) {
  Entries<G, kEach>::load(static_cast<const typename G::Store *>(t.g) + i, count, g);
#pragma unroll
  for (int e = 0; e < kEach; ++e) g[e] *= scale;
}

template <int Bits>
__device__ __forceinline__ void load_moments(const Tensor &t, int64_t i, int count, float (&m)[kEach], float (&v)[kEach]) {
  if constexpr (Bits == 32) {
    Entries<F32, kEach>::load(reinterpret_cast<const float *>(t.state) + i, count, m);
    Entries<F32, kEach>::load(reinterpret_cast<const float *>(t.state + t.v) + i, count, v);
  } else {
    uint32_t qm[2], qv[2];
    load_bytes<kEach>(reinterpret_cast<const int8_t *>(t.state) + i, count, qm);
    load_bytes<kEach>(reinterpret_cast<const int8_t *>(t.state + t.v) + i, count, qv);
    const int64_t b = i / kBlock;
    const float um = count > 0 ? read_unit(static_cast<uint8_t>(t.state[t.m_exps + b])) : 0.f;
    const float uv = count > 0 ? read_unit(static_cast<uint8_t>(t.state[t.v_exps + b])) : 0.f;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      m[e] = Moment<false>::read(qm[e / 4] >> 8 * (e % 4) & 255u, um);
      v[e] = Moment<true>::read(qv[e / 4] >> 8 * (e % 4) & 255u, uv);
    }
  }
}

// All 16 lanes of a block call it.  Nearest: to the nearest, ties to even, in place of the sequence.
template <int Bits, bool Nearest>
__device__ __forceinline__ void store_moments(const Tensor &t, int64_t i, int count, const float (&m)[kEach], const float (&v)[kEach],
                                              uint32_t step) {
  if constexpr (Bits == 32) {
    if (count <= 0) return;
    Entries<F32, kEach>::store(reinterpret_cast<float *>(t.state) + i, count, m);
    Entries<F32, kEach>::store(reinterpret_cast<float *>(t.state + t.v) + i, count, v);
  } else {
    const uint32_t bm = moment_byte(most_of_block(m)), bv = moment_byte(most_of_block(v));
    if (count <= 0) return;
    const float im = inverse_unit(bm), iv = inverse_unit(bv);
    uint32_t qm[2] = {0, 0}, qv[2] = {0, 0};
    const uint32_t h0 = spread(i, step);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      uint32_t am, av;
      if constexpr (Nearest) {
        am = 0x7ffffu + (__float_as_uint(__builtin_fabsf(m[e]) * im * Moment<false>::kDown) >> 20 & 1u);
        av = 0x7ffffu + (__float_as_uint(__builtin_fabsf(v[e]) * iv * Moment<true>::kDown) >> 20 & 1u);
      } else {
        const uint32_t h = h0 + static_cast<uint32_t>(e) * 2654435769u;
        am = h >> 12, av = ~h >> 12;
      }
      qm[e / 4] |= (Moment<false>::write(m[e], im, am) & 255u) << 8 * (e % 4);
      qv[e / 4] |= (Moment<true>::write(v[e], iv, av) & 255u) << 8 * (e % 4);
    }
    store_bytes<kEach>(reinterpret_cast<int8_t *>(t.state) + i, count, qm);
    store_bytes<kEach>(reinterpret_cast<int8_t *>(t.state + t.v) + i, count, qv);
    if (i % kBlock == 0) {
      t.state[t.m_exps + i / kBlock] = static_cast<char>(bm);
      t.state[t.v_exps + i / kBlock] = static_cast<char>(bv);
    }
  }
}

template <typename G, int Bits>
__device__ __forceinline__ void step_chunk(const Tensor &t, int64_t first, const StepArgs &a, const Step &s, uint32_t number, float scale) {
  for (int at = static_cast<int>(threadIdx.x) * kEach; at < kChunk; at += kThreads * kEach) {
    const int64_t i = first + at;
    const int count = i >= t.n ? 0 : t.n - i < kEach ? static_cast<int>(t.n - i) : kEach;
    float p[kEach], g[kEach], m[kEach], v[kEach];
    load_gradients<G>(t, i, count, scale, g);
    Entries<F32, kEach>::load(t.p + i, count, p);
    load_moments<Bits>(t, i, count, m, v);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      m[e] = moment1(a, m[e], g[e]);
      v[e] = moment2(a, v[e], g[e]);
      p[e] = p[e] * s.keep - s.rate * m[e] / (sqrtf(v[e]) * s.root + s.eps);
    }
    store_moments<Bits, false>(t, i, count, m, v, number);
    if (count <= 0) continue;
    Entries<F32, kEach>::store(t.p + i, count, p);
    if (t.copy == nullptr) continue;
    if (t.copy_type == GOSH_BF16) Entries<Bf16, kEach>::store(static_cast<__bf16 *>(t.copy) + i, count, p);
    else Entries<F16, kEach>::store(static_cast<_Float16 *>(t.copy) + i, count, p);
  }
}

__global__ __launch_bounds__(kThreads) void step_kernel(const Tensor *tensors, const Chunk *chunks, const StepArgs a) {
  const Chunk c = chunks[blockIdx.x];
  const Tensor t = tensors[c.tensor];
  float scale = 1.f, lr = a.lr, rate = a.rate, root = a.root;
  uint32_t number = static_cast<uint32_t>(a.t);
  if (a.scale != nullptr) {
    scale = *a.scale;
    if (!(__builtin_fabsf(scale) < INFINITY)) return;
  }
  if (a.lr_dev != nullptr) lr = *a.lr_dev;
  if (a.steps != nullptr || a.lr_dev != nullptr) {
    const int64_t n = a.steps != nullptr ? *a.steps + 1 : a.t;
    number = static_cast<uint32_t>(n);
    // 1 - beta^t = -(e^(t log beta) - 1), which loses nothing where t log beta is small
    rate = lr / -expm1f(static_cast<float>(n) * a.log1);
    root = 1.f / sqrtf(-expm1f(static_cast<float>(n) * a.log2));
  }
  const Step s{rate, root, a.eps, 1.f - lr * t.decay};
  const int64_t first = static_cast<int64_t>(c.index) * kChunk;
  if (t.bits == 8) {
    if (t.g_type == GOSH_F32) step_chunk<F32, 8>(t, first, a, s, number, scale);
    else if (t.g_type == GOSH_BF16) step_chunk<Bf16, 8>(t, first, a, s, number, scale);
    else step_chunk<F16, 8>(t, first, a, s, number, scale);
  } else {
    if (t.g_type == GOSH_F32) step_chunk<F32, 32>(t, first, a, s, number, scale);
    else if (t.g_type == GOSH_BF16) step_chunk<Bf16, 32>(t, first, a, s, number, scale);
    else step_chunk<F16, 32>(t, first, a, s, number, scale);
  }
}

// Behind the step: its number has been read by then.
__global__ void count_kernel(int64_t *steps, const float *scale) {
  if (scale == nullptr || __builtin_fabsf(*scale) < INFINITY) *steps += 1;
}

// Moments to flat arrays of To and, with them as the source, back.
template <typename To, bool Back>
__global__ __launch_bounds__(kThreads) void moments_kernel(const Tensor *tensors, const Chunk *chunks, typename To::Store *m_flat,
                                                           typename To::Store *v_flat) {
  const Chunk c = chunks[blockIdx.x];
  const Tensor t = tensors[c.tensor];
  const int64_t end = (t.n + kBlock - 1) / kBlock * kBlock;
  for (int at = static_cast<int>(threadIdx.x) * kEach; at < kChunk; at += kThreads * kEach) {
    const int64_t i = static_cast<int64_t>(c.index) * kChunk + at;
    if (i >= end) return;  // the 16 lanes of a block together
    const int count = i >= t.n ? 0 : t.n - i < kEach ? static_cast<int>(t.n - i) : kEach;
    float m[kEach], v[kEach];
    if constexpr (Back) {
      Entries<To, kEach>::load(m_flat + t.flat + i, count, m);
      Entries<To, kEach>::load(v_flat + t.flat + i, count, v);
      if (t.bits == 8) store_moments<8, true>(t, i, count, m, v, 0);
      else store_moments<32, true>(t, i, count, m, v, 0);
    } else {
      if (t.bits == 8) load_moments<8>(t, i, count, m, v);
      else load_moments<32>(t, i, count, m, v);
#pragma unroll
      for (int e = 0; e < kEach; ++e)  // what is not there, 0, times a block's NaN
        if (e >= count) m[e] = v[e] = 0.f;
      Entries<To, kEach>::store(m_flat + t.flat + i, kEach, m);
      Entries<To, kEach>::store(v_flat + t.flat + i, kEach, v);
    }
  }
}

// ---- host -------------------------------------------------------------------------------------------

constexpr int64_t kChunksPerLaunch = int64_t{1} << 22;  // a grid's threads stay below 2^31

template <typename F>
int in_launches(const Optimiser &o, const char *what, F launch) {
  for (int64_t at = 0; at < o.count; at += kChunksPerLaunch) {
    launch(dim3(static_cast<unsigned>(std::min(kChunksPerLaunch, o.count - at))), o.chunks + at);
    if (int rc = check_launch(what)) return rc;
  }
  return GOSH_OK;
}

struct Extent {
  uintptr_t from, to;
};
void note(std::vector<Extent> &all, const void *p, int64_t bytes) {
  if (bytes > 0) all.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes});
}

int check_param(const gosh_param &q, int32_t i, std::vector<Extent> &written, std::vector<Extent> &read) {
  if (q.n < 0 || q.n > kMostEntries) return fail(GOSH_EINVAL, "tensor %d: n = %lld: must be in [0, 2^40]", i, (long long)q.n);
  if (q.g_type != GOSH_F32 && q.g_type != GOSH_BF16 && q.g_type != GOSH_F16)
    return fail(GOSH_EINVAL, "tensor %d: g_type %d is none of gosh_type", i, q.g_type);
  if (q.bits != 8 && q.bits != 32) return fail(GOSH_EINVAL, "tensor %d: bits = %d: must be 8 or 32", i, q.bits);
  if (!(q.weight_decay >= 0.f) || !std::isfinite(q.weight_decay))
    return fail(GOSH_EINVAL, "tensor %d: weight_decay = %g: must be a number from 0 on", i, q.weight_decay);
  if (q.copy != nullptr && q.copy_type != GOSH_BF16 && q.copy_type != GOSH_F16)
    return fail(GOSH_EINVAL, "tensor %d: copy_type %d: must be GOSH_BF16 or GOSH_F16", i, q.copy_type);
  if (q.n == 0) return GOSH_OK;
  const int64_t g_size = q.g_type == GOSH_F32 ? 4 : 2;
  const struct { const void *p; int64_t bytes, align; const char *what; bool needed, out; } all[] = {
      {q.p, 4 * q.n, 4, "p", true, true}, {q.g, g_size * q.n, g_size, "g", true, false},
      {q.state, layout_of(q.n, q.bits).bytes, 16, "state", true, true}, {q.copy, 2 * q.n, 2, "copy", false, true}};
  for (const auto &a : all) {
    if (a.p == nullptr) {
      if (a.needed) return fail(GOSH_EINVAL, "tensor %d: %s is null", i, a.what);
      continue;
    }
    if (reinterpret_cast<uintptr_t>(a.p) % a.align != 0)
      return fail(GOSH_EINVAL, "tensor %d: %s must be %lld-byte aligned", i, a.what, (long long)a.align);
    if (int rc = check_device_span(a.p, static_cast<size_t>(a.bytes), a.what)) return rc;
    note(a.out ? written : read, a.p, a.bytes);
  }
  return GOSH_OK;
}

// Nothing that is written may be another's, or be read as a gradient.
int check_apart(std::vector<Extent> &written, const std::vector<Extent> &read) {
  std::sort(written.begin(), written.end(), [](const Extent &a, const Extent &b) { return a.from < b.from; });
  for (size_t i = 1; i < written.size(); ++i)
    if (written[i].from < written[i - 1].to) return fail(GOSH_EINVAL, "two arrays that a step writes overlap");
  for (const Extent &r : read) {
    auto next = std::upper_bound(written.begin(), written.end(), r.from, [](uintptr_t x, const Extent &e) { return x < e.from; });
    if ((next != written.end() && next->from < r.to) || (next != written.begin() && std::prev(next)->to > r.from))
      return fail(GOSH_EINVAL, "gradients overlap an array that a step writes");
  }
  return GOSH_OK;
}

int create(const gosh_param *params, int32_t count, void **out) {
  std::vector<Extent> written, read;
  for (int32_t i = 0; i < count; ++i)
    if (int rc = check_param(params[i], i, written, read)) return rc;
  if (int rc = check_apart(written, read)) return rc;
  std::vector<Tensor> tensors;
  std::vector<Chunk> chunks;
  auto o = std::make_unique<Optimiser>();
  for (int32_t i = 0; i < count; ++i) {
    const gosh_param &q = params[i];
    const StateLayout l = layout_of(q.n, q.bits);
    tensors.push_back({q.p, q.g, static_cast<char *>(q.state), q.copy, q.n, o->entries, l.v, l.m_exps, l.v_exps, q.g_type, q.copy_type,
                       q.bits, q.weight_decay});
    for (int64_t c = 0; c < ceil_div(q.n, kChunk); ++c) chunks.push_back({i, static_cast<int32_t>(c)});
    o->entries += padded(q.n, kBlock);
  }
  o->count = static_cast<int64_t>(chunks.size());
  GOSH_TRY_HIP(hipGetDevice(&o->device), "device of the optimiser");
  // what other streams are still writing (states that were cleared on one of them) is there before a step on any stream
  GOSH_TRY_HIP(hipDeviceSynchronize(), "what the optimiser's tensors wait for");
  if (o->count > 0) {
    const size_t at = padded(tensors.size() * sizeof(Tensor), 256);
    char *memory = nullptr;
    GOSH_TRY_HIP(device_malloc(&memory, at + chunks.size() * sizeof(Chunk)), "memory of the optimiser");
    hipError_t e = hipMemcpy(memory, tensors.data(), tensors.size() * sizeof(Tensor), hipMemcpyHostToDevice);
    if (e == hipSuccess) e = hipMemcpy(memory + at, chunks.data(), chunks.size() * sizeof(Chunk), hipMemcpyHostToDevice);
    if (e != hipSuccess) {
      (void)hipFree(memory);
      return hip_fail(e, "tensors of the optimiser");
    }
    o->tensors = reinterpret_cast<Tensor *>(memory);
    o->chunks = reinterpret_cast<Chunk *>(memory + at);
  }
  *out = o.release();
  return GOSH_OK;
}

int check_optimiser(const void *optimiser) {
  if (optimiser == nullptr) return fail(GOSH_EINVAL, "optimiser is null");
  int device = 0;
  GOSH_TRY_HIP(hipGetDevice(&device), "current device");
  const int made = static_cast<const Optimiser *>(optimiser)->device;
  if (device != made) return fail(GOSH_EINVAL, "the optimiser is device %d's, the current one is %d", made, device);
  return GOSH_OK;
}

template <typename S>
int check_flat(const Optimiser &o, const S *p, int64_t entries, const char *what) {
  if (entries < o.entries)
    return fail(GOSH_EINVAL, "%lld entries: the moments take %lld", (long long)entries, (long long)o.entries);
  if (o.entries == 0) return GOSH_OK;
  if (p == nullptr) return fail(GOSH_EINVAL, "%s is null", what);
  if (reinterpret_cast<uintptr_t>(p) % sizeof(S) != 0) return fail(GOSH_EINVAL, "%s must be aligned to its entries", what);
  return check_device_span(p, static_cast<size_t>(o.entries) * sizeof(S), what);
}

template <typename To>
int save(const Optimiser &o, void *m, void *v, int64_t entries, hipStream_t st) {
  typedef typename To::Store S;
  S *const sm = static_cast<S *>(m), *const sv = static_cast<S *>(v);
  if (int rc = check_flat(o, sm, entries, "m")) return rc;
  if (int rc = check_flat(o, sv, entries, "v")) return rc;
  return in_launches(o, "moments", [&](dim3 grid, const Chunk *chunks) {
    moments_kernel<To, false><<<grid, dim3(kThreads), 0, st>>>(o.tensors, chunks, sm, sv);
  });
}

}  // namespace
}  // namespace gosh

extern "C" {

uint64_t gosh_adamw_state_bytes(int64_t n, int32_t bits) {
  if (n <= 0 || n > gosh::kMostEntries || (bits != 8 && bits != 32)) return 0;
  return static_cast<uint64_t>(gosh::layout_of(n, bits).bytes);
}

int gosh_adamw_create(const gosh_param *params, int32_t count, void **optimiser_out) {
  using namespace gosh;
  if (optimiser_out == nullptr) return fail(GOSH_EINVAL, "optimiser_out is null");
  *optimiser_out = nullptr;
  if (count < 0) return fail(GOSH_EINVAL, "count = %d: must be 0 or more", count);
  if (count > 0 && params == nullptr) return fail(GOSH_EINVAL, "params is null");
  try {
    return create(params, count, optimiser_out);
  } catch (const std::bad_alloc &) {
    return fail(GOSH_ENOMEM, "optimiser: out of host memory");
  } catch (...) {
    return fail(GOSH_ENOMEM, "optimiser: too many tensors");
  }
}

void gosh_adamw_free(void *optimiser) {
  gosh::Optimiser *const o = static_cast<gosh::Optimiser *>(optimiser);
  if (o == nullptr) return;
  int device = 0;
  const bool other = o->tensors != nullptr && hipGetDevice(&device) == hipSuccess && device != o->device;
  if (other) (void)hipSetDevice(o->device);
  if (o->tensors != nullptr) (void)hipFree(o->tensors);
  if (other) (void)hipSetDevice(device);
  delete o;
}

int gosh_adamw_step(void *optimiser, const gosh_adamw_options *options, void *hip_stream) {
  using namespace gosh;
  if (options == nullptr) return fail(GOSH_EINVAL, "options is null");
  const gosh_adamw_options &q = *options;
  if (!(std::fabs(q.lr) <= FLT_MAX)) return fail(GOSH_EINVAL, "lr = %g: must be a number of 32 bits", q.lr);
  if (!(q.beta1 >= 0 && q.beta1 < 1) || !(q.beta2 >= 0 && q.beta2 < 1))
    return fail(GOSH_EINVAL, "beta1 = %g, beta2 = %g: must be in [0, 1)", q.beta1, q.beta2);
  if (!(q.eps >= 0 && q.eps <= FLT_MAX) || (q.eps > 0 && static_cast<float>(q.eps) == 0.f))  // as 0 it would make 0 / 0 of no gradient
    return fail(GOSH_EINVAL, "eps = %g: must be 0 or a number over it of 32 bits", q.eps);
  if (q.steps == nullptr && q.step < 1) return fail(GOSH_EINVAL, "step = %lld: the first is 1", (long long)q.step);
  if (int rc = check_optimiser(optimiser)) return rc;
  if (int rc = check_floats(q.lr_dev, 1, "lr_dev", true)) return rc;
  if (int rc = check_floats(q.scale, 1, "scale", true)) return rc;
  if (q.steps != nullptr) {
    if (reinterpret_cast<uintptr_t>(q.steps) % 8 != 0) return fail(GOSH_EINVAL, "steps must be 8-byte aligned");
    if (int rc = check_device_span(q.steps, 8, "steps")) return rc;
  }
  const Optimiser &o = *static_cast<const Optimiser *>(optimiser);
  const double t = static_cast<double>(q.step);
  StepArgs a;
  a.beta1 = static_cast<float>(q.beta1), a.rest1 = static_cast<float>(1 - q.beta1);
  a.beta2 = static_cast<float>(q.beta2), a.rest2 = static_cast<float>(1 - q.beta2);
  a.eps = static_cast<float>(q.eps), a.lr = static_cast<float>(q.lr);
  a.log1 = static_cast<float>(std::log(q.beta1)), a.log2 = static_cast<float>(std::log(q.beta2));
  a.rate = static_cast<float>(q.lr / -std::expm1(t * std::log(q.beta1)));
  a.root = static_cast<float>(1 / std::sqrt(-std::expm1(t * std::log(q.beta2))));
  a.t = q.step;
  a.lr_dev = q.lr_dev, a.scale = q.scale, a.steps = q.steps;
  hipStream_t st = as_stream(hip_stream);
  if (int rc = in_launches(o, "AdamW", [&](dim3 grid, const Chunk *chunks) {
        step_kernel<<<grid, dim3(kThreads), 0, st>>>(o.tensors, chunks, a);
      }))
    return rc;
  if (q.steps == nullptr) return GOSH_OK;
  count_kernel<<<dim3(1), dim3(1), 0, st>>>(q.steps, q.scale);
  return check_launch("number of the step");
}

int64_t gosh_adamw_entries(const void *optimiser) {
  return optimiser == nullptr ? 0 : static_cast<const gosh::Optimiser *>(optimiser)->entries;
}

int gosh_adamw_save(void *optimiser, void *m, void *v, int64_t entries, int32_t type, void *hip_stream) {
  using namespace gosh;
  if (type != GOSH_F32 && type != GOSH_BF16) return fail(GOSH_EINVAL, "type %d: must be GOSH_F32 or GOSH_BF16", type);
  if (int rc = check_optimiser(optimiser)) return rc;
  const Optimiser &o = *static_cast<const Optimiser *>(optimiser);
  if (type == GOSH_F32) return save<F32>(o, m, v, entries, as_stream(hip_stream));
  return save<Bf16>(o, m, v, entries, as_stream(hip_stream));
}

int gosh_adamw_load(void *optimiser, const float *m, const float *v, int64_t entries, void *hip_stream) {
  using namespace gosh;
  if (int rc = check_optimiser(optimiser)) return rc;
  const Optimiser &o = *static_cast<const Optimiser *>(optimiser);
  if (int rc = check_flat(o, m, entries, "m")) return rc;
  if (int rc = check_flat(o, v, entries, "v")) return rc;
  return in_launches(o, "moments", [&](dim3 grid, const Chunk *chunks) {
    moments_kernel<F32, true><<<grid, dim3(kThreads), 0, as_stream(hip_stream)>>>(o.tensors, chunks, const_cast<float *>(m),
                                                                                  const_cast<float *>(v));
  });
}

}  // extern "C"
