// The head in 8-bit floating point: gosh_pack_fp8, gosh_unpack_fp8, gosh_linear_fp8 and its gradient.
#include "gosh_fp8.h"

#include <algorithm>
#include <cmath>

namespace gosh {

int check_fp8(const gosh_fp8 *m, const char *what, int use) {
  if (m == nullptr) return (use & kOptional) ? GOSH_OK : fail(GOSH_EINVAL, "%s is null", what);
  if (m->block_rows != 1 && m->block_rows != kFp8Block)
    return fail(GOSH_EINVAL, "%s: block_rows = %d: must be 1 or 128", what, m->block_rows);
  if (!rows_fit(m->rows)) return fail(GOSH_EINVAL, "%s: rows = %lld: must be in [0, 2^31-1)", what, (long long)m->rows);
  if (m->cols < 0 || m->cols > GOSH_FP8_MAX_LD)
    return fail(GOSH_EINVAL, "%s: cols = %lld: must be in [0, %d]", what, (long long)m->cols, GOSH_FP8_MAX_LD);
  if (m->ld < m->cols || m->ld > GOSH_FP8_MAX_LD || m->ld % kFp8Block != 0)
    return fail(GOSH_EINVAL, "%s: ld = %lld: must be a multiple of 128 in [cols, %d]", what, (long long)m->ld, GOSH_FP8_MAX_LD);
  const int64_t groups = ceil_div(m->cols, kFp8Block);
  if (m->ld_exps < groups || m->ld_exps > GOSH_FP8_MAX_LD || m->ld_exps % 4 != 0)
    return fail(GOSH_EINVAL, "%s: ld_exps = %lld: must be a multiple of 4 in [ceil(cols / 128), %d]", what, (long long)m->ld_exps, GOSH_FP8_MAX_LD);
  if (m->rows == 0 || m->cols == 0) return GOSH_OK;
  if (m->data == nullptr) return fail(GOSH_EINVAL, "%s: data is null", what);
  if (m->exps == nullptr) return fail(GOSH_EINVAL, "%s: exps is null", what);
  if (reinterpret_cast<uintptr_t>(m->data) % 16 != 0) return fail(GOSH_EINVAL, "%s: data must be 16-byte aligned", what);
  if (reinterpret_cast<uintptr_t>(m->exps) % 4 != 0) return fail(GOSH_EINVAL, "%s: exps must be 4-byte aligned", what);
  if (int rc = check_device_span(m->data, static_cast<size_t>(m->rows - 1) * m->ld + groups * kFp8Block, what)) return rc;
  return check_device_span(m->exps, static_cast<size_t>(ceil_div(m->rows, m->block_rows) - 1) * m->ld_exps + ceil_div(groups, 4) * 4, what);
}

namespace {

int check_fp8_shape(const gosh_fp8 *m, const char *what, int64_t rows, int64_t cols) {
  if (m != nullptr && (m->rows != rows || m->cols != cols))
    return fail(GOSH_EINVAL, "%s is %lld x %lld: must be %lld x %lld", what, (long long)m->rows, (long long)m->cols, (long long)rows, (long long)cols);
  return GOSH_OK;
}

// ---- into 8 bits ----------------------------------------------------------------------------------

struct Fp8Out {
  uint8_t *data, *exps;
  int64_t ld, ld_exps, step;  // step: see Fp8Plane
};
Fp8Out fp8_out(const gosh_fp8 *m) {
  return m == nullptr ? Fp8Out{nullptr, nullptr, 0, 0, 0} : Fp8Out{static_cast<uint8_t *>(m->data), m->exps, m->ld, m->ld_exps, kFp8Block};
}

struct PackArgs {
  Plane x, z;       // z: x is multiplied by the activation's slope there
  Fp8Out q, qt;
  float *sums;      // of the columns of each 128 rows, cols of them
  int64_t rows, first;  // first: of the launch, in blocks of 128 rows
  int32_t cols, act, z_packed;
};

__device__ __forceinline__ float larger_of_16(float v) {  // v >= 0, whose bits order as it does
  uint32_t b = __float_as_uint(v);
  b = larger_of_lanes<0xb1>(b);
  b = larger_of_lanes<0x4e>(b);
  b = larger_of_lanes<0x141>(b);
  return __uint_as_float(larger_of_lanes<0x140>(b));
}

// A lane's 8 columns of 8 rows, from row, col on, as they lie in memory, all of them requested at once.  Full: all are there.
// Otherwise rows past the end read the last one and are made zero, and only lanes of fewer than 8 columns take them in
// pieces (with a branch for each row and piece 517 x 132 in f16 took 7.1 us, now 5.0).
template <typename T, bool Full>
struct Square8 {
  typename Entries<T, 8>::Vec raw[8];
  __device__ __forceinline__ Square8(const Plane &x, int64_t row, int col, int64_t rows, int count) {
    typedef typename T::Store S;
    const S *const p = static_cast<const S *>(x.data) + col;
    const auto at = [&](int i) { return p + (Full || row + i < rows ? row + i : rows - 1) * x.ld; };
    if (Full || count == 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) raw[i] = Entries<T, 8>::fetch(at(i), 8);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) raw[i] = Entries<T, 8>::fetch(at(i), count);
    }
    if (!Full) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (row + i >= rows) raw[i] = 0;
    }
  }
  __device__ __forceinline__ float at(int i, int e) const { return T::up(raw[i][e]); }
};
// The same of a packed matrix.
template <bool Full>
struct PackedSquare8 {
  uint32_t q[8][2];
  float unit[8];
  __device__ __forceinline__ PackedSquare8(const Plane &x, int64_t row, int col, int64_t rows, int count) {
    const int8_t *const p = static_cast<const int8_t *>(x.data) + col;
    const uint8_t *const exps = x.exps + col / kGroup;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = Full || row + i < rows ? row + i : rows - 1;
      const bool there = Full || (row + i < rows && count > 0);
      load_bytes<8>(p + r * x.ld, Full ? 8 : count, q[i]);
      unit[i] = there ? read_unit(exps[r * x.ld_exps]) : 0.f;
    }
  }
  __device__ __forceinline__ float at(int i, int e) const {
    return static_cast<float>(static_cast<int32_t>(q[i][e / 4] << (24 - 8 * (e % 4))) >> 24) * unit[i];
  }
};

// v = x, times the slope of the activation at z where there is one.  What is not there is 0, and slopes at 0 are finite.
template <typename T, bool Slope, bool Full>
__device__ __forceinline__ void load_square(const PackArgs &a, int64_t row, int col, int count, float (&v)[8][8]) {
  const Square8<T, Full> x(a.x, row, col, a.rows, count);
  const auto times = [&](const auto &z) {
    with_activation(a.act, [&](auto f) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = x.at(i, e) * decltype(f)::slope(z.at(i, e));
    });
  };
  if (Slope && a.act != GOSH_ACT_NONE) {
    if (a.z_packed) times(PackedSquare8<Full>(a.z, row, col, a.rows, count));
    else times(Square8<T, Full>(a.z, row, col, a.rows, count));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = x.at(i, e);
  }
}

// Squares of 128 x 128: a lane has 8 columns of 8 rows after each other, 16 lanes a row.  The largest magnitude along a row
// is joined over those 16 lanes, that along a column over the 16 lanes that have the others of its rows, through LDS, by one
// thread a column; the transposed bytes are turned round in LDS too.  Square: one exponent for all of it.  Maxima pass over NaN,
// which stays NaN in 8 bits by itself; infinities are made NaN first, where there are any.
// Bound by memory: 131,072 x 1024 in bf16, as it is, takes 51 to 65 us (403 MB), 65,536 x 1024 both ways 65; with GELU's
// slope, both ways and sums, 65,536 x 2048 take 170 us (805 MB, 4.7 TB/s; four wavefronts a SIMD instead of three spill and take 190).
template <typename T, bool Square, bool Slope>
__global__ __launch_bounds__(256, Slope && T::kType == GOSH_F32 ? 2 : 3) void pack_fp8_kernel(const PackArgs a) {
  __shared__ __attribute__((aligned(16))) float most_of[16][kFp8Block];  // by rows' lanes and column
  __shared__ __attribute__((aligned(16))) float sum_of[Slope ? 16 : 1][kFp8Block];
  __shared__ __attribute__((aligned(16))) float inverse_of[kFp8Block];   // of the columns' units
  __shared__ float all_of[4];
  __shared__ __attribute__((aligned(16))) uint8_t turned[kFp8Block * kFp8Block];
  const int c = threadIdx.x % 16, r = threadIdx.x / 16;
  const int tile_n = blockIdx.x, first = tile_n * kFp8Block, col0 = first + 8 * c;
  const int count = a.cols - col0 < 0 ? 0 : a.cols - col0 < 8 ? a.cols - col0 : 8;
  const bool turn = a.qt.data != nullptr;
  const int64_t block = a.first + blockIdx.y, row0 = block * kFp8Block + 8 * r;
  const bool full = (block + 1) * kFp8Block <= a.rows && first + kFp8Block <= a.cols;
  {
    float v[8][8];
    if (full) load_square<T, Slope, true>(a, row0, col0, count, v);
    else load_square<T, Slope, false>(a, row0, col0, count, v);
    if (Slope && a.sums != nullptr) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += v[i][e];
        sum_of[Slope ? r : 0][8 * c + e] = s;
      }
    }
    float along[8], down[8];
    const auto largest = [&]() {
#pragma unroll
      for (int i = 0; i < 8; ++i) along[i] = down[i] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          along[i] = fmaxf(along[i], __builtin_fabsf(v[i][e]));
          down[e] = fmaxf(down[e], __builtin_fabsf(v[i][e]));
        }
    };
    largest();
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, along[i]);
    if (__builtin_expect(__any(most == INFINITY), 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = __builtin_fabsf(v[i][e]) == INFINITY ? __uint_as_float(0x7fc00000u) : v[i][e];
      largest();
      most = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) most = fmaxf(most, along[i]);
    }
    uint32_t square = 0;  // the byte of all
    if constexpr (Square) {
      uint32_t b = __float_as_uint(larger_of_16(most));
      b = max(b, static_cast<uint32_t>(__shfl_xor(static_cast<int>(b), 16)));
      b = max(b, static_cast<uint32_t>(__shfl_xor(static_cast<int>(b), 32)));
      if (threadIdx.x % 64 == 0) all_of[threadIdx.x / 64] = __uint_as_float(b);
    } else if (turn) {
#pragma unroll
      for (int e = 0; e < 8; ++e) most_of[r][8 * c + e] = down[e];
    }
    if (Square || turn || Slope) __syncthreads();
    if constexpr (Square) {
      square = fp8_byte(__float_as_uint(fmaxf(fmaxf(all_of[0], all_of[1]), fmaxf(all_of[2], all_of[3]))));
      if (threadIdx.x == 0 && a.q.data != nullptr) a.q.exps[block * a.q.ld_exps + tile_n] = static_cast<uint8_t>(square);
      if (threadIdx.x == 0 && turn) a.qt.exps[tile_n * a.qt.ld_exps + block] = static_cast<uint8_t>(square);
    } else {
      const int col = threadIdx.x % kFp8Block;
      if (turn && threadIdx.x < kFp8Block) {
        float m = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) m = fmaxf(m, most_of[k][col]);
        const uint32_t byte = fp8_byte(__float_as_uint(m));
        inverse_of[col] = inverse_unit(byte);
        if (first + col < a.cols) a.qt.exps[(first + col) * a.qt.ld_exps + block] = static_cast<uint8_t>(byte);
      }
      if (Slope && a.sums != nullptr && threadIdx.x >= kFp8Block && first + col < a.cols) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) s += sum_of[Slope ? k : 0][col];
        a.sums[block * a.cols + first + col] = s;
      }
    }
    if (a.q.data != nullptr) {
      uint8_t *const to = a.q.data + row0 * a.q.ld + col0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t byte = Square ? square : fp8_byte(__float_as_uint(larger_of_16(along[i])));
        if (!full && row0 + i >= a.rows) continue;
        const float inv = inverse_unit(byte);
        *reinterpret_cast<U2 *>(to + i * a.q.ld) = U2{to_e4m3(v[i][0], v[i][1], v[i][2], v[i][3], inv), to_e4m3(v[i][4], v[i][5], v[i][6], v[i][7], inv)};
        if (!Square && c == 0) a.q.exps[(row0 + i) * a.q.ld_exps + tile_n] = static_cast<uint8_t>(byte);
      }
    }
    if (turn) {
      if (!Square) __syncthreads();
      // column 8 c + e of 8 rows: 8 bytes, at place r ^ c of the column's 16
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float inv = Square ? inverse_unit(square) : inverse_of[8 * c + e];
        *reinterpret_cast<U2 *>(turned + (8 * c + e) * kFp8Block + (r ^ c) * 8) =
            U2{to_e4m3(v[0][e], v[1][e], v[2][e], v[3][e], inv), to_e4m3(v[4][e], v[5][e], v[6][e], v[7][e], inv)};
      }
      __syncthreads();
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const int col = 32 * p + threadIdx.x / 8, pair = threadIdx.x % 8, shift = col / 8;
        if (first + col >= a.cols) continue;
        const U4 x = *reinterpret_cast<const U4 *>(turned + col * kFp8Block + (2 * pair ^ (shift & 14)) * 8);
        const U4 out = shift & 1 ? U4{x[2], x[3], x[0], x[1]} : x;
        *reinterpret_cast<U4 *>(a.qt.data + (first + col) * a.qt.ld + block * a.qt.step + 16 * pair) = out;
      }
    }
  }
}

constexpr int64_t kMostBlocks = int64_t{1} << 22;  // a grid's threads stay below 2^31

template <typename T>
int launch_pack_fp8(PackArgs a, bool square, bool slope, hipStream_t st) {
  constexpr int64_t kMostRows = 8192;  // of blocks; across are 512 at most
  const int64_t blocks = ceil_div(a.rows, kFp8Block);
  for (a.first = 0; a.first < blocks; a.first += kMostRows) {
    const dim3 grid(static_cast<unsigned>(ceil_div(a.cols, kFp8Block)), static_cast<unsigned>(std::min(blocks - a.first, kMostRows)));
    if (slope) pack_fp8_kernel<T, false, true><<<grid, dim3(256), 0, st>>>(a);
    else if (square) pack_fp8_kernel<T, true, false><<<grid, dim3(256), 0, st>>>(a);
    else pack_fp8_kernel<T, false, false><<<grid, dim3(256), 0, st>>>(a);
    if (int rc = check_launch("8-bit floating point")) return rc;
  }
  return GOSH_OK;
}
int pack_fp8(int32_t type, const PackArgs &a, bool square, bool slope, hipStream_t st) {
  if (type == GOSH_F32) return launch_pack_fp8<F32>(a, square, slope, st);
  if (type == GOSH_BF16) return launch_pack_fp8<Bf16>(a, square, slope, st);
  return launch_pack_fp8<F16>(a, square, slope, st);
}

template <typename T>
__global__ __launch_bounds__(256) void unpack_fp8_kernel(const Fp8Plane q, const Plane x, int64_t rows, int32_t cols, int32_t chunks) {
  const int64_t total = rows * chunks;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = i / chunks;
    const int col = static_cast<int>(i - row * chunks) * 8;
    const U2 w = *reinterpret_cast<const U2 *>(q.data + row * q.ld + col);
    const float unit = read_unit(q.exps[(row >> q.shift) * q.ld_exps + col / kFp8Block]);
    float v[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      typedef float Two __attribute__((ext_vector_type(2)));
      const Two lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[h]), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[h]), true);
      v[4 * h] = lo[0] * unit, v[4 * h + 1] = lo[1] * unit, v[4 * h + 2] = hi[0] * unit, v[4 * h + 3] = hi[1] * unit;
    }
    Entries<T, 8>::store(static_cast<typename T::Store *>(x.data) + row * x.ld + col, cols - col < 8 ? cols - col : 8, v);
  }
}

template <typename T>
void launch_unpack_fp8(const gosh_fp8 *q, const gosh_mat *x, hipStream_t st) {
  const int32_t chunks = static_cast<int32_t>(ceil_div(x->cols, 8));
  const dim3 grid(static_cast<unsigned>(std::min(ceil_div(x->rows * chunks, 256), kMostBlocks)));
  unpack_fp8_kernel<T><<<grid, dim3(256), 0, st>>>(fp8_plane(q), plane_of(x), x->rows, x->cols, chunks);
}

// ---- products -------------------------------------------------------------------------------------

Plane rows_of(Plane p, int64_t row, int32_t type, bool packed) { return rows_from(p, row, type, packed); }

int product_fp8(int32_t type, ProductOut out, const Fp8Args &a, hipStream_t st) {
  if (type == GOSH_F32) return launch_fp8<F32>(out, a, st);
  if (type == GOSH_BF16) return launch_fp8<Bf16>(out, a, st);
  return launch_fp8<F16>(out, a, st);
}

constexpr int64_t kTilesPerLaunch = int64_t{1} << 22;
// Bytes of y from which it, and z with it, is stored past the caches: the 256 MB of the cache beside the memory.  131,072 x 1024 ->
// 4096 (1.07 GB): 727 us, 643 with it.  By tiles of 256 alone; exact products (f16, f32, ReLU) have none here and store through the caches.
constexpr int64_t kPastCaches = int64_t{256} << 20;

constexpr int64_t kFewRows = 32;  // that are put into 8 bits in the product's launch

// The us that a product takes by its tiles, from what it took here (bf16 results with GELU, in a graph; us with few, 64, 128 and 256:
// 64 x 4096 -> 4096: 13.9, 18.4, 25.5, 50.2; 512 x 256 -> 1024: 5.3, 6.0, 7.4, 13.2; 4096 x 2048 -> 256: 24.4, 12.0, 15.5, 30.1;
// 8192 x 512 -> 512: 21.8, 14.0, 9.6, 17.2; 131,072 x 128 -> 128: 33.5, 35.5, 17.6, 32.5; 65,536 x 512 -> 512: 124, 89, 40.7, 34.6).
// A CU works on four tiles of 64 together, two of 128 or one of 256; each has its way out, and steps that are as long as a load
// is under way where it is alone.
// Exact products in tiles (see fp8_mma; 50,021 x 260 -> 1037 in f32 with 64 and 128: 123 and 96 us; 65,536 x 1024 -> 1024 in f16: 273
// and 158) take longer.  In tiles of 256 they took 105 and 169, by their times never the least, and are there for dw alone.
double fp8_time(int tile, int64_t tiles, int64_t blocks, bool exact) {
  const double k = static_cast<double>(blocks), per_cu = static_cast<double>(ceil_div(tiles, 256));
  if (tile == 32) return few_waves(blocks) == 4 ? 4.0 + per_cu * (0.5 + 0.12 * k) : 3.7 + per_cu * 0.32 * k;
  const double held = tile == 256 ? 1 : tile == 128 ? 2 : 4, together = std::min(per_cu, held), turns = std::ceil(per_cu / held);
  if (exact && tile == 128) return 2.0 + turns * (together > 1 ? 8.0 + 1.4 * k : 5.0 + 1.3 * k);
  if (exact) return 1.5 + turns * (2.5 + together + k * (0.4 + 0.25 * together));
  if (tile == 256) return 2.0 + turns * (10.0 + 1.2 * k);
  if (tile == 128) return 2.0 + turns * (4.5 + 0.75 * together + k * (together > 1 ? 0.95 : 0.6));
  return 1.5 + turns * (2.0 + 1.25 * together + k * (0.22 + 0.2 * together));
}
int fp8_tile_for(int64_t M, int64_t N, int64_t blocks, bool exact) {
  int best = 0;
  double least = 0;
  for (int s : {256, 128, 64, 32}) {
    if (s == 256 && exact) continue;
    if (s == 32 && M > 65535 * 32) continue;  // a grid's rows
    const double time = fp8_time(s, ceil_div(M, s) * ceil_div(N, s), blocks, exact);
    if (best == 0 || time < least) best = s, least = time;
  }
  return best;
}

// All rows of A, as many to a launch as a grid takes.
int product_of_rows_fp8(int32_t type, ProductOut out, Fp8Args a, int64_t rows, hipStream_t st) {
  const int tile = a.tile = a.pack.data != nullptr ? 32 : fp8_tile_for(rows, a.g.N, a.g.K, type != GOSH_BF16 || a.exact);
  a.g.tiles_n = static_cast<int32_t>(ceil_div(a.g.N, tile));
  a.g.splits = std::max(a.g.splits, 1);
  a.g.k_per_split = ceil_div(a.g.K, a.g.splits);
  const int64_t rows_per_launch = std::max<int64_t>(kTilesPerLaunch / a.g.tiles_n * tile / kFp8Block, 1) * kFp8Block;
  const Fp8Args all = a;
  for (int64_t r = 0; r < rows; r += rows_per_launch) {
    a.g.M = std::min(rows_per_launch, rows - r);
    a.g.tiles_m = static_cast<int32_t>(ceil_div(a.g.M, tile));
    set_reciprocals(a);
    a.x.data = all.x.data + r * all.x.ld;
    a.x.exps = all.x.exps + (r >> all.x.shift) * all.x.ld_exps;
    a.g.out = rows_of(all.g.out, r, type, false);
    a.g.forward.residual = rows_of(all.g.forward.residual, r, type, false);
    a.g.forward.y = rows_of(all.g.forward.y, r, type, false);
    a.g.forward.z = rows_of(all.g.forward.z, r, type, all.g.forward.z_packed != 0);
    if (int rc = product_fp8(type, out, a, st)) return rc;
  }
  return GOSH_OK;
}

// Whether GOSH_FP8_EXACT is in act, which it is taken out of.
bool take_exact(int32_t &act) {
  const bool exact = act >= 0 && (act & GOSH_FP8_EXACT) != 0;
  if (exact) act -= GOSH_FP8_EXACT;
  return exact;
}

uint64_t round_up(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

// How dw is split along the rows: the parts are written and read again, at 5 TB/s.  Few results (32) are not split; what is not is
// stored as it is.  By the times of products that are not exact, whatever dw's type: with those of exact ones, which are of the forward
// pass, 65,536 x 1024 -> 2048 in f16 takes 330 us (with the pass over dy; 306 by these, in tiles of 256), 4,096 x 512 -> 512 18.6 (17.0), and
// 16,384 x 2048 -> 4096, 8,192 x 1024 -> 1024 and 32,768 x 512 -> 512 take the same.
struct Fp8DwPlan {
  int32_t tile, tiles_m, tiles_n, splits;
  int64_t blocks_per_split;
};
Fp8DwPlan plan_dw_fp8(int64_t rows, int32_t in, int32_t out) {
  Fp8DwPlan best{};
  double least = 0;
  const int64_t blocks = ceil_div(rows, kFp8Block);
  for (int s : {256, 128, 64, 32}) {
    const int64_t tiles_m = ceil_div(out, s), tiles_n = ceil_div(in, s), tiles = tiles_m * tiles_n;
    for (int64_t want = 1; want <= (s == 32 ? 1 : std::min<int64_t>(std::max<int64_t>(blocks, 1), 1024)); want *= 2) {
      const int64_t per = std::max<int64_t>(1, ceil_div(blocks, want)), splits = ceil_div(blocks, per);
      if (want > 1 && tiles * splits > 2048) break;
      const double time = fp8_time(s, tiles * splits, per, false) + (splits <= 1 ? 0 : 2.5 + 1.6e-6 * static_cast<double>(splits) * in * out);
      if (best.tile != 0 && time >= least) continue;
      least = time;
      best = Fp8DwPlan{s, static_cast<int32_t>(tiles_m), static_cast<int32_t>(tiles_n), static_cast<int32_t>(splits), per};
    }
  }
  return best;
}

// What the gradient's workspace holds, as offsets.
struct Fp8BackwardPlan {
  Fp8DwPlan dw;
  int64_t ld, ld_exps, step_t, ld_exps_t;  // the transposed dz: a block of 128 rows of all columns lies together
  uint64_t q, exps, qt, exps_t, sums, dw_parts, bytes;
};
Fp8BackwardPlan plan_backward_fp8(int64_t rows, int32_t in, int32_t out) {
  Fp8BackwardPlan p;
  p.dw = plan_dw_fp8(rows, in, out);
  const int64_t blocks = ceil_div(out, kFp8Block), blocks_t = ceil_div(rows, kFp8Block);
  p.ld = blocks * kFp8Block, p.ld_exps = ceil_div(blocks, 4) * 4;
  p.step_t = static_cast<int64_t>(out) * kFp8Block, p.ld_exps_t = ceil_div(blocks_t, 4) * 4;
  uint64_t at = 0;
  const auto take = [&](uint64_t bytes) {
    const uint64_t from = at;
    at += round_up(bytes);
    return from;
  };
  p.q = take(static_cast<uint64_t>(rows) * p.ld);
  p.exps = take(static_cast<uint64_t>(rows) * p.ld_exps);
  p.qt = take(static_cast<uint64_t>(blocks_t) * p.step_t);
  p.exps_t = take(static_cast<uint64_t>(out) * p.ld_exps_t);
  p.sums = take(static_cast<uint64_t>(blocks_t) * out * 4);
  p.dw_parts = take(p.dw.splits == 1 ? 0 : static_cast<uint64_t>(p.dw.splits) * in * out * 4);
  p.bytes = at;
  return p;
}

}  // namespace
}  // namespace gosh

extern "C" {

int gosh_pack_fp8(const gosh_mat *x, const gosh_fp8 *q, const gosh_fp8 *qt, void *hip_stream) {
  using namespace gosh;
  if (int rc = check_mat(x, "x")) return rc;
  if (int rc = check_fp8(q, "q", kOptional)) return rc;
  if (int rc = check_fp8(qt, "qt", kOptional)) return rc;
  if (int rc = check_fp8_shape(q, "q", x->rows, x->cols)) return rc;
  if (int rc = check_fp8_shape(qt, "qt", x->cols, x->rows)) return rc;
  if (q != nullptr && qt != nullptr && q->block_rows != qt->block_rows)
    return fail(GOSH_EINVAL, "q and qt: block_rows = %d and %d: must be the same", q->block_rows, qt->block_rows);
  if (x->rows == 0 || (q == nullptr && qt == nullptr)) return GOSH_OK;
  PackArgs a{};
  a.x = plane_of(x);
  a.q = fp8_out(q);
  a.qt = fp8_out(qt);
  a.rows = x->rows;
  a.cols = x->cols;
  return pack_fp8(x->type, a, (q != nullptr ? q : qt)->block_rows == kFp8Block, false, as_stream(hip_stream));
}

int gosh_unpack_fp8(const gosh_fp8 *q, const gosh_mat *x, void *hip_stream) {
  using namespace gosh;
  if (int rc = check_fp8(q, "q")) return rc;
  if (int rc = check_mat(x, "x")) return rc;
  if (int rc = check_fp8_shape(q, "q", x->rows, x->cols)) return rc;
  if (x->rows == 0) return GOSH_OK;
  hipStream_t st = as_stream(hip_stream);
  if (x->type == GOSH_F32) launch_unpack_fp8<F32>(q, x, st);
  else if (x->type == GOSH_BF16) launch_unpack_fp8<Bf16>(q, x, st);
  else launch_unpack_fp8<F16>(q, x, st);
  return check_launch("8-bit floating point back");
}

int gosh_linear_fp8(const gosh_mat *x, const gosh_fp8 *x8, const gosh_fp8 *w, const float *bias, int32_t act,
                    const gosh_mat *residual, const gosh_mat *y, const gosh_mat *z, void *hip_stream) {
  using namespace gosh;
  if (int rc = check_mat(x, "x", kOptional)) return rc;
  if (int rc = check_fp8(x8, "x8")) return rc;
  if (int rc = check_fp8(w, "w")) return rc;
  if (int rc = check_mat(y, "y")) return rc;
  if (int rc = check_mat(residual, "residual", kOptional)) return rc;
  if (int rc = check_mat(z, "z", kOptional | kMayBePacked)) return rc;
  const bool exact = take_exact(act);
  if (act < GOSH_ACT_NONE || act > GOSH_ACT_SILU) return fail(GOSH_EINVAL, "act = %d: no activation", act);
  if (w->rows < 1 || w->rows > GOSH_MAT_MAX_COLS)
    return fail(GOSH_EINVAL, "w: rows = %lld: must be in [1, %d]", (long long)w->rows, GOSH_MAT_MAX_COLS);
  if (w->cols < 1 || w->cols > GOSH_MAT_MAX_COLS)
    return fail(GOSH_EINVAL, "w: cols = %lld: must be in [1, %d]", (long long)w->cols, GOSH_MAT_MAX_COLS);
  if (x8->block_rows != 1) return fail(GOSH_EINVAL, "x8: block_rows = %d: must be 1", x8->block_rows);
  const int32_t out = static_cast<int32_t>(w->rows), in = static_cast<int32_t>(w->cols);
  const int64_t rows = x8->rows;
  if (int rc = check_fp8_shape(x8, "x8", rows, in)) return rc;
  if (int rc = check_shape(x, "x", rows, in)) return rc;
  const struct { const gosh_mat *m; const char *what; } outs[] = {{y, "y"}, {residual, "residual"}, {z, "z"}};
  for (const auto &o : outs) {
    if (int rc = check_shape(o.m, o.what, rows, out)) return rc;
    if (int rc = check_type(o.m, o.what, y->type)) return rc;
  }
  if (int rc = check_floats(bias, out, "bias", true)) return rc;
  if (rows == 0) return GOSH_OK;
  hipStream_t st = as_stream(hip_stream);
  Fp8Args a{};
  a.x = fp8_plane(x8);
  a.w = fp8_plane(w);
  a.exact = exact || act == GOSH_ACT_RELU;
  a.g.N = out;
  a.g.K = ceil_div(in, kFp8Block);
  a.g.forward = ForwardOut{bias, plane_of(residual), plane_of(y), plane_of(z), Plane{nullptr, nullptr, 0, 0}, act, z != nullptr && z->packed,
                           rows * out * (y->type == GOSH_F32 ? 4 : 2) >= kPastCaches};
  if (x != nullptr && rows <= kFewRows && fp8_tile_for(rows, out, a.g.K, y->type != GOSH_BF16 || a.exact) == 32) {
    a.pack = plane_of(x);  // in the product's launch
    a.pack_type = x->type;
    a.pack_cols = in;
  } else if (x != nullptr) {
    if (int rc = gosh_pack_fp8(x, x8, nullptr, hip_stream)) return rc;
  }
  return product_of_rows_fp8(y->type, kForward, a, rows, st);
}

uint64_t gosh_linear_fp8_backward_workspace(int64_t rows, int32_t in, int32_t out) {
  if (!gosh::rows_fit(rows) || in < 1 || out < 1 || in > GOSH_MAT_MAX_COLS || out > GOSH_MAT_MAX_COLS) return 0;
  return gosh::plan_backward_fp8(rows, in, out).bytes;
}

int gosh_linear_fp8_backward(const gosh_mat *dy, const gosh_fp8 *xt, const gosh_fp8 *wt, const gosh_mat *z, int32_t act,
                             const gosh_mat *dx, const gosh_mat *dw, float *db, void *workspace, uint64_t workspace_bytes,
                             void *hip_stream) {
  using namespace gosh;
  if (int rc = check_mat(dy, "dy")) return rc;
  if (int rc = check_fp8(xt, "xt", dw == nullptr ? kOptional : 0)) return rc;
  if (int rc = check_fp8(wt, "wt", dx == nullptr ? kOptional : 0)) return rc;
  const bool exact = take_exact(act);
  if (act < GOSH_ACT_NONE || act > GOSH_ACT_SILU) return fail(GOSH_EINVAL, "act = %d: no activation", act);
  if (int rc = check_mat(z, "z", kMayBePacked | (act == GOSH_ACT_NONE ? kOptional : 0))) return rc;
  if (int rc = check_mat(dx, "dx", kOptional)) return rc;
  if (int rc = check_mat(dw, "dw", kOptional)) return rc;
  if (dx == nullptr && dw == nullptr) return fail(GOSH_EINVAL, "dx and dw are null: gosh_linear_backward gives db alone");
  const int64_t rows = dy->rows;
  const int32_t out = dy->cols, in = dx != nullptr ? dx->cols : dw->cols;
  if (out > GOSH_MAT_MAX_COLS) return fail(GOSH_EINVAL, "dy: cols = %d: must be at most %d", out, GOSH_MAT_MAX_COLS);
  if (dw != nullptr && rows > GOSH_FP8_MAX_LD)
    return fail(GOSH_EINVAL, "dy: rows = %lld: dw takes at most %d", (long long)rows, GOSH_FP8_MAX_LD);
  if (int rc = check_fp8_shape(xt, "xt", in, rows)) return rc;
  if (int rc = check_fp8_shape(wt, "wt", in, out)) return rc;
  if (xt != nullptr && xt->block_rows != 1) return fail(GOSH_EINVAL, "xt: block_rows = %d: must be 1", xt->block_rows);
  if (int rc = check_shape(z, "z", rows, out)) return rc;
  if (int rc = check_shape(dx, "dx", rows, in)) return rc;
  if (int rc = check_shape(dw, "dw", out, in)) return rc;
  if (int rc = check_type(z, "z", dy->type)) return rc;
  if (int rc = check_type(dx, "dx", dy->type)) return rc;
  if (dw != nullptr && dw->type != GOSH_F32)
    if (int rc = check_type(dw, "dw", dy->type)) return rc;
  if (int rc = check_floats(db, out, "db", true)) return rc;
  const Fp8BackwardPlan p = plan_backward_fp8(rows, in, out);
  if (int rc = check_workspace(workspace, workspace_bytes, p.bytes)) return rc;
  hipStream_t st = as_stream(hip_stream);
  uint8_t *const ws = static_cast<uint8_t *>(workspace);
  float *const sums = reinterpret_cast<float *>(ws + p.sums), *const dw_parts = reinterpret_cast<float *>(ws + p.dw_parts);
  if (rows > 0) {
    PackArgs a{};
    a.x = plane_of(dy);
    a.z = plane_of(act == GOSH_ACT_NONE ? nullptr : z);
    if (dx != nullptr) a.q = Fp8Out{ws + p.q, ws + p.exps, p.ld, p.ld_exps, kFp8Block};
    if (dw != nullptr) a.qt = Fp8Out{ws + p.qt, ws + p.exps_t, kFp8Block, p.ld_exps_t, p.step_t};
    a.sums = db != nullptr ? sums : nullptr;
    a.rows = rows;
    a.cols = out;
    a.act = act;
    a.z_packed = act != GOSH_ACT_NONE && z->packed;
    if (int rc = pack_fp8(dy->type, a, false, true, st)) return rc;
  }
  Fp8Args gx{}, gw{};
  gx.exact = gw.exact = exact;
  if (dx != nullptr) {
    gx.x = Fp8Plane{ws + p.q, ws + p.exps, p.ld, p.ld_exps, 0, kFp8Block};
    gx.w = fp8_plane(wt);
    gx.g.N = in;
    gx.g.K = ceil_div(out, kFp8Block);
    gx.g.out = plane_of(dx);
  }
  if (dw != nullptr) {
    gw.x = Fp8Plane{ws + p.qt, ws + p.exps_t, kFp8Block, p.ld_exps_t, 0, p.step_t};
    gw.w = fp8_plane(xt);
    gw.tile = p.dw.tile;
    gw.g.M = out;
    gw.g.N = in;
    gw.g.K = ceil_div(rows, kFp8Block);
    gw.g.tiles_m = p.dw.tiles_m;
    gw.g.tiles_n = p.dw.tiles_n;
    gw.g.splits = p.dw.splits;
    gw.g.k_per_split = p.dw.blocks_per_split;
    gw.g.out = plane_of(dw);
    gw.g.parts = dw_parts;
    set_reciprocals(gw);
  }
  const JoinJob db_job{sums, out, db != nullptr ? out : 0, out, db, static_cast<int32_t>(ceil_div(rows, kFp8Block)), out, GOSH_F32};
  const bool few = rows > 0 && dw != nullptr && p.dw.tile == 32;
  if (few && (dx == nullptr || fp8_tile_for(rows, in, gx.g.K, dy->type != GOSH_BF16 || exact) == 32)) {
    if (dx != nullptr) {
      gx.g.M = rows;
      gx.g.tiles_m = static_cast<int32_t>(ceil_div(rows, 32));
      gx.g.tiles_n = static_cast<int32_t>(ceil_div(in, 32));
    }
    if (dy->type == GOSH_F32) return launch_fp8_gradients<F32>(gx, gw, dw->type, db_job, st);
    if (dy->type == GOSH_BF16) return launch_fp8_gradients<Bf16>(gx, gw, dw->type, db_job, st);
    return launch_fp8_gradients<F16>(gx, gw, dw->type, db_job, st);
  }
  if (dx != nullptr && rows > 0)
    if (int rc = product_of_rows_fp8(dx->type, kStore, gx, rows, st)) return rc;
  JoinJob jobs[3];
  int joins = 0;
  if (dw != nullptr && rows > 0) {
    // parts are in 32 bits: here the type says by which products
    if (int rc = p.dw.splits == 1 ? product_fp8(dw->type, kStore, gw, st)
                     : dw->type == GOSH_BF16 && !exact ? launch_fp8<Bf16>(kParts, gw, st) : launch_fp8<F32>(kParts, gw, st))
      return rc;
  }
  if (dw != nullptr && (rows == 0 || p.dw.splits > 1)) {
    const int64_t n = static_cast<int64_t>(out) * in;
    jobs[joins++] = {dw_parts, n, n, dw->ld, dw->data, rows > 0 ? p.dw.splits : 0, in, dw->type};
  }
  if (db != nullptr) jobs[joins++] = db_job;
  return join_parts(jobs, joins, st);
}

}  // extern "C"
