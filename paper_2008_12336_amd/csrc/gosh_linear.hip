// Linear layers: gosh_linear and gosh_linear_backward.  The products of many rows are gosh_product.h's; here are those
// of a few rows, and the gradient of the activation.
#include <algorithm>

#include "gosh_product.h"

namespace gosh {
namespace {

// ---- a few rows -----------------------------------------------------------------------------

constexpr int kFewCols = 2;  // rows of w a wavefront takes together (4: 6.2 instead of 4.9 us for 8 rows of 512 -> 2048)

// Rows for which reading w once for each 8 of them beats tiles, whose steps along k come one after the other.  Measured
// (us of a call, GELU and residual): 4.3 and 1 for each 8 rows and million entries of w, against 6 and 0.005 (16 bits,
// straight to LDS) or 0.024 (32 bits) for each column of w; 32 rows of 512 -> 2048: 8.1 and 8.3 (bf16), 8.5 and 16.6
// (f32), of 2048 -> 512: 7.5 and 15.4, 8.6 and 53.
bool few_rows(int64_t rows, int64_t k, int64_t n, int32_t type) {
  if (rows <= 8) return true;
  if (rows > 1024) return false;
  const int64_t whole = type == GOSH_F32 ? 256 : 512;  // columns that a wavefront takes at a time, there or not
  const double by_rows = static_cast<double>(ceil_div(rows, 8)) * (ceil_div(k, whole) * whole) * n * 1e-6;
  return by_rows < 1.7 + k * (type == GOSH_F32 ? 0.024 : 0.005);
}

// y = act(x w^T + bias) + residual for R rows: every lane has 8 (16-bit) or 4 entries of a row of w at a time, and its
// wavefront sums the lanes' products.
template <typename T, int R>
__global__ __launch_bounds__(256) void few_rows_kernel(const Plane x, const Plane w, const ForwardOut f, int rows, int n, int k) {
  constexpr int E = T::kType == GOSH_F32 ? 4 : 8;
  typedef typename T::Store S;
  const int wave = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
  const int col = wave * kFewCols, row0 = blockIdx.y * R;
  if (col >= n) return;
  float acc[kFewCols][R];
#pragma unroll
  for (int c = 0; c < kFewCols; ++c)
#pragma unroll
    for (int r = 0; r < R; ++r) acc[c][r] = 0.f;
  for (int k0 = lane * E; k0 < k; k0 += 64 * E) {
    const int count = k - k0;
    float wv[kFewCols][E];
#pragma unroll
    for (int c = 0; c < kFewCols; ++c)
      Entries<T, E>::load(static_cast<const S *>(w.data) + (col + c < n ? col + c : col) * w.ld + k0, count, wv[c]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float xv[E];
      Entries<T, E>::load(static_cast<const S *>(x.data) + (row0 + r < rows ? row0 + r : row0) * x.ld + k0, count, xv);
#pragma unroll
      for (int c = 0; c < kFewCols; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[c][r] = fmaf(wv[c][e], xv[e], acc[c][r]);
    }
  }
  float v = 0.f;
#pragma unroll
  for (int c = 0; c < kFewCols; ++c)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float sum = acc[c][r];
#pragma unroll
      for (int s = 32; s > 0; s /= 2) sum += __shfl_xor(sum, s);
      if (lane == c * R + r) v = sum;
    }
  const int r = row0 + lane % R, to = col + lane / R;
  if (lane >= kFewCols * R || r >= rows || to >= n) return;
  if (f.bias != nullptr) v += f.bias[to];
  if (f.z.data != nullptr) static_cast<S *>(f.z.data)[r * f.z.ld + to] = T::down(v);
  with_activation(f.act, [&](auto a) { v = decltype(a)::value(v); });
  if (f.residual.data != nullptr) v += T::up(static_cast<const S *>(f.residual.data)[r * f.residual.ld + to]);
  static_cast<S *>(f.y.data)[r * f.y.ld + to] = T::down(v);
}

template <typename T>
int launch_few_rows(const gosh_mat *x, const gosh_mat *w, const ForwardOut &f, hipStream_t st) {
  const int rows = static_cast<int>(x->rows), n = static_cast<int>(w->rows), k = x->cols;
  const dim3 grid(static_cast<unsigned>(ceil_div(n, 4 * kFewCols)), static_cast<unsigned>(ceil_div(rows, 8))), block(256);
  const Plane xp = plane_of(x), wp = plane_of(w);
  if (rows == 1) few_rows_kernel<T, 1><<<grid, block, 0, st>>>(xp, wp, f, rows, n, k);
  else if (rows == 2) few_rows_kernel<T, 2><<<grid, block, 0, st>>>(xp, wp, f, rows, n, k);
  else if (rows <= 4) few_rows_kernel<T, 4><<<grid, block, 0, st>>>(xp, wp, f, rows, n, k);
  else few_rows_kernel<T, 8><<<grid, block, 0, st>>>(xp, wp, f, rows, n, k);
  return check_launch("linear layer of a few rows");
}

// ---- tiles ------------------------------------------------------------------------------------

constexpr int64_t kTilesPerLaunch = int64_t{1} << 22;  // a grid's threads stay below 2^31

// Time of an entry of the result in tiles of one size, against that in the largest: smaller tiles fetch more of the
// operands for it, and larger ones waste more at the edges.  us of 65,536 x 512 -> 512 in tiles of 64, 128 and 256:
// 147, 67, 55 in bf16, 308 and 249 in f32 (whose tiles pass through registers); of 131,072 x 128 -> 128: 32, 19, 34 and
// 55, 48.
double weight_of(TileSize s, bool direct) {
  if (direct) return s == kLarge ? 1.0 : s == kMiddle ? 1.2 : 2.6;
  return s == kLarge ? 1e9 : s == kMiddle ? 1.0 : 1.25;
}

// Bytes of y from which tiles of kLarge store it past the caches, where nothing else is written: the 256 MB of the cache
// beside the memory, in which the next reader would not find it anyway.  us with and without, in bf16: 65,536 x 512 ->
// 2048 with GELU 167 and 187; layer norm, 512 -> 2048 with GELU and 2048 -> 512 after each other, which read what was
// written, 131,072 rows (y of 537 MB) 695 and 743, 65,536 rows 346 and 360, but 32,768 rows 184 and 178.
constexpr int64_t kPastCaches = int64_t{256} << 20;

// The tiles of which the busiest of the device's 256 CUs has the least work.  (8,192 x 512 -> 512 in bf16: 18, 15 and
// 25 us, with 4 tiles, one and a quarter of one to each CU.)
TileSize tiles_for(int64_t M, int64_t N, bool direct) {
  TileSize best = kSmall;
  double least = 0;
  for (TileSize s : {kSmall, kMiddle, kLarge}) {
    const double turns = static_cast<double>(ceil_div(ceil_div(M, tile_m(s)) * ceil_div(N, tile_n(s)), 256));
    const double work = turns * tile_m(s) * tile_n(s) * weight_of(s, direct);
    if (s == kSmall || work <= least) best = s, least = work;
  }
  return best;
}

// The length of `splits` parts of a sum over k: whole steps of every kind of tile.
int64_t split_length(int64_t k, int64_t splits) { return ceil_div(ceil_div(k, splits), 64) * 64; }

template <typename T>
TileSize shape_rows(ProductKind kind, int64_t rows, ProductArgs &g) {
  g.direct = T::kType != GOSH_F32 && can_be_direct(g.a, g.K) && can_be_direct(g.b, kind == kProductForward ? g.K : g.N);
  // a split sum was planned in tiles of kSmall, before it was known whether they are direct; only those store parts
  const TileSize size = g.parts != nullptr ? kSmall : tiles_for(rows, g.N, g.direct);
  g.M = rows;
  g.tiles_m = static_cast<int32_t>(std::min<int64_t>(ceil_div(rows, tile_m(size)), 1 << 30));
  g.tiles_n = static_cast<int32_t>(ceil_div(g.N, tile_n(size)));
  g.splits = std::max(g.splits, 1);
  g.k_per_split = split_length(g.K, g.splits);
  return size;
}

template <typename T>
int product_of_rows(ProductKind kind, ProductArgs g, int64_t rows, hipStream_t st) {
  const TileSize size = shape_rows<T>(kind, rows, g);
  const int64_t rows_per_launch = kTilesPerLaunch / g.tiles_n * tile_m(size);
  const ProductArgs all = g;
  for (int64_t r = 0; r < rows; r += rows_per_launch) {
    g.M = std::min(rows_per_launch, rows - r);
    g.tiles_m = static_cast<int32_t>(ceil_div(g.M, tile_m(size)));
    g.a = rows_from(all.a, r, T::kType, false);
    g.out = rows_from(all.out, r, T::kType, false);
    g.forward.residual = rows_from(all.forward.residual, r, T::kType, false);
    g.forward.y = rows_from(all.forward.y, r, T::kType, false);
    g.forward.z = rows_from(all.forward.z, r, T::kType, all.forward.z_packed != 0);
    g.forward.y8 = rows_from(all.forward.y8, r, T::kType, true);
    if (int rc = launch_product<T>(kind, size, g, st)) return rc;
  }
  return GOSH_OK;
}

// How dw is split along the rows: enough workgroups for every CU's eight wavefronts, at least 256 rows each.  The parts
// are summed by join_parts: 64 MB written and read for 65,536 x 512 -> 2048, 16 of its 145 + 17 us.
struct DwPlan {
  TileSize size;
  int32_t tiles_m, tiles_n, splits;
  int64_t k_per_split;
};
DwPlan plan_dw(int64_t rows, int32_t in, int32_t out, bool direct) {
  DwPlan best{};
  double least = 0;
  for (TileSize s : {kSmall, kMiddle, kLarge}) {
    DwPlan p;
    p.size = s;
    p.tiles_m = static_cast<int32_t>(ceil_div(out, tile_m(s)));
    p.tiles_n = static_cast<int32_t>(ceil_div(in, tile_n(s)));
    const int64_t tiles = static_cast<int64_t>(p.tiles_m) * p.tiles_n;
    const int64_t want = std::min(std::max<int64_t>(1, rows / 256), std::max<int64_t>(1, (s == kLarge ? 256 : 512) / tiles));
    p.k_per_split = split_length(std::max<int64_t>(rows, 1), want);
    p.splits = static_cast<int32_t>(ceil_div(rows, p.k_per_split));
    // of the busiest CU
    const double work = static_cast<double>(ceil_div(tiles * p.splits, 256)) * tile_m(s) * tile_n(s) * weight_of(s, direct) * p.k_per_split;
    if (s == kSmall || work <= least) best = p, least = work;
  }
  return best;
}

// Few tiles of dx are split along its long sum, the columns of dy, at least 256 of them each; 1: not split.  The backward
// call of 90 x 97 -> 1844 in f32: 75 us with the 58 steps one after the other, 35 split.
int32_t plan_dx_splits(int64_t rows, int32_t in, int32_t out, int32_t type) {
  if (rows == 0 || tiles_for(rows, in, type != GOSH_F32) != kSmall) return 1;
  const int64_t tiles = ceil_div(rows, 64) * ceil_div(in, 64);
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(out / 256, 256 / tiles));
  return static_cast<int32_t>(ceil_div(out, split_length(out, want)));
}

// ---- the activation's gradient ------------------------------------------------------------------

// dz = dy * act'(z) and its sums over rows, bound by memory: 65,536 x 2048 in bf16 reads and writes 805 MB in 158 us,
// 5.1 TB/s.  Taking the slope inside the products instead would take it again for every tile along the other side, 4
// times there (2 in dx, 2 in dw), each some 0.1 ms of all SIMDs' time by the instructions counted here.  dz is rounded to
// the activations' type: the matrix cores take 16 bits, and so does memory.  Of 16-bit types dx and dw end 1.4 times as
// far from 64 bits for it (rms 0.0023 of the entries' for bf16, of which 0.0017 is the rounding of dx and dw themselves).
// A lane has 16 bytes of a row; `along` lanes lie along a row, the others of the workgroup on rows of their own.  parts:
// gridDim.y x n sums.
template <typename T>
struct SlopeChunk {
  static constexpr int E = T::kType == GOSH_F32 ? 4 : 8;
};
template <typename T>
__global__ __launch_bounds__(256) void slope_kernel(const Plane dy, const Plane z, bool z_packed, int act, const Plane dz,
                                                    float *parts, int64_t rows, int n, int along, int64_t rows_per_block) {
  constexpr int E = SlopeChunk<T>::E;
  typedef typename T::Store S;
  __shared__ float lds[256][E];
  const int step = 256 / along, chunk = threadIdx.x % along, first = threadIdx.x / along;
  const int col = (static_cast<int>(blockIdx.x) * along + chunk) * E;
  const int count = first >= step ? 0 : n - col < E ? n - col : E;
  const int64_t r0 = blockIdx.y * rows_per_block, r1 = r0 + rows_per_block < rows ? r0 + rows_per_block : rows;
  float sum[E];
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.f;
  if (count > 0) {
    with_activation(act, [&](auto a) {
      typedef decltype(a) A;
      constexpr int kTogether = 2;  // rows whose loads are under way at once
      for (int64_t r = r0 + first; r < r1; r += kTogether * step) {
        float g[kTogether][E], s[kTogether][E];
#pragma unroll
        for (int t = 0; t < kTogether; ++t) {
          const int here = r + t * step < r1 ? count : 0;
          Entries<T, E>::load(static_cast<const S *>(dy.data) + (r + t * step) * dy.ld + col, here, g[t]);
          if (z.data != nullptr) load_entries<T, E>(z, z_packed, r + t * step, col, here, s[t]);
        }
#pragma unroll
        for (int t = 0; t < kTogether; ++t) {
          if (r + t * step >= r1) break;
          if (z.data != nullptr) {
#pragma unroll
            for (int e = 0; e < E; ++e) g[t][e] *= A::slope(s[t][e]);
          }
          if (dz.data != nullptr) Entries<T, E>::store(static_cast<S *>(dz.data) + (r + t * step) * dz.ld + col, count, g[t]);
#pragma unroll
          for (int e = 0; e < E; ++e) sum[e] += g[t][e];
        }
      }
    });
  }
  if (parts == nullptr) return;
#pragma unroll
  for (int e = 0; e < E; ++e) lds[threadIdx.x][e] = sum[e];
  __syncthreads();
  if (first != 0 || count <= 0) return;
  for (int s = 1; s < step; ++s)
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] += lds[s * along + chunk][e];
  Entries<F32, E>::store(parts + static_cast<int64_t>(blockIdx.y) * n + col, count, sum);
}

struct SlopePlan {
  int along;
  unsigned blocks_x, blocks_y;
  int64_t rows_per_block;
};
SlopePlan plan_slope(int64_t rows, int32_t n, int32_t type) {
  SlopePlan p;
  const int64_t chunks = ceil_div(n, type == GOSH_F32 ? 4 : 8);
  const int64_t fewest = ceil_div(chunks, 256);
  int64_t busy = 0;
  for (int64_t blocks = fewest; blocks < fewest + 4; ++blocks) {  // the split of a row that keeps most lanes busy
    const int64_t along = ceil_div(chunks, blocks);
    if (256 / along * along <= busy || ceil_div(chunks, along) != blocks) continue;
    busy = 256 / along * along;
    p.along = static_cast<int>(along);
    p.blocks_x = static_cast<unsigned>(blocks);
  }
  const int64_t step = 256 / p.along;
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(ceil_div(rows, 4 * step), ceil_div(1024, p.blocks_x)));
  p.rows_per_block = ceil_div(ceil_div(std::max<int64_t>(rows, 1), want), step) * step;
  p.blocks_y = static_cast<unsigned>(ceil_div(rows, p.rows_per_block));
  return p;
}

uint64_t round_up(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

// Tiles of dx up to which dx and dw share a launch: what the device holds at once.  71 x 55 -> 92 in f16: 25 us a
// backward call with two launches, 19 with one; 4,430 x 36 -> 275 in f32: 40 and 29.
constexpr int64_t kMostOfBoth = 1024;

struct BackwardPlan {
  DwPlan dw, dw_direct;
  SlopePlan slope;
  int64_t dz_ld;
  int32_t dx_splits;
  uint64_t dz, dw_parts, db_parts, dx_parts, bytes;  // offsets, and the whole
  uint64_t db_alone() const { return dx_parts - db_parts; }  // the whole where db is all that is asked for
};
BackwardPlan plan_backward(int64_t rows, int32_t in, int32_t out, int32_t type, int32_t act) {
  BackwardPlan p;
  p.dw = plan_dw(rows, in, out, false);
  p.dw_direct = plan_dw(rows, in, out, type != GOSH_F32);
  p.slope = plan_slope(rows, out, type);
  p.dz_ld = (out + 7) / 8 * 8;
  p.dz = 0;
  p.dw_parts = act == GOSH_ACT_NONE ? 0 : round_up(static_cast<uint64_t>(rows) * p.dz_ld * (type == GOSH_F32 ? 4 : 2));
  p.db_parts = p.dw_parts + round_up(static_cast<uint64_t>(std::max(p.dw.splits, p.dw_direct.splits)) * in * out * 4);
  p.dx_splits = plan_dx_splits(rows, in, out, type);
  p.dx_parts = p.db_parts + round_up(static_cast<uint64_t>(p.slope.blocks_y) * out * 4);
  p.bytes = p.dx_parts + (p.dx_splits > 1 ? round_up(static_cast<uint64_t>(p.dx_splits) * rows * in * 4) : 0);
  return p;
}

template <typename T>
int linear_backward(const gosh_mat *dy, const gosh_mat *x, const gosh_mat *w, const gosh_mat *z, int32_t act,
                    const gosh_mat *dx, const gosh_mat *dw, float *db, void *workspace, int32_t in, int32_t out,
                    hipStream_t st) {
  const int64_t rows = dy->rows;
  const BackwardPlan p = plan_backward(rows, in, out, T::kType, act);
  char *const ws = static_cast<char *>(workspace);
  float *const dw_parts = reinterpret_cast<float *>(ws + p.dw_parts);
  float *const db_parts = reinterpret_cast<float *>(ws + (dx != nullptr || dw != nullptr ? p.db_parts : 0));
  Plane dz = plane_of(dy);
  if (rows > 0 && (db != nullptr || act != GOSH_ACT_NONE)) {
    Plane to{nullptr, nullptr, 0, 0};
    if (act != GOSH_ACT_NONE && (dx != nullptr || dw != nullptr)) dz = to = Plane{ws + p.dz, nullptr, p.dz_ld, 0};
    slope_kernel<T><<<dim3(p.slope.blocks_x, p.slope.blocks_y), dim3(256), 0, st>>>(
        plane_of(dy), act == GOSH_ACT_NONE ? Plane{nullptr, nullptr, 0, 0} : plane_of(z), z != nullptr && z->packed, act, to,
        db != nullptr ? db_parts : nullptr, rows, out, p.slope.along, p.slope.rows_per_block);
    if (int rc = check_launch("gradient of the activation")) return rc;
  }
  JoinJob jobs[3];
  int sums = 0;
  if (db != nullptr) jobs[sums++] = {db_parts, out, out, out, db, static_cast<int32_t>(p.slope.blocks_y), out, GOSH_F32};
  // a packed x has its entries widened in registers: the alignment of its rows does not matter
  const bool dw_direct = T::kType != GOSH_F32 && dw != nullptr && can_be_direct(dz, out) &&
                         (x->packed ? in % 8 == 0 : can_be_direct(plane_of(x), in));
  const DwPlan &d = dw_direct ? p.dw_direct : p.dw;
  ProductArgs gx{}, gw{};
  if (dx != nullptr) {
    gx.a = dz;
    gx.b = plane_of(w);
    gx.N = in;
    gx.K = out;
    gx.out = plane_of(dx);
    if (p.dx_splits > 1) {
      gx.parts = reinterpret_cast<float *>(ws + p.dx_parts);
      gx.splits = p.dx_splits;
      const int64_t n = rows * in;
      jobs[sums++] = {gx.parts, n, n, dx->ld, dx->data, p.dx_splits, in, T::kType};
    }
  }
  if (dw != nullptr) {
    gw.a = dz;
    gw.b = plane_of(x);
    gw.direct = dw_direct;
    gw.M = out;
    gw.N = in;
    gw.K = rows;
    gw.k_per_split = d.k_per_split;
    gw.tiles_m = d.tiles_m;
    gw.tiles_n = d.tiles_n;
    gw.splits = d.splits;
    gw.parts = dw_parts;
    const int64_t n = static_cast<int64_t>(out) * in;
    jobs[sums++] = {dw_parts, n, n, dw->ld, dw->data, d.splits, in, dw->type};
  }
  if (rows > 0) {
    ProductArgs both = gx;
    if (dx != nullptr && dw != nullptr && d.size == kSmall && shape_rows<T>(kProductDx, rows, both) == kSmall &&
        static_cast<int64_t>(both.tiles_m) * both.tiles_n * both.splits <= kMostOfBoth) {
      if (int rc = launch_both<T>(x->packed != 0, both, gw, st)) return rc;
    } else {
      if (dx != nullptr)
        if (int rc = product_of_rows<T>(kProductDx, gx, rows, st)) return rc;
      if (dw != nullptr)
        if (int rc = launch_product<T>(x->packed ? kProductDwPacked : kProductDw, d.size, gw, st)) return rc;
    }
  }
  return join_parts(jobs, sums, st);
}

}  // namespace
}  // namespace gosh

extern "C" {

int gosh_linear(const gosh_mat *x, const gosh_mat *w, const float *bias, int32_t act, const gosh_mat *residual,
                const gosh_mat *y, const gosh_mat *z, const gosh_mat *y8, void *hip_stream) {
  using namespace gosh;
  if (int rc = check_mat(x, "x")) return rc;
  if (int rc = check_mat(w, "w")) return rc;
  if (int rc = check_mat(y, "y")) return rc;
  if (int rc = check_mat(residual, "residual", kOptional)) return rc;
  if (int rc = check_mat(z, "z", kOptional | kMayBePacked)) return rc;
  if (int rc = check_mat(y8, "y8", kOptional | kMustBePacked)) return rc;
  if (act < GOSH_ACT_NONE || act > GOSH_ACT_SILU) return fail(GOSH_EINVAL, "act = %d: no activation", act);
  if (w->rows < 1 || w->rows > GOSH_MAT_MAX_COLS)
    return fail(GOSH_EINVAL, "w: rows = %lld: must be in [1, %d]", (long long)w->rows, GOSH_MAT_MAX_COLS);
  const int32_t out = static_cast<int32_t>(w->rows);
  if (int rc = check_shape(w, "w", out, x->cols)) return rc;
  const struct { const gosh_mat *m; const char *what; } outs[] = {{y, "y"}, {residual, "residual"}, {z, "z"}, {y8, "y8"}};
  for (const auto &o : outs) {
    if (int rc = check_shape(o.m, o.what, x->rows, out)) return rc;
    if (int rc = check_type(o.m, o.what, x->type)) return rc;
  }
  if (int rc = check_type(w, "w", x->type)) return rc;
  if (int rc = check_floats(bias, out, "bias", true)) return rc;
  if (x->rows == 0) return GOSH_OK;
  hipStream_t st = as_stream(hip_stream);
  const int32_t past = z == nullptr && y8 == nullptr && x->rows * out * (x->type == GOSH_F32 ? 4 : 2) >= kPastCaches;
  ForwardOut f{bias, plane_of(residual), plane_of(y), plane_of(z), plane_of(y8), act, z != nullptr && z->packed, past};
  if (few_rows(x->rows, x->cols, out, x->type) && !f.z_packed && y8 == nullptr) {
    if (x->type == GOSH_F32) return launch_few_rows<F32>(x, w, f, st);
    if (x->type == GOSH_BF16) return launch_few_rows<Bf16>(x, w, f, st);
    return launch_few_rows<F16>(x, w, f, st);
  }
  ProductArgs g{};
  g.a = plane_of(x);
  g.b = plane_of(w);
  g.N = out;
  g.K = x->cols;
  g.forward = f;
  if (x->type == GOSH_F32) return product_of_rows<F32>(kProductForward, g, x->rows, st);
  if (x->type == GOSH_BF16) return product_of_rows<Bf16>(kProductForward, g, x->rows, st);
  return product_of_rows<F16>(kProductForward, g, x->rows, st);
}

uint64_t gosh_linear_backward_workspace(int64_t rows, int32_t in, int32_t out, int32_t type, int32_t act) {
  if (!gosh::rows_fit(rows) || in < 1 || out < 1 || in > GOSH_MAT_MAX_COLS || out > GOSH_MAT_MAX_COLS) return 0;
  if (type < GOSH_F32 || type > GOSH_F16 || act < GOSH_ACT_NONE || act > GOSH_ACT_SILU) return 0;
  return gosh::plan_backward(rows, in, out, type, act).bytes;
}

int gosh_linear_backward(const gosh_mat *dy, const gosh_mat *x, const gosh_mat *w, const gosh_mat *z, int32_t act,
                         const gosh_mat *dx, const gosh_mat *dw, float *db, void *workspace, uint64_t workspace_bytes,
                         void *hip_stream) {
  using namespace gosh;
  if (int rc = check_mat(dy, "dy")) return rc;
  if (int rc = check_mat(x, "x", kMayBePacked | (dw == nullptr ? kOptional : 0))) return rc;
  if (int rc = check_mat(w, "w", dx == nullptr ? kOptional : 0)) return rc;
  if (act < GOSH_ACT_NONE || act > GOSH_ACT_SILU) return fail(GOSH_EINVAL, "act = %d: no activation", act);
  if (int rc = check_mat(z, "z", kMayBePacked | (act == GOSH_ACT_NONE ? kOptional : 0))) return rc;
  if (int rc = check_mat(dx, "dx", kOptional)) return rc;
  if (int rc = check_mat(dw, "dw", kOptional)) return rc;
  const int32_t out = dy->cols;
  if (dx == nullptr && dw == nullptr && db == nullptr) return GOSH_OK;
  const int32_t in = dx != nullptr ? dx->cols : dw != nullptr ? dw->cols : x != nullptr ? x->cols : w != nullptr ? w->cols : 1;
  if (int rc = check_shape(x, "x", dy->rows, in)) return rc;
  if (int rc = check_shape(w, "w", out, in)) return rc;
  if (int rc = check_shape(z, "z", dy->rows, out)) return rc;
  if (int rc = check_shape(dx, "dx", dy->rows, in)) return rc;
  if (int rc = check_shape(dw, "dw", out, in)) return rc;
  const struct { const gosh_mat *m; const char *what; } all[] = {{x, "x"}, {w, "w"}, {z, "z"}, {dx, "dx"}};
  for (const auto &o : all)
    if (int rc = check_type(o.m, o.what, dy->type)) return rc;
  if (dw != nullptr && dw->type != GOSH_F32)
    if (int rc = check_type(dw, "dw", dy->type)) return rc;
  if (int rc = check_floats(db, out, "db", true)) return rc;
  const BackwardPlan plan = plan_backward(dy->rows, in, out, dy->type, act);
  if (int rc = check_workspace(workspace, workspace_bytes, dx != nullptr || dw != nullptr ? plan.bytes : plan.db_alone())) return rc;
  hipStream_t st = as_stream(hip_stream);
  if (dy->type == GOSH_F32) return linear_backward<F32>(dy, x, w, z, act, dx, dw, db, workspace, in, out, st);
  if (dy->type == GOSH_BF16) return linear_backward<Bf16>(dy, x, w, z, act, dx, dw, db, workspace, in, out, st);
  return linear_backward<F16>(dy, x, w, z, act, dx, dw, db, workspace, in, out, st);
}

}  // extern "C"
