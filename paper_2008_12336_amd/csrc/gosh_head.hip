// What the units of the head share: checks of matrix arguments, the sum of partial results, and the 8-bit form.
#include "gosh_head.h"

#include <algorithm>

namespace gosh {

namespace {

size_t entry_bytes(const gosh_mat *m) { return m->packed ? 1 : m->type == GOSH_F32 ? 4 : 2; }

}  // namespace

int check_mat(const gosh_mat *m, const char *what, int use) {
  if (m == nullptr) return (use & kOptional) ? GOSH_OK : fail(GOSH_EINVAL, "%s is null", what);
  if (m->type != GOSH_F32 && m->type != GOSH_BF16 && m->type != GOSH_F16)
    return fail(GOSH_EINVAL, "%s: type %d is none of gosh_type", what, m->type);
  if (m->packed != 0 && m->packed != 1) return fail(GOSH_EINVAL, "%s: packed = %d: must be 0 or 1", what, m->packed);
  if (m->packed && !(use & (kMayBePacked | kMustBePacked))) return fail(GOSH_EINVAL, "%s must not be packed", what);
  if (!m->packed && (use & kMustBePacked)) return fail(GOSH_EINVAL, "%s must be packed", what);
  if (!rows_fit(m->rows))
    return fail(GOSH_EINVAL, "%s: rows = %lld: must be in [0, 2^31-1)", what, (long long)m->rows);
  if (m->cols < 1 || m->cols > GOSH_MAT_MAX_COLS)
    return fail(GOSH_EINVAL, "%s: cols = %d: must be in [1, %d]", what, m->cols, GOSH_MAT_MAX_COLS);
  if (m->ld < m->cols || m->ld > GOSH_MAT_MAX_LD)
    return fail(GOSH_EINVAL, "%s: ld = %lld: must be in [cols, %d]", what, (long long)m->ld, GOSH_MAT_MAX_LD);
  if (m->rows == 0) return GOSH_OK;
  if (m->data == nullptr) return fail(GOSH_EINVAL, "%s: data is null", what);
  const size_t size = entry_bytes(m);
  if (reinterpret_cast<uintptr_t>(m->data) % size != 0)
    return fail(GOSH_EINVAL, "%s: data must be aligned to its entries of %zu bytes", what, size);
  if (int rc = check_device_span(m->data, (static_cast<size_t>(m->rows - 1) * m->ld + m->cols) * size, what)) return rc;
  if (m->packed) {
    const int64_t groups = ceil_div(m->cols, kGroup);
    if (m->exps == nullptr) return fail(GOSH_EINVAL, "%s: exps is null", what);
    if (m->ld_exps < groups || m->ld_exps > GOSH_MAT_MAX_LD)
      return fail(GOSH_EINVAL, "%s: ld_exps = %lld: must be in [ceil(cols / 32), %d]", what, (long long)m->ld_exps, GOSH_MAT_MAX_LD);
    return check_device_span(m->exps, static_cast<size_t>(m->rows - 1) * m->ld_exps + groups, what);
  }
  return GOSH_OK;
}

int check_shape(const gosh_mat *m, const char *what, int64_t rows, int32_t cols) {
  if (m != nullptr && (m->rows != rows || m->cols != cols))
    return fail(GOSH_EINVAL, "%s is %lld x %d: must be %lld x %d", what, (long long)m->rows, m->cols, (long long)rows, cols);
  return GOSH_OK;
}

int check_type(const gosh_mat *m, const char *what, int32_t type) {
  if (m != nullptr && m->type != type) return fail(GOSH_EINVAL, "%s: type %d: must be %d as the others'", what, m->type, type);
  return GOSH_OK;
}

int check_floats(const float *p, int64_t count, const char *what, bool optional) {
  if (p == nullptr) return optional || count == 0 ? GOSH_OK : fail(GOSH_EINVAL, "%s is null", what);
  if (reinterpret_cast<uintptr_t>(p) % 4 != 0) return fail(GOSH_EINVAL, "%s must be 4-byte aligned", what);
  return count == 0 ? GOSH_OK : check_device_span(p, static_cast<size_t>(count) * 4, what);
}

int check_workspace(const void *p, uint64_t have, uint64_t need) {
  if (need == 0) return GOSH_OK;
  if (p == nullptr || have < need)
    return fail(GOSH_EINVAL, "workspace: %llu bytes are needed", (unsigned long long)need);
  if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return fail(GOSH_EINVAL, "workspace must be 16-byte aligned");
  return check_device_span(p, need, "workspace");
}

// ---- sums of partial results --------------------------------------------------------------

namespace {

__device__ __forceinline__ void store_sum(float sum, int64_t i, int32_t cols, void *out, int64_t ld, int32_t type) {
  const int64_t to = i / cols * ld + i % cols;
  if (type == GOSH_F32) static_cast<float *>(out)[to] = sum;
  else if (type == GOSH_BF16) static_cast<__bf16 *>(out)[to] = static_cast<__bf16>(sum);
  else static_cast<_Float16 *>(out)[to] = static_cast<_Float16>(sum);
}

constexpr int kMostJobs = 3;
struct JoinJobs {
  JoinJob job[kMostJobs];
  unsigned first[kMostJobs + 1];  // workgroup of each job; the last: how many there are
};

// Few entries have few threads to sum their many parts: 16 share them then.
__host__ __device__ inline bool shared(const JoinJob &j) { return j.n <= 16384 && j.count > 16; }

__global__ __launch_bounds__(256) void join_kernel(const JoinJobs jobs) {
  const int which = blockIdx.x < jobs.first[1] ? 0 : blockIdx.x < jobs.first[2] ? 1 : 2;
  const JoinJob &j = jobs.job[which];
  const int64_t block = blockIdx.x - jobs.first[which];
  if (!shared(j)) {
    const int64_t step = static_cast<int64_t>(jobs.first[which + 1] - jobs.first[which]) * 256;
    for (int64_t i = block * 256 + threadIdx.x; i < j.n; i += step) {
      float sum = 0.f;
#pragma unroll 8
      for (int s = 0; s < j.count; ++s) sum += j.parts[s * j.stride + i];
      store_sum(sum, i, j.cols, j.out, j.ld, j.type);
    }
    return;
  }
  __shared__ float lds[256];
  const int x = threadIdx.x % 16, y = threadIdx.x / 16;
  const int64_t i = block * 16 + x;
  float sum = 0.f;
  if (i < j.n)
#pragma unroll 8
    for (int s = y; s < j.count; s += 16) sum += j.parts[s * j.stride + i];
  lds[threadIdx.x] = sum;
  __syncthreads();
  if (y != 0 || i >= j.n) return;
#pragma unroll
  for (int s = 1; s < 16; ++s) sum += lds[s * 16 + x];
  store_sum(sum, i, j.cols, j.out, j.ld, j.type);
}

}  // namespace

int join_parts(const JoinJob *jobs, int how_many, hipStream_t st) {
  if (how_many == 0) return GOSH_OK;
  const auto blocks = [](const JoinJob &j) {
    return static_cast<unsigned>(std::min<int64_t>(ceil_div(j.n, shared(j) ? 16 : 256), 1 << 20));
  };
  JoinJobs all{};
  for (int i = 0; i < kMostJobs; ++i) {
    if (i < how_many) all.job[i] = jobs[i];
    all.first[i + 1] = all.first[i] + (i < how_many ? blocks(jobs[i]) : 0);
  }
  join_kernel<<<dim3(all.first[kMostJobs]), dim3(256), 0, st>>>(all);
  return check_launch("sum of parts");
}

// ---- the 8-bit form -------------------------------------------------------------------------

namespace {

// A lane has 8 columns, four lanes a group; 64 groups a workgroup and turn.  Bound by memory: 2^20 x 512 in bf16 are packed
// in 290 us and unpacked in 265, 5.6 and 6.1 TB/s (reads are cheaper than writes).
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const Plane x, const Plane q, int64_t rows, int32_t cols, int32_t groups) {
  const int64_t total = rows * groups;
  const int sub = threadIdx.x & 3;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x / 4; i < total; i += static_cast<int64_t>(gridDim.x) * 64) {
    const int64_t row = i / groups;
    const int col = static_cast<int>(i - row * groups) * kGroup + 8 * sub;
    const int count = cols - col < 8 ? cols - col : 8;
    float v[8];
    load_entries<T, 8>(x, false, row, col, count, v);
    store_packed<T, 8>(q, row, col, count, v, sub == 0, 4);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void unpack_kernel(const Plane q, const Plane x, int64_t rows, int32_t cols, int32_t groups) {
  const int64_t total = rows * groups;
  const int sub = threadIdx.x & 3;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x / 4; i < total; i += static_cast<int64_t>(gridDim.x) * 64) {
    const int64_t row = i / groups;
    const int col = static_cast<int>(i - row * groups) * kGroup + 8 * sub;
    const int count = cols - col < 8 ? cols - col : 8;
    if (count <= 0) continue;
    float v[8];
    load_entries<T, 8>(q, true, row, col, count, v);
    Entries<T, 8>::store(static_cast<typename T::Store *>(x.data) + row * x.ld + col, count, v);
  }
}

template <typename T>
void launch_pack(const gosh_mat *x, const gosh_mat *q, bool back, hipStream_t st) {
  const int32_t groups = static_cast<int32_t>(ceil_div(x->cols, kGroup));
  const int64_t blocks = std::min<int64_t>(ceil_div(x->rows * groups, 64), int64_t{1} << 22);
  if (back)
    unpack_kernel<T><<<dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st>>>(plane_of(q), plane_of(x), x->rows, x->cols, groups);
  else
    pack_kernel<T><<<dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st>>>(plane_of(x), plane_of(q), x->rows, x->cols, groups);
}

int pack_either(const gosh_mat *x, const gosh_mat *q, bool back, void *stream) {
  if (int rc = check_mat(x, "x")) return rc;
  if (int rc = check_mat(q, "q", kMustBePacked)) return rc;
  if (int rc = check_shape(q, "q", x->rows, x->cols)) return rc;
  if (!back)
    if (int rc = check_type(q, "q", x->type)) return rc;
  if (x->rows == 0) return GOSH_OK;
  hipStream_t st = as_stream(stream);
  if (x->type == GOSH_F32) launch_pack<F32>(x, q, back, st);
  else if (x->type == GOSH_BF16) launch_pack<Bf16>(x, q, back, st);
  else launch_pack<F16>(x, q, back, st);
  return check_launch(back ? "unpack" : "pack");
}

}  // namespace
}  // namespace gosh

extern "C" {

int gosh_pack8(const gosh_mat *x, const gosh_mat *q, void *hip_stream) { return gosh::pack_either(x, q, false, hip_stream); }

int gosh_unpack8(const gosh_mat *q, const gosh_mat *x, void *hip_stream) { return gosh::pack_either(x, q, true, hip_stream); }

}  // extern "C"
