// Host-only exercise of the head's host code under AddressSanitizer and UndefinedBehaviorSanitizer (built and run by
// tests/test_head_sanitizers.py): plans and workspaces over the whole range of sizes, and every refusal that comes before a
// device call, so it runs without a GPU.
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <random>
#include "gosh.h"

static int failures = 0;

static void expect(bool ok, const char *what) {
  if (!ok) printf("%s: %s\n", what, gosh_last_error()), ++failures;
}

static gosh_mat mat(int64_t rows, int32_t cols, int32_t type = GOSH_F32, int32_t packed = 0) {
  return {nullptr, nullptr, rows, cols, (cols + 31) / 32, cols, type, packed};
}

static bool refused(int rc, const char *text) { return rc == GOSH_EINVAL && strstr(gosh_last_error(), text) != nullptr; }

int main() {
  std::mt19937_64 rng(11);
  const auto size = [&](int bits) { return static_cast<int64_t>(rng() >> (64 - 1 - rng() % bits)); };  // of any magnitude
  for (int trial = 0; trial < 200000; ++trial) {
    int64_t rows = size(31), in = 1 + size(16), out = 1 + size(16);
    if (rows > 2147483646) rows = 2147483646;
    in = in > 65536 ? 65536 : in, out = out > 65536 ? 65536 : out;
    const int32_t type = rng() % 3, act = rng() % 4;
    const uint64_t need = gosh_linear_backward_workspace(rows, in, out, type, act);
    const uint64_t bare = gosh_linear_backward_workspace(rows, in, out, type, GOSH_ACT_NONE);
    expect(rows == 0 ? need == 0 : need % 256 == 0 && bare >= static_cast<uint64_t>(in) * out * 4 + out * 4, "workspace of a layer");
    expect(need >= bare + (act == GOSH_ACT_NONE ? 0 : static_cast<uint64_t>(rows) * out * (type == GOSH_F32 ? 4 : 2)), "workspace of dz");
    const uint64_t norm = gosh_layer_norm_workspace(rows, in);
    expect(rows == 0 ? norm == 0 : norm % (8 * in) == 0 && norm <= 1024 * 8 * static_cast<uint64_t>(in), "workspace of a norm");
    // anything at all
    gosh_linear_backward_workspace(static_cast<int64_t>(rng()), static_cast<int32_t>(rng()), static_cast<int32_t>(rng()),
                                   static_cast<int32_t>(rng() % 5) - 1, static_cast<int32_t>(rng() % 6) - 1);
    gosh_layer_norm_workspace(static_cast<int64_t>(rng()), static_cast<int32_t>(rng()));
  }
  for (int64_t rows : {INT64_MAX, INT64_MIN, int64_t{2147483647}, int64_t{-1}}) {
    expect(gosh_linear_backward_workspace(rows, 64, 64, GOSH_BF16, GOSH_ACT_GELU) == 0, "rows that are none");
    expect(gosh_layer_norm_workspace(rows, 64) == 0, "rows that are none");
  }

  const gosh_mat m = mat(0, 8), q = mat(0, 8, GOSH_F32, 1);
  gosh_mat bad[] = {mat(-1, 8), mat(INT64_MAX, 8), mat(0, 0), mat(0, 65537), mat(0, INT32_MIN), mat(0, 8, 3), mat(0, 8, -1), mat(0, 8, 0, 2), mat(1, 8)};
  for (const gosh_mat &b : bad)
    for (const gosh_mat *other : {&m, &q}) {
      expect(gosh_linear(&b, other, nullptr, 0, nullptr, other, nullptr, nullptr, nullptr) == GOSH_EINVAL, "linear");
      expect(gosh_linear_backward(&b, other, nullptr, nullptr, 0, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == GOSH_EINVAL, "backward");
      expect(gosh_layer_norm(&b, nullptr, nullptr, 0.f, other, nullptr, nullptr, nullptr, nullptr, nullptr) == GOSH_EINVAL, "norm");
      expect(gosh_layer_norm_backward(&b, other, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == GOSH_EINVAL, "norm backward");
      expect(gosh_pack8(&b, other, nullptr) == GOSH_EINVAL && gosh_unpack8(other, &b, nullptr) == GOSH_EINVAL, "pack");
    }
  for (int64_t ld : {int64_t{7}, int64_t{0}, INT64_MIN, int64_t{GOSH_MAT_MAX_LD + 1}, INT64_MAX}) {
    gosh_mat b = m;
    b.ld = ld;
    expect(refused(gosh_pack8(&b, &q, nullptr), "ld"), "ld");
  }
  const gosh_mat wide = mat(0, 9), half = mat(0, 8, GOSH_F16), half8 = mat(0, 8, GOSH_F16, 1);
  expect(refused(gosh_pack8(&wide, &q, nullptr), "must be 0 x 9"), "shapes");
  expect(refused(gosh_pack8(&half, &q, nullptr), "type"), "types");
  expect(gosh_pack8(&m, &q, nullptr) == GOSH_OK && gosh_unpack8(&q, &half, nullptr) == GOSH_OK, "nothing to pack");
  expect(refused(gosh_layer_norm(&m, nullptr, nullptr, -1.f, &m, nullptr, nullptr, nullptr, nullptr, nullptr), "eps"), "eps");
  expect(refused(gosh_layer_norm(&m, nullptr, nullptr, 0.f, &m, nullptr, nullptr, &half8, nullptr, nullptr), "xhat8: type"), "xhat8");
  expect(refused(gosh_layer_norm(&m, nullptr, nullptr, 0.f, &m, nullptr, nullptr, &q, &m, nullptr), "y8 must be packed"), "y8");
  expect(refused(gosh_layer_norm(&m, nullptr, nullptr, 0.f, &m, nullptr, nullptr, &q, &q, nullptr), "gamma is null"), "gamma");
  float one = 0;
  expect(refused(gosh_layer_norm_backward(&m, &m, nullptr, nullptr, nullptr, nullptr, nullptr, &one, nullptr, nullptr, 0, nullptr), "both or neither"), "dgamma");
  for (int32_t act : {-1, 4, INT32_MAX, INT32_MIN}) {
    expect(refused(gosh_linear(&m, &m, nullptr, act, nullptr, &m, nullptr, nullptr, nullptr), "act"), "act");
    expect(refused(gosh_linear_backward(&m, nullptr, nullptr, nullptr, act, nullptr, nullptr, nullptr, nullptr, 0, nullptr), "act"), "act");
  }
  expect(refused(gosh_linear(&m, &m, nullptr, 0, nullptr, &m, nullptr, nullptr, nullptr), "w: rows"), "w of no rows");
  expect(refused(gosh_linear_backward(&m, &m, nullptr, nullptr, GOSH_ACT_SILU, nullptr, nullptr, &one, nullptr, 0, nullptr), "z is null"), "z");
  expect(refused(gosh_linear_backward(&m, nullptr, nullptr, nullptr, 0, &m, nullptr, nullptr, nullptr, 0, nullptr), "w is null"), "w");
  expect(refused(gosh_linear_backward(&m, nullptr, nullptr, nullptr, 0, nullptr, &m, nullptr, nullptr, 0, nullptr), "x is null"), "x");
  expect(gosh_linear_backward(&m, nullptr, nullptr, nullptr, 0, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == GOSH_OK, "nothing asked for");
  if (failures == 0) printf("head driver ok\n");
  return failures != 0;
}
