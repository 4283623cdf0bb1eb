// Host-only exercise of the host code of the 8-bit layers, the optimiser and the loss under AddressSanitizer and
// UndefinedBehaviorSanitizer (built and run by tests/test_step_sanitizers.py): plans, workspaces and states over the whole
// range of sizes, and every refusal that comes before a device call, so it runs without a GPU.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <random>
#include "gosh.h"

static int failures = 0;

static void expect(bool ok, const char *what) {
  if (!ok) printf("%s: %s\n", what, gosh_last_error()), ++failures;
}

static bool refused(int rc, const char *text) { return rc == GOSH_EINVAL && strstr(gosh_last_error(), text) != nullptr; }

int main() {
  std::mt19937_64 rng(12);
  const auto size = [&](int bits) { return static_cast<int64_t>(rng() >> (64 - 1 - rng() % bits)); };  // of any magnitude
  for (int trial = 0; trial < 100000; ++trial) {
    int64_t rows = size(31), in = 1 + size(16), out = 1 + size(16);
    if (rows > 2147483646) rows = 2147483646;
    in = in > 65536 ? 65536 : in, out = out > 65536 ? 65536 : out;
    const uint64_t need = gosh_linear_fp8_backward_workspace(rows, in, out);
    expect(rows == 0 ? need == 0 : need % 256 == 0 && need >= 2 * static_cast<uint64_t>(rows) * out, "workspace of a layer");
    // anything at all
    gosh_linear_fp8_backward_workspace(static_cast<int64_t>(rng()), static_cast<int32_t>(rng()), static_cast<int32_t>(rng()));
    const int64_t n = size(41);
    for (int32_t bits : {8, 32}) {
      const uint64_t state = gosh_adamw_state_bytes(n, bits);
      expect(n <= 0 || n > (int64_t{1} << 40) ? state == 0 : state >= static_cast<uint64_t>(n) * bits / 4, "bytes of a state");
    }
    expect(gosh_adamw_state_bytes(static_cast<int64_t>(rng()), static_cast<int32_t>(rng() | 64)) == 0, "bits that are none");
  }
  const gosh_mat m{nullptr, nullptr, 0, 128, 4, 128, GOSH_F32, 0};
  const gosh_fp8 f{nullptr, nullptr, 0, 128, 128, 4, 1};
  for (int64_t v : {INT64_MIN, int64_t{-1}, INT64_MAX, int64_t{130}}) {
    for (int field = 0; field < 4; ++field) {
      gosh_fp8 b = f;
      if (v == 130 && field < 2) continue;
      (field == 0 ? b.rows : field == 1 ? b.cols : field == 2 ? b.ld : b.ld_exps) = v;
      expect(gosh_pack_fp8(&m, &b, nullptr, nullptr) == GOSH_EINVAL && gosh_pack_fp8(&m, nullptr, &b, nullptr) == GOSH_EINVAL &&
                 gosh_unpack_fp8(&b, &m, nullptr) == GOSH_EINVAL, "forms that are none");
      expect(gosh_linear_fp8(nullptr, &b, &f, nullptr, 0, nullptr, &m, nullptr, nullptr) == GOSH_EINVAL, "x8");
      expect(gosh_linear_fp8(nullptr, &f, &b, nullptr, 0, nullptr, &m, nullptr, nullptr) == GOSH_EINVAL, "w");
      expect(gosh_linear_fp8_backward(&m, &b, &f, nullptr, 0, nullptr, &m, nullptr, nullptr, 0, nullptr) == GOSH_EINVAL, "xt");
      expect(gosh_linear_fp8_backward(&m, nullptr, &b, nullptr, 0, &m, nullptr, nullptr, nullptr, 0, nullptr) == GOSH_EINVAL, "wt");
    }
  }
  expect(refused(gosh_linear_fp8(nullptr, &f, &f, nullptr, 0, nullptr, &m, nullptr, nullptr), "w: rows"), "w of no rows");
  expect(refused(gosh_linear_fp8_backward(&m, nullptr, nullptr, nullptr, 0, nullptr, nullptr, nullptr, nullptr, 0, nullptr), "dx and dw"), "db alone");
  expect(gosh_pack_fp8(&m, &f, nullptr, nullptr) == GOSH_OK && gosh_unpack_fp8(&f, &m, nullptr) == GOSH_OK, "nothing to pack");
  expect(gosh_softmax_loss(&m, nullptr, 0, nullptr, 1.f, nullptr, &m, nullptr) == GOSH_OK, "no rows");
  expect(refused(gosh_softmax_loss(&m, nullptr, -1, nullptr, 1.f, nullptr, nullptr, nullptr), "targets_are64"), "targets");

  float word = 0;
  gosh_param q{&word, &word, &word, nullptr, 1, GOSH_F32, GOSH_BF16, 8, 0.f};
  void *out = &word;
  for (int64_t n : {int64_t{-1}, INT64_MIN, INT64_MAX, (int64_t{1} << 40) + 1}) {
    gosh_param b = q;
    b.n = n;
    expect(refused(gosh_adamw_create(&b, 1, &out), "n =") && out == nullptr, "sizes");
  }
  for (int32_t v : {-1, 3, INT32_MAX}) {
    gosh_param b = q;
    b.g_type = v;
    expect(refused(gosh_adamw_create(&b, 1, &out), "g_type"), "types");
    b = q, b.bits = v;
    expect(refused(gosh_adamw_create(&b, 1, &out), "bits"), "bits");
    b = q, b.copy = &word, b.copy_type = v;
    expect(refused(gosh_adamw_create(&b, 1, &out), "copy_type"), "copies");
  }
  expect(refused(gosh_adamw_create(nullptr, 1, &out), "params is null") && refused(gosh_adamw_create(&q, INT32_MIN, &out), "count"), "tensors");
  gosh_adamw_options ok{1e-3, 0.9, 0.999, 1e-8, 1, nullptr, nullptr, nullptr};
  for (double v : {-1.0, 1.0, static_cast<double>(NAN), static_cast<double>(INFINITY)}) {
    gosh_adamw_options b = ok;
    b.beta1 = v;
    expect(refused(gosh_adamw_step(nullptr, &b, nullptr), "beta1"), "beta1");
    b = ok, b.beta2 = v;
    expect(refused(gosh_adamw_step(nullptr, &b, nullptr), "beta2"), "beta2");
  }
  for (int64_t t : {int64_t{0}, INT64_MIN}) {
    gosh_adamw_options b = ok;
    b.step = t;
    expect(refused(gosh_adamw_step(nullptr, &b, nullptr), "step ="), "step");
  }
  expect(refused(gosh_adamw_step(nullptr, &ok, nullptr), "optimiser is null"), "no optimiser");
  gosh_adamw_free(nullptr);
  if (failures == 0) printf("step driver ok\n");
  return failures != 0;
}
