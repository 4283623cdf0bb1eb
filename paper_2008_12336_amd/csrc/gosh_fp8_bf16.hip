// Matrix products in 8-bit floating point, results of type Bf16.
#include "gosh_fp8_product.h"

namespace gosh {

template <>
int launch_fp8<Bf16>(ProductOut out, const Fp8Args &args, hipStream_t st) {
  return launch_fp8_any<Bf16>(out, args, st);
}

template <>
int launch_fp8_gradients<Bf16>(const Fp8Args &dx, const Fp8Args &dw, int32_t dw_type, const JoinJob &db, hipStream_t st) {
  if (dw_type == GOSH_F32) return launch_fp8_few_gradients<Bf16, F32>(dx, dw, db, st);
  return launch_fp8_few_gradients<Bf16, Bf16>(dx, dw, db, st);
}

}  // namespace gosh
