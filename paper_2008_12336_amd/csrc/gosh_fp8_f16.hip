// Matrix products in 8-bit floating point, results of type F16.
#include "gosh_fp8_product.h"

namespace gosh {

template <>
int launch_fp8<F16>(ProductOut out, const Fp8Args &args, hipStream_t st) {
  return launch_fp8_any<F16>(out, args, st);
}

template <>
int launch_fp8_gradients<F16>(const Fp8Args &dx, const Fp8Args &dw, int32_t dw_type, const JoinJob &db, hipStream_t st) {
  if (dw_type == GOSH_F32) return launch_fp8_few_gradients<F16, F32>(dx, dw, db, st);
  return launch_fp8_few_gradients<F16, F16>(dx, dw, db, st);
}

}  // namespace gosh
