// Matrix products in 8-bit floating point, results of type F32.
#include "gosh_fp8_product.h"

namespace gosh {

template <>
int launch_fp8<F32>(ProductOut out, const Fp8Args &args, hipStream_t st) {
  return launch_fp8_any<F32>(out, args, st);
}

template <>
int launch_fp8_gradients<F32>(const Fp8Args &dx, const Fp8Args &dw, int32_t dw_type, const JoinJob &db, hipStream_t st) {
  return launch_fp8_few_gradients<F32, F32>(dx, dw, db, st);
}

}  // namespace gosh
