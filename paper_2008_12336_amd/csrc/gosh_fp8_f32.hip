// Matrix products in 8-bit floating point, results of type F32.
#include "gosh_fp8_product.h"

namespace gosh {

template <>
int launch_fp8<F32>(ProductOut out, const Fp8Args &args, hipStream_t st) {
  return launch_fp8_any<F32>(out, args, st);
}

}  // namespace gosh
