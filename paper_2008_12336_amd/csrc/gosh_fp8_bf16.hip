// Matrix products in 8-bit floating point, results of type Bf16.
#include "gosh_fp8_product.h"

namespace gosh {

template <>
int launch_fp8<Bf16>(ProductOut out, const Fp8Args &args, hipStream_t st) {
  return launch_fp8_any<Bf16>(out, args, st);
}

}  // namespace gosh
