// Matrix products of the linear layer, entries of type Bf16.
#include "gosh_product.h"

namespace gosh {

template <>
int launch_product<Bf16>(ProductKind kind, bool small, const ProductArgs &args, hipStream_t st) {
  return small ? launch_sized<Bf16, 64>(kind, args, st) : launch_sized<Bf16, 128>(kind, args, st);
}

}  // namespace gosh
