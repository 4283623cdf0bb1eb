// Matrix products of the linear layer, entries of type F32.
#include "gosh_product.h"

namespace gosh {

template <>
int launch_product<F32>(ProductKind kind, bool small, const ProductArgs &args, hipStream_t st) {
  return small ? launch_sized<F32, 64>(kind, args, st) : launch_sized<F32, 128>(kind, args, st);
}

}  // namespace gosh
