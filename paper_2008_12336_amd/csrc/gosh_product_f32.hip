// Matrix products of the linear layer, entries of type F32.
#include "gosh_product.h"

namespace gosh {

template <>
int launch_product<F32>(ProductKind kind, TileSize size, const ProductArgs &args, hipStream_t st) {
  return launch_any<F32>(kind, size, args, st);
}

template <>
int launch_both<F32>(bool packed, const ProductArgs &dx, const ProductArgs &dw, hipStream_t st) {
  return launch_both_any<F32>(packed, dx, dw, st);
}

}  // namespace gosh
