// Matrix products of the linear layer, entries of type F32.
#include "gosh_product.h"

namespace gosh {

template <>
int launch_product<F32>(ProductKind kind, TileSize size, const ProductArgs &args, hipStream_t st) {
  return launch_any<F32>(kind, size, args, st);
}

}  // namespace gosh
