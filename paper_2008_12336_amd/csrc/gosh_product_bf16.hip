// Matrix products of the linear layer, entries of type Bf16.
#include "gosh_product.h"

namespace gosh {

template <>
int launch_product<Bf16>(ProductKind kind, TileSize size, const ProductArgs &args, hipStream_t st) {
  return launch_any<Bf16>(kind, size, args, st);
}

template <>
int launch_both<Bf16>(bool packed, const ProductArgs &dx, const ProductArgs &dw, hipStream_t st) {
  return launch_both_any<Bf16>(packed, dx, dw, st);
}

}  // namespace gosh
