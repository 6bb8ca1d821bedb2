// The vocabulary head's products: see psattn_head_tiles.h.
#include "psattn_head_tiles.h"

namespace psattn {
namespace gemm {

int head_product_bf16(Pass pass, bool qkc, TileSize size, const Product& d, hipStream_t s) { return launch_head<uint16_t, true>(pass, qkc, size, d, s); }
int head_tokens_bf16(TileSize size, const Product& w, hipStream_t s) { return launch_sized<uint16_t, true, false, false, kTokens, 0>(size, w, s); }
int head_outer_bf16(const Product& w, hipStream_t s) { return launch_outer<uint16_t, true>(w, s); }

int head_grads_bf16(const Product& x, const Product& w, hipStream_t s) { return launch_grads<uint16_t, true>(x, w, s); }

}  // namespace gemm
}  // namespace psattn
