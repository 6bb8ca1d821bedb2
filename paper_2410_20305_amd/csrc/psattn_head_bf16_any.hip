// The vocabulary head's products: see psattn_head_tiles.h.
#include "psattn_head_tiles.h"

namespace psattn {
namespace gemm {

int head_product_bf16_any(Pass pass, bool qkc, TileSize size, const Product& d, hipStream_t s) { return launch_head<uint16_t, false>(pass, qkc, size, d, s); }

}  // namespace gemm
}  // namespace psattn
