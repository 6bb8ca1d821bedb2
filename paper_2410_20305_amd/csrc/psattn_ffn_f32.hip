// The feed-forward block's products: see psattn_ffn_tiles.h.
#include "psattn_ffn_tiles.h"

namespace psattn {
namespace gemm {

int product_f32(Pass pass, int act, bool pkc, bool qkc, TileSize size, const Product& d, hipStream_t s) { return launch_product<float, false>(pass, act, pkc, qkc, size, d, s); }

}  // namespace gemm
}  // namespace psattn
