// The vocabulary head's products: see psattn_head_tiles.h.
#include "psattn_head_tiles.h"

namespace psattn {
namespace gemm {

int head_product_f32(Pass pass, bool qkc, TileSize size, const Product& d, hipStream_t s) { return launch_head<float, false>(pass, qkc, size, d, s); }
int head_grads_f32(const Product& x, const Product& w, hipStream_t s) { return launch_grads<float, false>(x, w, s); }

}  // namespace gemm
}  // namespace psattn
