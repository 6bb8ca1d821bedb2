// The vocabulary head's products: see psattn_head_tiles.h.
#include "psattn_head_tiles.h"

namespace psattn {
namespace gemm {

int head_product_f32_whole(Pass pass, bool qkc, TileSize size, const Product& d, hipStream_t s) { return launch_head<float, true>(pass, qkc, size, d, s); }

int head_grads_f32_whole(const Product& x, const Product& w, hipStream_t s) { return launch_grads<float, true>(x, w, s); }

// dz and the rows of X are whole in either of dW's products
int head_outer_f32(const Product& w, hipStream_t s) { return launch_outer<float, true>(w, s); }

}  // namespace gemm
}  // namespace psattn
