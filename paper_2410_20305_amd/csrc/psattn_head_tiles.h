// The vocabulary head's products, on the tiles and the loop over k of psattn_ffn_tiles.h: see psattn_head.hip.
#pragma once
#include "psattn_ffn_tiles.h"
#include "psattn_head.h"

namespace psattn {
namespace gemm {

template <typename E, bool ASYNC>
int launch_head(Pass pass, TileSize size, const Product& d, hipStream_t s) {
    if (pass == kLse) return launch_sized<E, ASYNC, true, true, kLse, 0>(size, d, s);
    if (pass == kDlogit) return launch_sized<E, ASYNC, true, true, kDlogit, 0>(size, d, s);
    return launch_sized<E, ASYNC, true, false, kSums, 0>(size, d, s);
}

}  // namespace gemm
}  // namespace psattn
