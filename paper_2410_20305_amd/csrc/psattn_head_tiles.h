// The vocabulary head's products, on the tiles and the loop over k of psattn_ffn_tiles.h: see psattn_head.hip.
#pragma once
#include "psattn_ffn_tiles.h"
#include "psattn_head.h"

namespace psattn {
namespace gemm {

// The logits of few rows: W has to be read, with a third buffer of it on its way
template <typename E, bool ASYNC, Pass PASS>
int launch_logits(TileSize size, const Product& d, hipStream_t s) {
    constexpr int kBuffers = ASYNC ? 3 : 2;
    if (size == k32) return launch_tiles<E, ASYNC, true, true, PASS, 0, Shape<32, 128, 1, 2, kBuffers>>(d, s);
    if (size == k64) return launch_tiles<E, ASYNC, true, true, PASS, 0, Shape<64, 128, 1, 2, kBuffers>>(d, s);
    return launch_sized<E, ASYNC, true, true, PASS, 0>(size, d, s);
}

template <typename E, bool ASYNC>
int launch_head(Pass pass, TileSize size, const Product& d, hipStream_t s) {
    if (pass == kLse) return launch_logits<E, ASYNC, kLse>(size, d, s);
    if (pass == kDlogit) return launch_logits<E, ASYNC, kDlogit>(size, d, s);
    return launch_sized<E, ASYNC, true, false, kSums, 0>(size, d, s);
}

}  // namespace gemm
}  // namespace psattn
