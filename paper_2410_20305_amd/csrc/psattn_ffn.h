// The feed-forward block's products: what psattn_ffn.hip (arguments, order and sizes of the products) calls.
#pragma once
#include <hip/hip_runtime.h>

#include "psattn_gemm.h"

namespace psattn {
namespace gemm {

// m x n of a workgroup's tile: 32 x 128, 64 x 128, 128 x 128, 256 x 256 (kGate: half the n, of two matrices)
enum TileSize { k32, k64, k128, k256 };

// One product, enqueued on s.  pkc, qkc: k is the contiguous axis of P, Q.  Returns a psattn_status.
// bf16 where every row of P, Q and what is stored is whole 16-byte groups on 16-byte boundaries; bf16; fp32
int product_bf16(Pass pass, int act, bool pkc, bool qkc, TileSize size, const Product& d, hipStream_t s);
int product_bf16_any(Pass pass, int act, bool pkc, bool qkc, TileSize size, const Product& d, hipStream_t s);
int product_f32(Pass pass, int act, bool pkc, bool qkc, TileSize size, const Product& d, hipStream_t s);

}  // namespace gemm
}  // namespace psattn
