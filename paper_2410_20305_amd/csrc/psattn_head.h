// The vocabulary head's products: what psattn_head.hip calls.
#pragma once
#include <hip/hip_runtime.h>

#include "psattn_ffn.h"

namespace psattn {
namespace gemm {

// One product (kLse, kDlogit: k contiguous in both operands; kSums: in P), enqueued on s.  Returns a psattn_status.
// bf16 where every row of P, Q and what is stored is whole 16-byte groups on 16-byte boundaries; bf16; fp32
int head_product_bf16(Pass pass, TileSize size, const Product& d, hipStream_t s);
int head_product_bf16_any(Pass pass, TileSize size, const Product& d, hipStream_t s);
int head_product_f32(Pass pass, TileSize size, const Product& d, hipStream_t s);

}  // namespace gemm
}  // namespace psattn
