// The vocabulary head's products: what psattn_head.hip calls.
#pragma once
#include <hip/hip_runtime.h>

#include "psattn_ffn.h"

namespace psattn {
namespace gemm {

// One product (k is the contiguous axis of P, and of Q with kLse, kDlogit, or as kSums is told), enqueued on s.  Returns a psattn_status.
// bf16 and fp32, where every row of P and Q is whole 16-byte groups on 16-byte boundaries, and of any alignment
int head_product_bf16(Pass pass, bool qkc, TileSize size, const Product& d, hipStream_t s);
int head_product_bf16_any(Pass pass, bool qkc, TileSize size, const Product& d, hipStream_t s);
int head_product_f32_whole(Pass pass, bool qkc, TileSize size, const Product& d, hipStream_t s);
int head_product_f32(Pass pass, bool qkc, TileSize size, const Product& d, hipStream_t s);

// dW of bf16 (kTokens); dz and the rows of X are whole
int head_tokens_bf16(TileSize size, const Product& w, hipStream_t s);
// dX's sums and dW (kTokens, of fp32 kPlain) of a piece in one launch, of tiles of 256 x 256, or 128 x 128 of fp32; dz and the rows of X are whole, W may be not in fp32
int head_grads_bf16(const Product& x, const Product& w, hipStream_t s);
int head_grads_f32_whole(const Product& x, const Product& w, hipStream_t s);
int head_grads_f32(const Product& x, const Product& w, hipStream_t s);
// dW alone, of few items: k is theirs, and behind them stand rows of zeros up to a multiple of 64.  bf16: as kTokens, where there is an out[1]
int head_outer_bf16(const Product& w, hipStream_t s);
int head_outer_f32(const Product& w, hipStream_t s);

}  // namespace gemm
}  // namespace psattn
