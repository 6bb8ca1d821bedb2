// The feed-forward block's products: what psattn_ffn.hip (arguments, order of the products) calls.
#pragma once
#include <hip/hip_runtime.h>

#include "psattn_gemm.h"

namespace psattn {
namespace gemm {

// One product, enqueued on s.  pkc, qkc: k is the contiguous axis of P, Q.  Returns a psattn_status.
int product_any(int dt, Pass pass, int act, bool pkc, bool qkc, const Product& d, hipStream_t s);
// The same for bf16 where product_mfma_ok says so.
bool product_mfma_ok(bool pkc, bool qkc, const Product& d);
int product_mfma(Pass pass, int act, bool pkc, bool qkc, const Product& d, hipStream_t s);

}  // namespace gemm
}  // namespace psattn
