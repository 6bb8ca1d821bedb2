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
int launch_head(Pass pass, bool qkc, TileSize size, const Product& d, hipStream_t s) {
    if (pass == kLse) return launch_logits<E, ASYNC, kLse>(size, d, s);
    if (pass == kDlogit) return launch_logits<E, ASYNC, kDlogit>(size, d, s);
    if (qkc) return launch_logits<E, ASYNC, kSums>(size, d, s);
    return launch_sized<E, ASYNC, true, false, kSums, 0>(size, d, s);
}

// A piece's two products of dz in one launch, tiles of 256 x 256, or 128 x 128 of fp32: first dX's, whose k is the piece, then dW's, whose k is the items and
// which fill the chip to the end of the launch
template <typename E, bool ASYNC, typename S>
__global__ __launch_bounds__(S::kThreads, S::kWavesToSimd) void psattn_head_grads(Product x, Product w, int x_tiles_m, int x_tiles_n, int w_tiles_m, int w_tiles_n) {
    __shared__ __attribute__((aligned(1024))) char lds[kLds<S>];
    const int n = x_tiles_m * x_tiles_n, first = n * x.n_split, b = blockIdx.x;
    if (b < first) product_tile<E, ASYNC, true, false, kSums, 0, S>(lds, x, x_tiles_m, x_tiles_n, b % n, b / n);
    else product_tile<E, ASYNC, false, false, kPlain, 0, S>(lds, w, w_tiles_m, w_tiles_n, b - first, 0);
}

template <typename E, bool ASYNC>
int launch_grads(const Product& x, const Product& w, hipStream_t s) {
    using S = std::conditional_t<ASYNC, Shape<256, 256, 2, 4, 3>, Shape<128, 128, 2, 2, 2>>;
    auto tiles = [](int64_t n) { return (n + S::BM - 1) / S::BM; };
    const int64_t xm = tiles(x.M), xn = tiles(x.N), wm = tiles(w.M), wn = tiles(w.N), n = xm * xn * x.n_split + wm * wn;
    if (n >= (int64_t{1} << 31) / S::kThreads) return PSATTN_EUNSUPPORTED;
    psattn_head_grads<E, ASYNC, S><<<static_cast<uint32_t>(n), S::kThreads, 0, s>>>(x, w, static_cast<int>(xm), static_cast<int>(xn), static_cast<int>(wm), static_cast<int>(wn));
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

}  // namespace gemm
}  // namespace psattn
