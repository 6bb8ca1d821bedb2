// Embedding rows by token id, scaled, and the gradient of the table.
//   X[t] = scale W[id_t],  dW[v] = scale sum of dX[t] over the tokens t with id_t = v, in the order of the tokens, in fp32
// A token whose id is not in [0, vocab) (padding) has a row of zeros and gives no gradient.
#include <hip/hip_runtime.h>

#include <cmath>

#include "psattn.h"
#include "psattn_gemm.h"

namespace {

using psattn::gemm::store1;
using psattn::gemm::to_f32;

constexpr int kThreads = 256;

template <typename E>
__global__ __launch_bounds__(kThreads) void psattn_embed_rows(int64_t n, int hidden, int vocab, float scale, const int32_t* ids, const E* W, E* X) {
    for (int64_t i = blockIdx.x * static_cast<int64_t>(kThreads) + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int id = ids[i / hidden];
        store1(X + i, id >= 0 && id < vocab ? to_f32(W[static_cast<int64_t>(id) * hidden + i % hidden]) * scale : 0.f);
    }
}

// one workgroup per row of the table and kThreads columns: looks for its tokens among all
template <typename E>
__global__ __launch_bounds__(kThreads) void psattn_embed_grad(int n_tokens, int hidden, float scale, const int32_t* ids, const E* dX, E* dW) {
    __shared__ int found[kThreads];
    const int v = blockIdx.x, col = blockIdx.y * kThreads + threadIdx.x;
    float sum = 0.f;
    for (int t0 = 0; t0 < n_tokens; t0 += kThreads) {
        const int t = t0 + threadIdx.x;
        found[threadIdx.x] = t < n_tokens && ids[t] == v;
        if (!__syncthreads_or(found[threadIdx.x])) continue;
        for (int j = 0; j < kThreads; ++j)
            if (found[j] && col < hidden) sum += to_f32(dX[static_cast<int64_t>(t0 + j) * hidden + col]);
        __syncthreads();
    }
    if (col < hidden) store1(dW + static_cast<int64_t>(v) * hidden + col, sum * scale);
}

bool bad_shape(int32_t dt, int32_t n_tokens, int32_t vocab, int32_t hidden, float scale) {
    return (dt != PSATTN_F32 && dt != PSATTN_BF16) || n_tokens < 0 || vocab <= 0 || hidden <= 0 || !std::isfinite(scale);
}

}  // namespace

extern "C" {

int psattn_embed_fwd(int32_t dt, int32_t n_tokens, int32_t vocab, int32_t hidden, float scale, const int32_t* token_ids, const void* W, void* X,
                     void* hip_stream) {
    if (bad_shape(dt, n_tokens, vocab, hidden, scale)) return PSATTN_EINVAL;
    if (n_tokens == 0) return PSATTN_OK;
    if (!token_ids || !W || !X) return PSATTN_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const int64_t n = static_cast<int64_t>(n_tokens) * hidden;
    const int grid = static_cast<int>(n / kThreads < 65536 ? n / kThreads + 1 : 65536);
    if (dt == PSATTN_BF16) psattn_embed_rows<<<grid, kThreads, 0, s>>>(n, hidden, vocab, scale, token_ids, static_cast<const uint16_t*>(W), static_cast<uint16_t*>(X));
    else psattn_embed_rows<<<grid, kThreads, 0, s>>>(n, hidden, vocab, scale, token_ids, static_cast<const float*>(W), static_cast<float*>(X));
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

size_t psattn_embed_bwd_workspace_bytes(int32_t dt, int32_t n_tokens, int32_t vocab, int32_t hidden) {
    if (bad_shape(dt, n_tokens, vocab, hidden, 1.f)) return 0;
    return 256;
}

int psattn_embed_bwd(int32_t dt, int32_t n_tokens, int32_t vocab, int32_t hidden, float scale, const int32_t* token_ids, const void* dX, void* dW,
                     void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (bad_shape(dt, n_tokens, vocab, hidden, scale) || !dW || (n_tokens > 0 && (!token_ids || !dX))) return PSATTN_EINVAL;
    const size_t need = psattn_embed_bwd_workspace_bytes(dt, n_tokens, vocab, hidden);
    if (!workspace || workspace_bytes < need) return PSATTN_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const dim3 grid(vocab, (hidden + kThreads - 1) / kThreads);
    if (dt == PSATTN_BF16) psattn_embed_grad<<<grid, kThreads, 0, s>>>(n_tokens, hidden, scale, token_ids, static_cast<const uint16_t*>(dX), static_cast<uint16_t*>(dW));
    else psattn_embed_grad<<<grid, kThreads, 0, s>>>(n_tokens, hidden, scale, token_ids, static_cast<const float*>(dX), static_cast<float*>(dW));
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

}  // extern "C"
