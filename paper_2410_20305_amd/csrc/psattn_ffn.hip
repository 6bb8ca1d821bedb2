// Gated feed-forward block, forward and backward: Y = (act(X Wg^T) o (X Wu^T)) Wd^T.
//
// The paper's sequences share a prompt, and the block acts on single tokens, so sharing saves the same part of it as of the
// projections.  Forward: gate and up projection, activation and product in one kernel (they share X, and G, U, H leave once),
// then the down projection.  Backward: dH = dY Wd with dG, dU in its epilogue; dX = dG Wg + dU Wu as one product over both
// weights' rows; dWg, dWu in one launch; dWd.  All sums over k are fp32; G, U, H, dG and dU are held in the element type like any
// activation, H being rounded once, from the fp32 sums.
#include <hip/hip_runtime.h>

#include "psattn.h"
#include "psattn_ffn.h"

namespace {

using namespace psattn::gemm;

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
size_t elem_bytes(int32_t dt) { return dt == PSATTN_BF16 ? 2 : 4; }

bool bad_shape(int32_t dt, int32_t act, int32_t n_tokens, int32_t hidden, int32_t inner) {
    return (dt != PSATTN_F32 && dt != PSATTN_BF16) || (act != PSATTN_ACT_SILU && act != PSATTN_ACT_GELU) || n_tokens < 0 || hidden <= 0 || inner <= 0;
}

int product(int32_t dt, Pass pass, int act, bool pkc, bool qkc, const Product& d, hipStream_t s) {
    if (dt == PSATTN_BF16 && product_mfma_ok(pkc, qkc, d)) return product_mfma(pass, act, pkc, qkc, d, s);
    return product_any(dt, pass, act, pkc, qkc, d, s);
}

// zeros without a memset, which a captured graph would not replay faithfully
__global__ void psattn_ffn_zero(uint16_t* p, size_t n) {
    for (size_t i = blockIdx.x * static_cast<size_t>(blockDim.x) + threadIdx.x; i < n; i += static_cast<size_t>(gridDim.x) * blockDim.x) p[i] = 0;
}

}  // namespace

extern "C" {

size_t psattn_ffn_bwd_workspace_bytes(int32_t dt, int32_t n_tokens, int32_t hidden, int32_t inner) {
    if (bad_shape(dt, PSATTN_ACT_SILU, n_tokens, hidden, inner)) return 0;
    return 2 * align_up(static_cast<size_t>(n_tokens) * inner * elem_bytes(dt), 256) + 256;
}

size_t psattn_ffn_fwd_workspace_bytes(int32_t dt, int32_t n_tokens, int32_t hidden, int32_t inner) {
    if (bad_shape(dt, PSATTN_ACT_SILU, n_tokens, hidden, inner)) return 0;
    return 256;
}

int psattn_ffn_fwd(int32_t dt, int32_t act, int32_t n_tokens, int32_t hidden, int32_t inner, const void* X, const void* Wg, const void* Wu,
                   const void* Wd, void* G, void* U, void* H, void* Y, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (bad_shape(dt, act, n_tokens, hidden, inner)) return PSATTN_EINVAL;
    if (n_tokens == 0) return PSATTN_OK;
    if (!X || !Wg || !Wu || !Wd || !H || !Y || (!G) != (!U)) return PSATTN_EINVAL;
    if (!workspace || workspace_bytes < psattn_ffn_fwd_workspace_bytes(dt, n_tokens, hidden, inner)) return PSATTN_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    Product gate{};
    gate.p[0] = X; gate.q[0] = Wg; gate.q[1] = Wu; gate.G = G; gate.U = U; gate.H = H;
    gate.ldp = gate.ldq = hidden; gate.ldo = inner;
    gate.M = n_tokens; gate.N = inner; gate.K = hidden; gate.n_seg = gate.n_prod = 1;
    int rc = product(dt, kGate, act, true, true, gate, s);
    if (rc != PSATTN_OK) return rc;
    Product down{};
    down.p[0] = H; down.q[0] = Wd; down.out[0] = Y;
    down.ldp = down.ldq = inner; down.ldo = hidden;
    down.M = n_tokens; down.N = hidden; down.K = inner; down.n_seg = down.n_prod = 1;
    return product(dt, kPlain, act, true, true, down, s);
}

int psattn_ffn_bwd(int32_t dt, int32_t act, int32_t n_tokens, int32_t hidden, int32_t inner, const void* X, const void* Wg, const void* Wu,
                   const void* Wd, const void* G, const void* U, const void* H, const void* dY, void* dX, void* dWg, void* dWu, void* dWd,
                   void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (bad_shape(dt, act, n_tokens, hidden, inner)) return PSATTN_EINVAL;
    if (!dWg || !dWu || !dWd) return PSATTN_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (n_tokens == 0) {  // no tokens: sums over nothing
        const size_t n = static_cast<size_t>(hidden) * inner * elem_bytes(dt) / 2;
        for (void* d : {dWg, dWu, dWd}) psattn_ffn_zero<<<1024, 256, 0, s>>>(static_cast<uint16_t*>(d), n);
        return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
    }
    if (!X || !Wg || !Wu || !Wd || !G || !U || !H || !dY || !dX || !workspace) return PSATTN_EINVAL;
    if (workspace_bytes < psattn_ffn_bwd_workspace_bytes(dt, n_tokens, hidden, inner)) return PSATTN_EINVAL;
    char* const dG = reinterpret_cast<char*>(align_up(reinterpret_cast<uintptr_t>(workspace), 256));
    char* const dU = dG + align_up(static_cast<size_t>(n_tokens) * inner * elem_bytes(dt), 256);
    int rc;
    Product a{};  // dH = dY Wd, dG and dU
    a.p[0] = dY; a.q[0] = Wd; a.G = const_cast<void*>(G); a.U = const_cast<void*>(U); a.out[0] = dG; a.out[1] = dU;
    a.ldp = hidden; a.ldq = a.ldo = inner;
    a.M = n_tokens; a.N = inner; a.K = hidden; a.n_seg = a.n_prod = 1;
    if ((rc = product(dt, kDact, act, true, false, a, s)) != PSATTN_OK) return rc;
    Product x{};  // dX = dG Wg + dU Wu
    x.p[0] = dG; x.p[1] = dU; x.q[0] = Wg; x.q[1] = Wu; x.out[0] = dX;
    x.ldp = inner; x.ldq = x.ldo = hidden;
    x.M = n_tokens; x.N = hidden; x.K = inner; x.n_seg = 2; x.n_prod = 1;
    if ((rc = product(dt, kPlain, act, true, false, x, s)) != PSATTN_OK) return rc;
    Product gu{};  // dWg = dG^T X, dWu = dU^T X
    gu.p[0] = dG; gu.p[1] = dU; gu.q[0] = X; gu.out[0] = dWg; gu.out[1] = dWu;
    gu.ldp = inner; gu.ldq = gu.ldo = hidden;
    gu.M = inner; gu.N = hidden; gu.K = n_tokens; gu.n_seg = 1; gu.n_prod = 2;
    if ((rc = product(dt, kPlain, act, false, false, gu, s)) != PSATTN_OK) return rc;
    Product wd{};  // dWd = dY^T H
    wd.p[0] = dY; wd.q[0] = H; wd.out[0] = dWd;
    wd.ldp = hidden; wd.ldq = wd.ldo = inner;
    wd.M = hidden; wd.N = inner; wd.K = n_tokens; wd.n_seg = wd.n_prod = 1;
    return product(dt, kPlain, act, false, false, wd, s);
}

}  // extern "C"
