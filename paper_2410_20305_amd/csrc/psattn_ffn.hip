// Gated feed-forward block, forward and backward: Y = (act(X Wg^T) o (X Wu^T)) Wd^T.
//
// The paper's sequences share a prompt, and the block acts on single tokens, so sharing saves the same part of it as of the
// projections.  Forward: gate and up projection, activation and product in one kernel (they share X, and G, U, H leave once),
// then the down projection.  Backward: dH = dY Wd with dG, dU in its epilogue; dX = dG Wg + dU Wu as one product over both
// weights' rows; dWg, dWu in one launch; dWd.  All sums over k are fp32; G, U, H, dG and dU are held in the element type like any
// activation, H being rounded once, from the fp32 sums.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>

#include "psattn.h"
#include "psattn_ffn.h"

namespace {

using namespace psattn::gemm;

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
size_t elem_bytes(int32_t dt) { return dt == PSATTN_BF16 ? 2 : 4; }

bool bad_shape(int32_t dt, int32_t act, int32_t n_tokens, int32_t hidden, int32_t inner) {
    return (dt != PSATTN_F32 && dt != PSATTN_BF16) || (act != PSATTN_ACT_SILU && act != PSATTN_ACT_GELU) || n_tokens < 0 || hidden <= 0 || inner <= 0;
}

bool at16(std::initializer_list<const void*> p) {
    uintptr_t a = 0;
    for (const void* x : p) a |= reinterpret_cast<uintptr_t>(x);
    return a % 16 == 0;
}

// Every row of P, Q and out a whole number of 16-byte groups on 16-byte boundaries
bool whole_rows(bool pkc, const Product& d) {
    return at16({d.p[0], d.p[1], d.q[0], d.q[1], d.out[0], d.out[1], d.G, d.U, d.H}) && d.ldp % 8 == 0 && d.ldq % 8 == 0 && d.ldo % 8 == 0 && d.N % 8 == 0 &&
           (pkc || d.M % 8 == 0);
}

struct Plan {
    TileSize size;
    int32_t split;
};

constexpr int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

Plan plan(int32_t dt, Pass pass, bool pkc, int64_t M, int64_t N, int64_t K, int n_seg, int n_prod) {
    static constexpr int bm[] = {32, 64, 128, 256}, bn[] = {128, 128, 128, 256}, per_cu[] = {4, 3, 2, 1};
    auto tiles = [&](TileSize t) { return cdiv(M, bm[t]) * cdiv(N * (pass == kGate ? 2 : 1), bn[t]) * n_prod; };
    Plan p{};
    p.size = pkc && M <= 32 ? k32 : pkc && M <= 64 ? k64 : tiles(k256) >= 200 ? k256 : k128;
    const int64_t steps = K / (dt == PSATTN_BF16 ? 64 : 32) * n_seg, n = tiles(p.size), want = 256 * per_cu[p.size];
    p.split = static_cast<int32_t>(std::max<int64_t>(1, std::min(want / n, steps / 4)));
    return p;
}

int64_t ld_part(int64_t N) { return (N + 7) / 8 * 8; }

size_t part_bytes(int32_t dt, Pass pass, bool pkc, int64_t M, int64_t N, int64_t K, int n_seg, int n_prod) {
    if (M == 0 || K == 0) return 0;  // no tokens: no products
    const Plan p = plan(dt, pass, pkc, M, N, K, n_seg, n_prod);
    return p.split > 1 ? sizeof(float) * p.split * (pass == kGate ? 2 : n_prod) * M * ld_part(N) : 0;
}

// joins the parts of a product: the epilogue of psattn_ffn_tiles on sums from memory.  grid (columns, rows, products)
template <typename E, Pass PASS, int ACT>
__global__ __launch_bounds__(256) void psattn_ffn_join(Product d) {
    const int n = blockIdx.x * 256 + threadIdx.x, z = blockIdx.z;
    if (n >= d.N) return;
    const int n_out = PASS == kGate ? 2 : d.n_prod;
    for (int m = blockIdx.y; m < d.M; m += gridDim.y) {
        const float* p = d.parts + static_cast<int64_t>(m) * d.ld_part + n;
        const int64_t one = static_cast<int64_t>(d.M) * d.ld_part;
        float x = 0.f, up = 0.f;
        for (int i = 0; i < d.n_split; ++i) {
            x += p[(static_cast<int64_t>(i) * n_out + z) * one];
            if constexpr (PASS == kGate) up += p[(static_cast<int64_t>(i) * n_out + 1) * one];
        }
        const int64_t at = m * d.ldo + n;
        if constexpr (PASS == kGate) {
            if (d.G) store1(static_cast<E*>(d.G) + at, x);
            if (d.U) store1(static_cast<E*>(d.U) + at, up);
            store1(static_cast<E*>(d.H) + at, act<ACT>(x) * up);
        } else if constexpr (PASS == kDact) {
            float a, da;
            act_grad<ACT>(to_f32(static_cast<const E*>(d.G)[at]), a, da);
            store1(static_cast<E*>(d.out[0]) + at, x * to_f32(static_cast<const E*>(d.U)[at]) * da);
            store1(static_cast<E*>(d.out[1]) + at, x * a);
        } else {
            store1(static_cast<E*>(d.out[z]) + at, x);
        }
    }
}

template <typename E>
void join(Pass pass, int act, const Product& d, hipStream_t s) {
    const dim3 grid(static_cast<uint32_t>(cdiv(d.N, 256)), std::min(d.M, 4096), pass == kPlain ? d.n_prod : 1);
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, s>>>(d); };
    if (pass == kPlain) go(psattn_ffn_join<E, kPlain, 0>);
    else if (pass == kGate) act == PSATTN_ACT_SILU ? go(psattn_ffn_join<E, kGate, 0>) : go(psattn_ffn_join<E, kGate, 1>);
    else act == PSATTN_ACT_SILU ? go(psattn_ffn_join<E, kDact, 0>) : go(psattn_ffn_join<E, kDact, 1>);
}

// `parts`: room of part_bytes()
int product(int32_t dt, Pass pass, int act, bool pkc, bool qkc, Product d, void* parts, hipStream_t s) {
    if (std::max(d.ldp, d.ldq) * elem_bytes(dt) * 256 >= (int64_t{1} << 31)) return PSATTN_EUNSUPPORTED;  // a tile's copies have 32-bit offsets
    const Plan p = plan(dt, pass, pkc, d.M, d.N, d.K, d.n_seg, d.n_prod);
    d.n_split = p.split;
    d.parts = static_cast<float*>(parts);
    d.ld_part = ld_part(d.N);
    const int rc = dt != PSATTN_BF16 ? product_f32(pass, act, pkc, qkc, p.size, d, s) : whole_rows(pkc, d) ? product_bf16(pass, act, pkc, qkc, p.size, d, s)
                                                                                                  : product_bf16_any(pass, act, pkc, qkc, p.size, d, s);
    if (rc != PSATTN_OK || d.n_split == 1) return rc;
    if (dt == PSATTN_BF16) join<uint16_t>(pass, act, d, s);
    else join<float>(pass, act, d, s);
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

// zeros without a memset, which a captured graph would not replay faithfully
__global__ void psattn_ffn_zero(uint16_t* p, size_t n) {
    for (size_t i = blockIdx.x * static_cast<size_t>(blockDim.x) + threadIdx.x; i < n; i += static_cast<size_t>(gridDim.x) * blockDim.x) p[i] = 0;
}

}  // namespace

extern "C" {

size_t psattn_ffn_bwd_workspace_bytes(int32_t dt, int32_t n_tokens, int32_t hidden, int32_t inner) {
    if (bad_shape(dt, PSATTN_ACT_SILU, n_tokens, hidden, inner)) return 0;
    const size_t parts = std::max({part_bytes(dt, kDact, true, n_tokens, inner, hidden, 1, 1), part_bytes(dt, kPlain, true, n_tokens, hidden, inner, 2, 1),
                                   part_bytes(dt, kPlain, false, inner, hidden, n_tokens, 1, 2), part_bytes(dt, kPlain, false, hidden, inner, n_tokens, 1, 1)});
    return 2 * align_up(static_cast<size_t>(n_tokens) * inner * elem_bytes(dt), 256) + align_up(parts, 256) + 256;
}

size_t psattn_ffn_fwd_workspace_bytes(int32_t dt, int32_t n_tokens, int32_t hidden, int32_t inner) {
    if (bad_shape(dt, PSATTN_ACT_SILU, n_tokens, hidden, inner)) return 0;
    const size_t parts = std::max(part_bytes(dt, kGate, true, n_tokens, inner, hidden, 1, 1), part_bytes(dt, kPlain, true, n_tokens, hidden, inner, 1, 1));
    return align_up(parts, 256) + 256;
}

int psattn_ffn_fwd(int32_t dt, int32_t act, int32_t n_tokens, int32_t hidden, int32_t inner, const void* X, const void* Wg, const void* Wu,
                   const void* Wd, void* G, void* U, void* H, void* Y, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (bad_shape(dt, act, n_tokens, hidden, inner)) return PSATTN_EINVAL;
    if (n_tokens == 0) return PSATTN_OK;
    if (!X || !Wg || !Wu || !Wd || !H || !Y || (!G) != (!U)) return PSATTN_EINVAL;
    if (!workspace || workspace_bytes < psattn_ffn_fwd_workspace_bytes(dt, n_tokens, hidden, inner)) return PSATTN_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    char* const parts = reinterpret_cast<char*>(align_up(reinterpret_cast<uintptr_t>(workspace), 256));
    Product gate{};
    gate.p[0] = X; gate.q[0] = Wg; gate.q[1] = Wu; gate.G = G; gate.U = U; gate.H = H;
    gate.ldp = gate.ldq = hidden; gate.ldo = inner;
    gate.M = n_tokens; gate.N = inner; gate.K = hidden; gate.n_seg = gate.n_prod = 1;
    int rc = product(dt, kGate, act, true, true, gate, parts, s);
    if (rc != PSATTN_OK) return rc;
    Product down{};
    down.p[0] = H; down.q[0] = Wd; down.out[0] = Y;
    down.ldp = down.ldq = inner; down.ldo = hidden;
    down.M = n_tokens; down.N = hidden; down.K = inner; down.n_seg = down.n_prod = 1;
    return product(dt, kPlain, act, true, true, down, parts, s);
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
    char* const parts = dU + align_up(static_cast<size_t>(n_tokens) * inner * elem_bytes(dt), 256);
    int rc;
    Product a{};  // dH = dY Wd, dG and dU
    a.p[0] = dY; a.q[0] = Wd; a.G = const_cast<void*>(G); a.U = const_cast<void*>(U); a.out[0] = dG; a.out[1] = dU;
    a.ldp = hidden; a.ldq = a.ldo = inner;
    a.M = n_tokens; a.N = inner; a.K = hidden; a.n_seg = a.n_prod = 1;
    if ((rc = product(dt, kDact, act, true, false, a, parts, s)) != PSATTN_OK) return rc;
    Product x{};  // dX = dG Wg + dU Wu
    x.p[0] = dG; x.p[1] = dU; x.q[0] = Wg; x.q[1] = Wu; x.out[0] = dX;
    x.ldp = inner; x.ldq = x.ldo = hidden;
    x.M = n_tokens; x.N = hidden; x.K = inner; x.n_seg = 2; x.n_prod = 1;
    if ((rc = product(dt, kPlain, act, true, false, x, parts, s)) != PSATTN_OK) return rc;
    Product gu{};  // dWg = dG^T X, dWu = dU^T X
    gu.p[0] = dG; gu.p[1] = dU; gu.q[0] = X; gu.out[0] = dWg; gu.out[1] = dWu;
    gu.ldp = inner; gu.ldq = gu.ldo = hidden;
    gu.M = inner; gu.N = hidden; gu.K = n_tokens; gu.n_seg = 1; gu.n_prod = 2;
    if ((rc = product(dt, kPlain, act, false, false, gu, parts, s)) != PSATTN_OK) return rc;
    Product wd{};  // dWd = dY^T H
    wd.p[0] = dY; wd.q[0] = H; wd.out[0] = dWd;
    wd.ldp = hidden; wd.ldq = wd.ldo = inner;
    wd.M = hidden; wd.N = inner; wd.K = n_tokens; wd.n_seg = wd.n_prod = 1;
    return product(dt, kPlain, act, false, false, wd, parts, s);
}

}  // extern "C"
