// Gated feed-forward block, forward and backward: Y = (act(X Wg^T) o (X Wu^T)) Wd^T.
//
// The paper's sequences share a prompt, and the block acts on single tokens, so sharing saves the same part of it as of the
// projections.  Forward: gate and up projection, activation and product in one kernel (they share X, and G, U, H leave once),
// then the down projection.  Backward: dH = dY Wd with dG, dU in its epilogue; dX = dG Wg + dU Wu as one product over both
// weights' rows; dWg, dWu in one launch; dWd.  All sums over k are fp32.  H, dG and dU are operands of the
// matrix cores and are held in the element type, each rounded once, from fp32.  G and U are kept in fp32: rounded to bf16 they would
// put two more roundings into dG and dU, and gradients of weights off by 3.1e-3 (relative L2 against 64 bits) instead of 2.3e-3 (their
// own rounding alone is 1.7e-3); that costs 3 % of a large step (16 384 tokens 13.91 -> 14.33 ms in turn: gate and up 3 023 -> 3 313 us, dG and dU 1 926 -> 2 031).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "psattn.h"
#include "psattn_ffn.h"
#include "psattn_rows.h"

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

// Every row of P and Q a whole number of 16-byte groups on 16-byte boundaries; what is stored in the element type likewise
bool whole_operands(bool pkc, bool qkc, const Product& d) {
    return at16({d.p[0], d.p[1], d.q[0], d.q[1]}) && d.ldp % 8 == 0 && d.ldq % 8 == 0 && (pkc || d.m_load % 8 == 0) && (qkc || d.n_load % 8 == 0);
}
bool whole_results(const Product& d) { return at16({d.out[0], d.out[1], d.H}) && d.ldo % 8 == 0 && d.N % 8 == 0; }

struct Plan {
    TileSize size;
    int32_t split;
};

constexpr int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// How a product's operands and results are moved: kWhole in 16-byte groups on boundaries, kOdd not, kFloat fp32
enum Move { kWhole, kOdd, kFloat };

// What a product takes, in us, from the rounds of workgroups that its tiles make: which tile size, and k in how many parts.  A step is 128
// bytes of k.  Measured, hidden 4 096, inner 14 336: 256 x 256, one workgroup to a CU, 1.6 us a step (1.25 where few CUs have one);
// 128 x 128, two to a CU, 1.05 a step, 0.65 by itself; through registers half as much again; fp32 at 158 TFLOP/s, of which large products reach
// 139.  A round's start and end take 3 us, or 14 (gate) and 30 (dG, dU) with 256 x 256, whose workgroups have nothing beside them to cover it, 3 and 12 with
// 128 x 128.  The two sizes, in turn: 8 192 tokens 7.0 and 8.5 ms, 1 024 tokens 1.72 and 1.49, 256 tokens 1.16 and 0.72 (unsplit).
// Parts have no end but their sums' way to memory, and are joined by another launch; sums that outgrow the 256 MB cache go to HBM and back
// (dWd of 16 384 tokens, 3.5 rounds of 256 x 256: 1 602 us, in two parts 1 637; dG and dU of 4 096 tokens 556 and 669).
//   Away from those widths the model tells the two sizes apart better than it tells their times: what a plain product stores is not in it (221
// tokens, 4 096 / 14 336: dWg and dWu 55 for 124 measured, gate and up 70 for 101).  By the rule / 128 x 128 alone / 256 x 256 alone, forward
// and backward in us: 221 tokens, 4 096 / 14 336 465 / 478 / 476; 1 000, 8 192 / 28 672 3 970 / 4 660 / 3 970; 1 037, 1 024 / 2 736 142 / 142 /
// 196; 8 192, 512 / 1 376 217 / 219 / 268; 4 096, 1 024 / 4 096 417 / 399 / 449; 16 384, 1 024 / 4 096 1 465 / 1 557 / 1 425; widths 1 001 / 2 731,
// 1 037 tokens 182 / 183 / 242.  fp32: 168, 512 / 1 376 125 / 125 / 313; 300, 4 096 / 14 336 3 195 / 3 200 / 3 840; 2 048, 2 048 / 8 192 5 065 /
// 5 165 / 4 600.
double cost(Move move, Pass pass, TileSize size, int64_t tiles, int64_t steps, int64_t split, double out_bytes) {
    const bool big = size == k256, parts = split > 1;
    const double per_wg = static_cast<double>(cdiv(steps, split)), odd = move == kOdd ? 1.5 : 1;
    const double full = (move == kFloat ? (big ? 6.8 : 3.4) : (big ? 1.6 : 1.05) * odd) * per_wg, few = (move == kFloat ? (big ? 6.8 : 1.7) : (big ? 1.25 : 0.65) * odd) * per_wg;
    const double end = parts || pass == kPlain ? 3 : pass == kGate ? (big ? 14 : 3) : (big ? 30 : 12);
    const int64_t wgs = tiles * split, slots = big ? 256 : 512, rest = wgs % slots;
    const bool little = rest > 0 && (big ? wgs <= 128 : rest <= 256);
    const double bytes = static_cast<double>(split) * out_bytes, ways = bytes > 2e8 ? 2 : 1.3;
    return static_cast<double>(wgs / slots) * (full + end) + (rest == 0 ? 0 : (little ? few : full) + end) + (parts ? 4 + bytes * ways / 4.5e6 : 0);
}

Plan plan(Move move, Pass pass, bool pkc, int64_t M, int64_t N, int64_t K, int n_seg, int n_prod) {
    static constexpr int bm[] = {32, 64, 128, 256}, bn[] = {128, 128, 128, 256};
    auto tiles = [&](TileSize t) { return cdiv(M, bm[t]) * cdiv(N * (pass == kGate ? 2 : 1), bn[t]) * n_prod; };
    const int64_t steps = K / (move == kFloat ? 32 : 64) * n_seg;
    Plan best{k128, 1};
    if (pkc && M <= 64) {
        // few tokens: the weights have to be read, and three or four workgroups to a CU keep enough of them in flight (one token, hidden 4 096,
        // inner 14 336: 5.5 TB/s)
        best.size = M <= 32 ? k32 : k64;
        best.split = static_cast<int32_t>(std::max<int64_t>(1, std::min((M <= 32 ? 1024 : 768) / tiles(best.size), steps / 4)));
        return best;
    }
    const double out = sizeof(float) * static_cast<double>(M) * N * (pass == kGate ? 2 : n_prod);
    double least = 0;
    for (const TileSize t : {k128, k256})
        for (const int64_t split : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 24, 32, 48, 64}) {
            if (split > 1 && steps / split < 4) break;
            const double us = cost(move, pass, t, tiles(t), steps, split, out);
            if ((t == k128 && split == 1) || us < least) {
                least = us;
                best = {t, static_cast<int32_t>(split)};
            }
        }
    return best;
}

int64_t ld_part(int64_t N) { return (N + 7) / 8 * 8; }

// bytes of one of a product's parts
size_t one_part(Pass pass, int64_t M, int64_t N, int n_prod) { return sizeof(float) * (pass == kGate ? 2 : n_prod) * static_cast<size_t>(M) * static_cast<size_t>(ld_part(N)); }

// room for a product's parts; `any`: whichever way its operands turn out to move
size_t part_bytes(int32_t dt, bool any, Pass pass, bool pkc, int64_t M, int64_t N, int64_t K, int n_seg, int n_prod) {
    if (M == 0 || K == 0) return 0;  // no tokens: no products
    auto room = [&](Move move) {
        const Plan p = plan(move, pass, pkc, M, N, K, n_seg, n_prod);
        return p.split > 1 ? p.split * one_part(pass, M, N, n_prod) : size_t{0};
    };
    if (dt != PSATTN_BF16) return room(kFloat);
    return any ? std::max(room(kWhole), room(kOdd)) : room(kWhole);
}

// joins the parts of a product: the epilogue of psattn_ffn_tiles on sums from memory, V columns to a lane (4 where rows allow it: dG and dU of
// 500 x 14 336 44 -> 20 us).  grid (columns, rows, products)
template <int V, typename E>
__device__ __forceinline__ void put(E* p, const float (&x)[V]) {
    if constexpr (V == 1) store1(p, x[0]);
    else if constexpr (sizeof(E) == 2) *reinterpret_cast<uint2*>(p) = make_uint2(psattn::mma::pack2(x[0], x[1]), psattn::mma::pack2(x[2], x[3]));
    else *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
template <int V, typename E>
__device__ __forceinline__ void get(const E* p, float (&x)[V]) {
    if constexpr (V == 1) {
        x[0] = to_f32(*p);
    } else if constexpr (sizeof(E) == 2) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        x[0] = __uint_as_float(u.x << 16); x[1] = __uint_as_float(u.x & 0xffff0000u);
        x[2] = __uint_as_float(u.y << 16); x[3] = __uint_as_float(u.y & 0xffff0000u);
    } else {
        const float4 u = *reinterpret_cast<const float4*>(p);
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
    }
}

template <typename E, Pass PASS, int ACT, int V>
__global__ __launch_bounds__(256) void psattn_ffn_join(Product d) {
    const int n = (blockIdx.x * 256 + threadIdx.x) * V, z = blockIdx.z;
    if (n >= d.N) return;
    constexpr int kOuts = PASS == kGate ? 2 : 1, kAtOnce = 4;
    const int n_out = PASS == kGate ? 2 : d.n_prod;
    for (int m = blockIdx.y; m < d.M; m += gridDim.y) {
        const float* p = d.parts + static_cast<int64_t>(m) * d.ld_part + n;
        const int64_t one = static_cast<int64_t>(d.M) * d.ld_part;
        float x[kOuts][V] = {};
        auto add = [&](int from, auto COUNT) {  // loads together, sums in order
            constexpr int count = decltype(COUNT)::value;
            float a[count][kOuts][V];
#pragma unroll
            for (int u = 0; u < count; ++u)
#pragma unroll
                for (int o = 0; o < kOuts; ++o) get<V>(p + (static_cast<int64_t>(from + u) * n_out + (PASS == kGate ? o : z)) * one, a[u][o]);
#pragma unroll
            for (int u = 0; u < count; ++u)
#pragma unroll
                for (int o = 0; o < kOuts; ++o)
#pragma unroll
                    for (int j = 0; j < V; ++j) x[o][j] += a[u][o][j];
        };
        int i = 0;
        for (; i + kAtOnce <= d.n_split; i += kAtOnce) add(i, std::integral_constant<int, kAtOnce>{});
        for (; i < d.n_split; ++i) add(i, std::integral_constant<int, 1>{});
        const int64_t at = m * d.ldo + n;
        if constexpr (PASS == kGate) {
            if (d.G) put<V>(d.G + at, x[0]);
            if (d.U) put<V>(d.U + at, x[1]);
            float h[V];
#pragma unroll
            for (int j = 0; j < V; ++j) h[j] = act<E, ACT>(x[0][j]) * x[1][j];
            put<V>(static_cast<E*>(d.H) + at, h);
        } else if constexpr (PASS == kDact) {
            float gate[V], up[V], dg[V], du[V];
            const int64_t kept = m * d.ld_kept + n;
            get<V>(d.G + kept, gate);
            get<V>(d.U + kept, up);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float a, da;
                act_grad<E, ACT>(gate[j], a, da);
                dg[j] = x[0][j] * up[j] * da;
                du[j] = x[0][j] * a;
            }
            put<V>(static_cast<E*>(d.out[0]) + at, dg);
            put<V>(static_cast<E*>(d.out[1]) + at, du);
        } else {
            put<V>(static_cast<E*>(d.out[z]) + at, x[0]);
        }
    }
}

template <typename E, int V>
void join(Pass pass, int act, const Product& d, hipStream_t s) {
    const dim3 grid(static_cast<uint32_t>(cdiv(d.N, 256 * V)), std::min(d.M, 4096), pass == kPlain ? d.n_prod : 1);
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, s>>>(d); };
    if (pass == kPlain) go(psattn_ffn_join<E, kPlain, 0, V>);
    else if (pass == kGate) act == PSATTN_ACT_SILU ? go(psattn_ffn_join<E, kGate, 0, V>) : go(psattn_ffn_join<E, kGate, 1, V>);
    else act == PSATTN_ACT_SILU ? go(psattn_ffn_join<E, kDact, 0, V>) : go(psattn_ffn_join<E, kDact, 1, V>);
}

// `parts`, up to `end`: room of part_bytes(), or, where operands move another way than that was asked for, fewer parts
int product(int32_t dt, Pass pass, int act, bool pkc, bool qkc, Product d, char* parts, const char* end, hipStream_t s) {
    d.odd = !whole_results(d);
    const Move move = dt != PSATTN_BF16 ? kFloat : whole_operands(pkc, qkc, d) ? kWhole : kOdd;
    const Plan p = plan(move, pass, pkc, d.M, d.N, d.K, d.n_seg, d.n_prod);
    const int64_t fit = (end - parts) / static_cast<int64_t>(one_part(pass, d.M, d.N, d.n_prod));
    d.n_split = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(p.split, fit)));
    d.parts = reinterpret_cast<float*>(parts);
    d.ld_part = ld_part(d.N);
    const int rc = (move == kFloat ? product_f32 : move == kWhole ? product_bf16 : product_bf16_any)(pass, act, pkc, qkc, p.size, d, s);
    if (rc != PSATTN_OK || d.n_split == 1) return rc;
    const bool four = at16({d.out[0], d.out[1], d.G, d.U, d.H}) && d.ldo % 4 == 0 && d.N % 4 == 0 && (pass != kDact || d.ld_kept % 4 == 0);
    if (dt == PSATTN_BF16) four ? join<uint16_t, 4>(pass, act, d, s) : join<uint16_t, 1>(pass, act, d, s);
    else four ? join<float, 4>(pass, act, d, s) : join<float, 1>(pass, act, d, s);
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

// ---- bf16 rows that are not whole 16-byte groups on boundaries, made so in the workspace.  The asynchronous copies need such rows; the way
// through registers does not, but takes 1.5 - 1.7 times as long.  What the rows' copies cost is made good from some 300 tokens on.  Through
// registers / made whole, forward and backward in us: hidden 4 095, inner 14 335, 300 tokens 1 079 / 1 074, 700 1 638 / 1 396, 1 200 2 659 /
// 1 921; hidden 1 001, inner 2 731, 150 tokens 116 / 114, 300 137 / 129, 1 037 238 / 187; hidden 2 047, inner 6 001, 3 001 tokens 1 500 / 1 030
// (890 on rows that are whole).  Tensors of a width that is no multiple of 8 always have their room.  Others need it only where they start off a
// boundary, which sizes do not tell: they are copied where the workspace has been made for that, and go through registers elsewhere (8 192
// tokens, hidden 4 096, inner 14 336, forward 2 374; all tensors off a boundary 2 524 with copies, 3 881 without; X alone 2 396 and 3 187).
constexpr int32_t kPadTokens = 320;

struct Pad {
    const uint16_t* src;
    uint16_t* dst;
    int32_t rows, width;
};
struct Pads {
    Pad p[6];
};
constexpr int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }

// dst[row][0 .. up8(width)) = src[row][0 .. width), zeros behind
__global__ __launch_bounds__(256) void psattn_ffn_pad(Pads pads) {
    const Pad p = pads.p[blockIdx.y];
    const int groups = (p.width + 7) / 8;
    const int64_t n = static_cast<int64_t>(p.rows) * groups;
    for (int64_t i = blockIdx.x * int64_t{256} + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t row = i / groups;
        const int c = static_cast<int>(i - row * groups) * 8;
        const auto at = psattn::rows::place<false, uint16_t>(c, p.width);
        const auto u = psattn::rows::settled<false>(psattn::rows::raw<false>(p.src + row * p.width, at, p.width), at.down);
        *reinterpret_cast<psattn::rows::u32x4*>(p.dst + (row * groups + i - row * groups) * 8) = u;
    }
}

bool may_pad(int32_t dt, int64_t n_tokens) { return dt == PSATTN_BF16 && n_tokens >= kPadTokens; }

// Makes rows whole: takes their room from a workspace, and copies them when told to
struct Wholes {
    char* p;
    bool may, roomy;  // whether rows are copied at all; those of whole widths that start off a boundary too
    Pad list[6];
    int n = 0;
    Wholes(void* base, bool may, bool roomy) : p(reinterpret_cast<char*>(align_up(reinterpret_cast<uintptr_t>(base), 256))), may(may), roomy(roomy) {}
    // the tensor itself where its rows are whole, or may stay as they are; else the place of its copy
    const void* add(const void* x, int32_t rows, int32_t width) {
        if (!may || (width % 8 == 0 && (at16({x}) || !roomy))) return x;
        uint16_t* const to = reinterpret_cast<uint16_t*>(p);
        p += bytes(rows, width);
        list[n++] = {static_cast<const uint16_t*>(x), to, rows, width};
        return to;
    }
    static size_t bytes(int64_t rows, int64_t width) { return align_up(static_cast<size_t>(rows) * static_cast<size_t>(up8(width)) * 2, 256); }
    int copy(hipStream_t s) {
        if (n == 0) return PSATTN_OK;
        Pads pads{};
        std::copy(list, list + n, pads.p);
        psattn_ffn_pad<<<dim3(2048, n), 256, 0, s>>>(pads);
        n = 0;
        return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
    }
};
// room for their copies: `acts` activations of width hidden (X; in the backward dY too), H and the weights
size_t whole_bytes(int32_t dt, int64_t n_tokens, int64_t hidden, int64_t inner, bool unaligned, int acts) {
    if (!may_pad(dt, n_tokens)) return 0;
    size_t n = 0;
    if (unaligned || hidden % 8) n += acts * Wholes::bytes(n_tokens, hidden) + 2 * Wholes::bytes(inner, hidden);
    if (unaligned || inner % 8) n += Wholes::bytes(hidden, inner) + Wholes::bytes(n_tokens, inner);
    return n;
}

size_t fwd_bytes(int32_t dt, int32_t n_tokens, int32_t hidden, int32_t inner, bool unaligned) {
    if (bad_shape(dt, PSATTN_ACT_SILU, n_tokens, hidden, inner)) return 0;
    const bool any = unaligned || hidden % 8 || inner % 8;
    const size_t parts = std::max(part_bytes(dt, any, kGate, true, n_tokens, inner, hidden, 1, 1), part_bytes(dt, any, kPlain, true, n_tokens, hidden, inner, 1, 1));
    return align_up(parts, 256) + whole_bytes(dt, n_tokens, hidden, inner, unaligned, 1) + 256;
}
size_t bwd_bytes(int32_t dt, int32_t n_tokens, int32_t hidden, int32_t inner, bool unaligned) {
    if (bad_shape(dt, PSATTN_ACT_SILU, n_tokens, hidden, inner)) return 0;
    const bool any = unaligned || hidden % 8 || inner % 8;
    const size_t parts = std::max({part_bytes(dt, any, kDact, true, n_tokens, inner, hidden, 1, 1), part_bytes(dt, any, kPlain, true, n_tokens, hidden, inner, 2, 1),
                                   part_bytes(dt, any, kPlain, false, inner, hidden, n_tokens, 1, 2), part_bytes(dt, any, kPlain, false, hidden, inner, n_tokens, 1, 1)});
    return 2 * align_up(static_cast<size_t>(n_tokens) * static_cast<size_t>(up8(inner)) * elem_bytes(dt), 256) + align_up(parts, 256) +
           whole_bytes(dt, n_tokens, hidden, inner, unaligned, 2) + 256;
}

// a tile's copies have 32-bit offsets, and grids stay below 2^31 threads
bool too_large(int32_t dt, int64_t n_tokens, int64_t hidden, int64_t inner) {
    if (std::max(hidden, inner) * static_cast<int64_t>(elem_bytes(dt)) * 256 >= (int64_t{1} << 31)) return true;
    const int64_t t = cdiv(n_tokens, 128), h = cdiv(hidden, 128), i = cdiv(inner, 128);
    return std::max({t * (2 * i + 1), t * h, 2 * i * h}) >= (int64_t{1} << 23);
}

// zeros without a memset, which a captured graph would not replay faithfully
__global__ void psattn_ffn_zero(uint16_t* p, size_t n) {
    for (size_t i = blockIdx.x * static_cast<size_t>(blockDim.x) + threadIdx.x; i < n; i += static_cast<size_t>(gridDim.x) * blockDim.x) p[i] = 0;
}

}  // namespace

extern "C" {

size_t psattn_ffn_fwd_workspace_bytes(int32_t dt, int32_t n_tokens, int32_t hidden, int32_t inner) { return fwd_bytes(dt, n_tokens, hidden, inner, false); }

size_t psattn_ffn_fwd_unaligned_workspace_bytes(int32_t dt, int32_t n_tokens, int32_t hidden, int32_t inner) { return fwd_bytes(dt, n_tokens, hidden, inner, true); }

size_t psattn_ffn_bwd_workspace_bytes(int32_t dt, int32_t n_tokens, int32_t hidden, int32_t inner) { return bwd_bytes(dt, n_tokens, hidden, inner, false); }

size_t psattn_ffn_bwd_unaligned_workspace_bytes(int32_t dt, int32_t n_tokens, int32_t hidden, int32_t inner) { return bwd_bytes(dt, n_tokens, hidden, inner, true); }

int psattn_ffn_fwd(int32_t dt, int32_t act, int32_t n_tokens, int32_t hidden, int32_t inner, const void* X, const void* Wg, const void* Wu,
                   const void* Wd, float* G, float* U, void* H, void* Y, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (bad_shape(dt, act, n_tokens, hidden, inner)) return PSATTN_EINVAL;
    if (n_tokens == 0) return PSATTN_OK;
    if (!X || !Wg || !Wu || !Wd || !H || !Y || (!G) != (!U)) return PSATTN_EINVAL;
    if (!workspace || workspace_bytes < psattn_ffn_fwd_workspace_bytes(dt, n_tokens, hidden, inner)) return PSATTN_EINVAL;
    if (too_large(dt, n_tokens, hidden, inner)) return PSATTN_EUNSUPPORTED;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const bool may = may_pad(dt, n_tokens);
    const int64_t hp = may ? up8(hidden) : hidden, ip = may ? up8(inner) : inner;
    Wholes room(workspace, may, workspace_bytes >= fwd_bytes(dt, n_tokens, hidden, inner, true));
    X = room.add(X, n_tokens, hidden), Wg = room.add(Wg, inner, hidden), Wu = room.add(Wu, inner, hidden), Wd = room.add(Wd, hidden, inner);
    int rc;
    if ((rc = room.copy(s)) != PSATTN_OK) return rc;
    const void* const Hp = room.add(H, n_tokens, inner);  // copied when it is there
    char* const parts = room.p;
    const char* const end = static_cast<const char*>(workspace) + workspace_bytes;
    Product gate{};
    gate.p[0] = X; gate.q[0] = Wg; gate.q[1] = Wu; gate.G = G; gate.U = U; gate.H = H;
    gate.ldp = gate.ldq = hp; gate.ldo = inner;
    gate.M = gate.m_load = n_tokens; gate.N = gate.n_load = inner; gate.K = hidden; gate.n_seg = gate.n_prod = 1;
    if ((rc = product(dt, kGate, act, true, true, gate, parts, end, s)) != PSATTN_OK) return rc;
    if ((rc = room.copy(s)) != PSATTN_OK) return rc;
    Product down{};
    down.p[0] = Hp; down.q[0] = Wd; down.out[0] = Y;
    down.ldp = down.ldq = ip; down.ldo = hidden;
    down.M = down.m_load = n_tokens; down.N = down.n_load = hidden; down.K = inner; down.n_seg = down.n_prod = 1;
    return product(dt, kPlain, act, true, true, down, parts, end, s);
}

int psattn_ffn_bwd(int32_t dt, int32_t act, int32_t n_tokens, int32_t hidden, int32_t inner, const void* X, const void* Wg, const void* Wu,
                   const void* Wd, const float* G, const float* U, const void* H, const void* dY, void* dX, void* dWg, void* dWu, void* dWd,
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
    if (too_large(dt, n_tokens, hidden, inner)) return PSATTN_EUNSUPPORTED;
    const bool may = may_pad(dt, n_tokens);
    const int64_t hp = may ? up8(hidden) : hidden, ip = may ? up8(inner) : inner;
    Wholes room(workspace, may, workspace_bytes >= bwd_bytes(dt, n_tokens, hidden, inner, true));
    const size_t kept = align_up(static_cast<size_t>(n_tokens) * static_cast<size_t>(up8(inner)) * elem_bytes(dt), 256);
    char *const dG = room.p, *const dU = dG + kept;
    room.p = dU + kept;
    X = room.add(X, n_tokens, hidden), dY = room.add(dY, n_tokens, hidden), Wg = room.add(Wg, inner, hidden), Wu = room.add(Wu, inner, hidden);
    Wd = room.add(Wd, hidden, inner), H = room.add(H, n_tokens, inner);
    int rc;
    if ((rc = room.copy(s)) != PSATTN_OK) return rc;
    char* const parts = room.p;
    const char* const end = static_cast<const char*>(workspace) + workspace_bytes;
    Product a{};  // dH = dY Wd, dG and dU.  G and U have rows of `inner`, dG and dU rows of ip
    a.p[0] = dY; a.q[0] = Wd; a.G = const_cast<float*>(G); a.U = const_cast<float*>(U); a.out[0] = dG; a.out[1] = dU;
    a.ldp = hp; a.ldq = a.ldo = ip; a.ld_kept = inner;
    a.M = a.m_load = n_tokens; a.N = inner; a.n_load = static_cast<int32_t>(ip); a.K = hidden; a.n_seg = a.n_prod = 1;
    if ((rc = product(dt, kDact, act, true, false, a, parts, end, s)) != PSATTN_OK) return rc;
    Product x{};  // dX = dG Wg + dU Wu
    x.p[0] = dG; x.p[1] = dU; x.q[0] = Wg; x.q[1] = Wu; x.out[0] = dX;
    x.ldp = ip; x.ldq = hp; x.ldo = hidden;
    x.M = x.m_load = n_tokens; x.N = hidden; x.n_load = static_cast<int32_t>(hp); x.K = inner; x.n_seg = 2; x.n_prod = 1;
    if ((rc = product(dt, kPlain, act, true, false, x, parts, end, s)) != PSATTN_OK) return rc;
    Product gu{};  // dWg = dG^T X, dWu = dU^T X
    gu.p[0] = dG; gu.p[1] = dU; gu.q[0] = X; gu.out[0] = dWg; gu.out[1] = dWu;
    gu.ldp = ip; gu.ldq = hp; gu.ldo = hidden;
    gu.M = inner; gu.m_load = static_cast<int32_t>(ip); gu.N = hidden; gu.n_load = static_cast<int32_t>(hp); gu.K = n_tokens; gu.n_seg = 1; gu.n_prod = 2;
    if ((rc = product(dt, kPlain, act, false, false, gu, parts, end, s)) != PSATTN_OK) return rc;
    Product wd{};  // dWd = dY^T H
    wd.p[0] = dY; wd.q[0] = H; wd.out[0] = dWd;
    wd.ldp = hp; wd.ldq = ip; wd.ldo = inner;
    wd.M = hidden; wd.m_load = static_cast<int32_t>(hp); wd.N = inner; wd.n_load = static_cast<int32_t>(ip); wd.K = n_tokens; wd.n_seg = wd.n_prod = 1;
    return product(dt, kPlain, act, false, false, wd, parts, end, s);
}

}  // extern "C"
