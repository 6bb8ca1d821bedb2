// Tiles of the feed-forward block's matrix products (gfx950).
//
// Every product has the form out[m][n] = sum_k P(m, k) Q(n, k).  An operand lies in memory either with k contiguous (rows of m or
// n: KC) or with k as its row (KS); the block's eight products need KC x KC (forward), KC x KS (gradients of activations) and
// KS x KS (gradients of weights).  Q is the MFMA's A operand and P its B operand, so that a lane's accumulator registers hold
// neighbouring n of one m: out is stored along its contiguous axis.
//
// An operand's tile in LDS holds 128 bytes of k (64 bf16, 32 fp32) by ROWS rows of m or n:
//   KC  rows of 128 bytes, one per m or n
//   KS  rows of 256 bytes, one per k, in sub-tiles of 128 bf16 or 64 fp32 columns
// 16-byte chunks are swizzled within a row (psattn_mfma_common.h); fp32 columns are read 32 at a time from two rows four
// apart, which the swizzle puts into different halves of the banks.
#pragma once
#include "psattn_mfma_common.h"

namespace psattn {
namespace gemm {

using mma::bf16x4;
using mma::bf16x8;
using mma::f32x16;
using mma::Frag8;
using mma::static_for;

// what a product's epilogue does
enum Pass {
    kPlain,  // out = acc
    kGate,   // Q is two matrices (gate, up): G, U, H = act(G) o U
    kDact,   // acc = dH: dG, dU from the kept G, U
    // of the vocabulary head, m an item (a row that predicts a token), n a token of the vocabulary
    kLse,     // acc = logits: maximum and sum of exponentials of each tile's part of a row, the logit of the row's token
    kDlogit,  // acc = logits: out = weight (1[n = token] - exp(acc - lse))
    kSums,    // parts = acc in fp32, or what is there and acc
    kTokens,  // acc = dW of bf16, m a token, k items: out = acc; of tokens that an item predicts also what the rounding leaves
};

struct Product {
    const void *p[2], *q[2];  // of the segments along k (n_seg), or of two products of one shape (n_prod, p and out only); kGate: q of gate and up
    void* out[2];             // kPlain: out[product]; kDact: dG, dU; kDlogit: dz and, of bf16 and 32 rows at most, what its rounding leaves (may be null); kTokens: dW and [items][ldo], what its rounding leaves
    float *G, *U;             // kGate: written (may be null); kDact: read; kLse: pairs [tile of n][M], logits [M], written; kDlogit: lse, weights [M]
    void* H;                  // kGate: written; kLse, kDlogit: tokens [M], int32; kTokens: an item of each token or -1, int32 [M]
    int64_t ldp, ldq, ldo;    // elements from one row in memory to the next
    int64_t ld_kept;          // kDact: of G and U
    int32_t M, N, K;          // K: of one segment
    int32_t n_seg, n_prod;
    int32_t m_load, n_load;   // M, N, or what rows in memory have of them and more (rows padded to whole 16-byte groups); kLse, kDlogit: n_load is the token of column 0
    int32_t odd;              // what is stored in the element type: rows that are not whole groups on 16-byte boundaries
    // k in n_split parts, whose sums go to `parts` in fp32 (rows of ld_part) and are joined by a kernel of their own
    int32_t n_split;
    int32_t add;              // kSums: parts hold sums already
    float* parts;             // kDlogit of bf16: [M], dz at the items' tokens, where out gets 0 then (may be null)
    int32_t* item_of;         // ... and, written too: one of the items of each token
    int64_t ld_part;
};

template <typename E>
constexpr int kChunk = 16 / static_cast<int>(sizeof(E));  // elements of a 16-byte chunk
template <typename E>
constexpr int kBK = 128 / static_cast<int>(sizeof(E));    // k of a tile

__device__ __forceinline__ float to_f32(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = static_cast<uint16_t>(mma::pack2(v, 0.f)); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

// ---- LDS layout
template <typename E, bool KC>
__device__ __forceinline__ int swizzle(int row) {
    if constexpr (KC) return mma::row_swizzle<64>(row);
    else if constexpr (sizeof(E) == 2) return mma::row_swizzle<128>(row);
    else return ((row >> 2) & 1) << 3;
}
// byte offset of chunk `c` (0 .. 8 ROWS - 1, in memory order along the contiguous axis) of a tile
template <typename E, bool KC, int ROWS>
__device__ __forceinline__ int chunk_off(int c) {
    if constexpr (KC) {
        const int row = c >> 3, ch = c & 7;
        return row * 128 + ((ch ^ swizzle<E, true>(row)) << 4);
    } else {
        constexpr int per_row = ROWS * static_cast<int>(sizeof(E)) / 16;
        const int row = c / per_row, ch = c % per_row;
        return (ch >> 4) * (kBK<E> * 256) + row * 256 + (((ch & 15) ^ swizzle<E, false>(row)) << 4);
    }
}

// ---- operands: what lane l holds for one step (16 k of bf16, 8 k of fp32) of a block of 32 rows of m or n
template <typename E>
struct Frag;
template <>
struct Frag<uint16_t> {
    bf16x8 v;
};
template <>
struct Frag<float> {
    float v[4];
};

// lane constants of the reads.  `first`: the wave's first block of 32; its blocks lie within whole sub-tiles, so that what
// distinguishes them is known at compile time
template <typename E, bool KC>
struct LaneRead {
    int a, b;
    __device__ LaneRead(int l, int first) {
        const int c32 = l & 31, g = l >> 5, i16 = l & 15;
        b = 0;
        if constexpr (KC) {
            a = c32 * 128 + ((g ^ swizzle<E, true>(c32)) << 4);
        } else if constexpr (sizeof(E) == 2) {
            // transposing reads: lane i of 16 names row i / 4, columns 4 (i % 4) .. of a block of 4 x 16 and gets its column i
            const int row = 8 * g + (i16 >> 2), col = 16 * ((l >> 4) & 1) + 4 * (i16 & 3);
            a = row * 256 + (((col >> 3) ^ swizzle<E, false>(row)) << 4) + (col & 7) * 2;
            b = (row + 4) * 256 + (((col >> 3) ^ swizzle<E, false>(row + 4)) << 4) + (col & 7) * 2;
        } else {
            // the swizzle depends on g alone: rows 8 t + 4 g + j
            a = 4 * g * 256 + (((c32 >> 2) ^ swizzle<E, false>(4 * g)) << 4) + (c32 & 3) * 4;
        }
        if constexpr (KC) {
            a += first * 32 * 128;
        } else {
            constexpr int per = 8 / static_cast<int>(sizeof(E));  // blocks of a sub-tile
            const int sub = (first / per) * (kBK<E> * 256), x = (first % per) * 32 * static_cast<int>(sizeof(E));
            a = (a ^ x) + sub;
            b = (b ^ x) + sub;
        }
    }
};

// step T of the wave's block BLK
template <typename E, bool KC, int BLK, int T>
__device__ __forceinline__ Frag<E> read_frag(const char* tile, const LaneRead<E, KC>& lr) {
    Frag<E> f;
    if constexpr (KC) {
        const char* at = tile + BLK * 32 * 128 + (lr.a ^ (T << 5));
        if constexpr (sizeof(E) == 2) {
            f.v = *reinterpret_cast<const bf16x8*>(at);
        } else {
            const float4 x = *reinterpret_cast<const float4*>(at);
            f.v[0] = x.x; f.v[1] = x.y; f.v[2] = x.z; f.v[3] = x.w;
        }
    } else if constexpr (sizeof(E) == 2) {
        const char* sub = tile + (BLK >> 2) * (kBK<E> * 256) + T * 16 * 256;
        Frag8 x;
        x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((mma::lds_bf16x4*)(sub + (lr.a ^ ((BLK & 3) << 6))));
        x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((mma::lds_bf16x4*)(sub + (lr.b ^ ((BLK & 3) << 6))));
        f.v = x.v;
    } else {
        const char* sub = tile + (BLK >> 1) * (kBK<E> * 256) + T * 8 * 256 + (lr.a ^ ((BLK & 1) << 7));
#pragma unroll
        for (int j = 0; j < 4; ++j) f.v[j] = *reinterpret_cast<const float*>(sub + j * 256);
    }
    return f;
}

__device__ __forceinline__ f32x16 mfma(const Frag<uint16_t>& a, const Frag<uint16_t>& b, f32x16 c) { return mma::mfma(a.v, b.v, c); }
__device__ __forceinline__ f32x16 mfma(const Frag<float>& a, const Frag<float>& b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
}

// ---- a tile through registers: any size, any alignment, zeros outside
struct __attribute__((packed, aligned(2))) Raw16 {
    uint32_t w[4];
};

template <typename E>
__device__ __forceinline__ uint4 load_part(const E* p, int n) {  // the first n of a chunk, the rest zero
    union { E e[kChunk<E>]; uint4 u; } x;
    x.u = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < kChunk<E>; ++j)
        if (j < n) x.e[j] = p[j];
    return x.u;
}

// chunk c of a tile; `row0`: its first m or n, k0 its first k.  `pick(row)` says which matrix and which of its rows a tile row stands for
template <typename E, bool KC, int ROWS, typename Pick>
__device__ __forceinline__ uint4 fetch(int c, int64_t ld, int k0, int K, int row0, int n_rows, Pick&& pick) {
    int k, row, n;
    const E* p;
    if constexpr (KC) {
        const auto [base, r] = pick(c >> 3);
        row = r;
        k = k0 + (c & 7) * kChunk<E>;
        n = row < n_rows ? K - k : 0;
        p = static_cast<const E*>(base) + row * ld + k;
    } else {
        constexpr int per_row = ROWS * static_cast<int>(sizeof(E)) / 16;
        const auto [base, r] = pick(0);
        row = r + (c % per_row) * kChunk<E>;
        k = k0 + c / per_row;
        n = k < K ? n_rows - row : 0;
        p = static_cast<const E*>(base) + k * ld + row;
    }
    if (n <= 0) return make_uint4(0, 0, 0, 0);
    if (n < kChunk<E>) return load_part(p, n);
    const Raw16 x = *reinterpret_cast<const Raw16*>(p);
    return make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
}

// ---- activation: ACT as psattn_act
// SiLU a = g s, a' = s (1 + g (1 - s)), s = 1 / (1 + exp(-g)); GELU a = g Phi(g), a' = Phi(g) + g phi(g), Phi by erfc, which
// keeps its relative accuracy where the gate is closed.  For bf16 the exponential is the hardware's (off by |g| 2^-24 relatively) and
// so is the reciprocal (2^-23): nothing beside the result's own 2^-8.
template <typename E>
__device__ __forceinline__ float exp_of(float x) {
    if constexpr (sizeof(E) == 2) return __expf(x);
    else return expf(x);
}
template <typename E>
__device__ __forceinline__ float logistic(float g) {
    if constexpr (sizeof(E) == 2) return __builtin_amdgcn_rcpf(1.f + __expf(-g));
    else return 1.f / (1.f + expf(-g));
}
template <typename E, int ACT>
__device__ __forceinline__ float act(float g) {
    if constexpr (ACT == 0) return g * logistic<E>(g);
    else return 0.5f * g * erfcf(-0.70710678118654752f * g);
}
template <typename E, int ACT>
__device__ __forceinline__ void act_grad(float g, float& a, float& da) {
    if constexpr (ACT == 0) {
        const float s = logistic<E>(g);
        a = g * s;
        da = s * (1.f + g * (1.f - s));
    } else {
        const float cdf = 0.5f * erfcf(-0.70710678118654752f * g);
        a = g * cdf;
        da = cdf + g * 0.3989422804014327f * exp_of<E>(-0.5f * g * g);
    }
}

}  // namespace gemm
}  // namespace psattn
