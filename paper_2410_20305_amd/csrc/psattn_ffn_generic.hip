// The feed-forward block's products for any type, size and alignment: fp32, and bf16 whose rows are not whole 16-byte groups.
//
// Workgroups of four waves, tiles of 128 x 128, 64 x 64 to a wave (64 accumulator registers), 128 bytes of k at a time.  The
// next tile's chunks are loaded into registers while the present one is multiplied, and go to LDS between two barriers.
// bf16 products use the bf16 MFMAs, fp32 ones v_mfma_f32_32x32x2_f32 (exact fp32 products, 157 TFLOP/s at most).
#include <hip/hip_runtime.h>

#include <tuple>

#include "psattn.h"
#include "psattn_ffn.h"

namespace psattn {
namespace gemm {
namespace {

constexpr int kTile = 128, kThreads = 256;

template <typename E, bool PKC, bool QKC, Pass PASS, int ACT>
__global__ __launch_bounds__(kThreads) void psattn_ffn_any(Product d, int tiles_n) {
    __shared__ __attribute__((aligned(16))) char lds[2 * kTile * 128];
    char *const tp = lds, *const tq = lds + kTile * 128;
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w >> 1, wn = w & 1;
    const int z = blockIdx.y;
    constexpr int kCols = PASS == kGate ? kTile / 2 : kTile;  // n of a tile: gate and up share it
    const int m0 = static_cast<int>(blockIdx.x / tiles_n) * kTile, n0 = static_cast<int>(blockIdx.x % tiles_n) * kCols;
    const int steps = (d.K + kBK<E> - 1) / kBK<E>, total = steps * d.n_seg;
    f32x16 acc[2][2] = {};  // [n block][m block]
    const LaneRead<E, PKC> lp(l, 2 * wm);
    const LaneRead<E, QKC> lq(l, 2 * wn);
    constexpr int kPer = kTile * 8 / kThreads;  // chunks of a thread and operand
    uint4 rp[kPer], rq[kPer];
    auto load = [&](int i) {
        const int seg = i / steps, k0 = (i - seg * steps) * kBK<E>;
        const void* pb = d.p[d.n_prod > 1 ? z : seg];
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int c = threadIdx.x + j * kThreads;
            rp[j] = fetch<E, PKC, kTile>(c, d.ldp, k0, d.K, m0, d.M, [&](int r) { return std::make_pair(pb, m0 + r); });
            rq[j] = fetch<E, QKC, kTile>(c, d.ldq, k0, d.K, n0, d.N, [&](int r) {
                // kGate: 32 rows of the gate, then the same 32 of up
                if constexpr (PASS == kGate) return std::make_pair(d.q[(r >> 5) & 1], n0 + (r >> 6) * 32 + (r & 31));
                else return std::make_pair(d.q[seg], n0 + r);
            });
        }
    };
    if (total > 0) load(0);
    for (int i = 0; i < total; ++i) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int c = threadIdx.x + j * kThreads;
            *reinterpret_cast<uint4*>(tp + chunk_off<E, PKC, kTile>(c)) = rp[j];
            *reinterpret_cast<uint4*>(tq + chunk_off<E, QKC, kTile>(c)) = rq[j];
        }
        __syncthreads();
        if (i + 1 < total) load(i + 1);
        static_for<0, 4>([&](auto T) {
            constexpr int t = decltype(T)::value;
            const Frag<E> p0 = read_frag<E, PKC, 0, t>(tp, lp), p1 = read_frag<E, PKC, 1, t>(tp, lp);
            const Frag<E> q0 = read_frag<E, QKC, 0, t>(tq, lq), q1 = read_frag<E, QKC, 1, t>(tq, lq);
            acc[0][0] = mfma(q0, p0, acc[0][0]);
            acc[0][1] = mfma(q0, p1, acc[0][1]);
            acc[1][0] = mfma(q1, p0, acc[1][0]);
            acc[1][1] = mfma(q1, p1, acc[1][1]);
        });
    }
    // accumulator register i: n = acc_row(i, l / 32) of its block, m = l % 32
    const int g = l >> 5;
#pragma unroll
    for (int mb = 0; mb < 2; ++mb) {
        const int m = m0 + wm * 64 + mb * 32 + (l & 31);
        if (m >= d.M) continue;
        if constexpr (PASS == kGate) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int n = n0 + wn * 32 + mma::acc_row(i, g);
                if (n >= d.N) continue;
                const int64_t at = m * d.ldo + n;
                const float gate = acc[0][mb][i], up = acc[1][mb][i];
                if (d.G) store1(static_cast<E*>(d.G) + at, gate);
                if (d.U) store1(static_cast<E*>(d.U) + at, up);
                store1(static_cast<E*>(d.H) + at, act<ACT>(gate) * up);
            }
        } else {
#pragma unroll
            for (int nb = 0; nb < 2; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int n = n0 + wn * 64 + nb * 32 + mma::acc_row(i, g);
                    if (n >= d.N) continue;
                    const int64_t at = m * d.ldo + n;
                    const float x = acc[nb][mb][i];
                    if constexpr (PASS == kPlain) {
                        store1(static_cast<E*>(d.out[d.n_prod > 1 ? z : 0]) + at, x);
                    } else {
                        float a, da;
                        act_grad<ACT>(to_f32(static_cast<const E*>(d.G)[at]), a, da);
                        const float up = to_f32(static_cast<const E*>(d.U)[at]);
                        store1(static_cast<E*>(d.out[0]) + at, x * up * da);
                        store1(static_cast<E*>(d.out[1]) + at, x * a);
                    }
                }
        }
    }
}

template <typename E, bool PKC, bool QKC, Pass PASS, int ACT>
int launch(const Product& d, hipStream_t s) {
    constexpr int kCols = PASS == kGate ? kTile / 2 : kTile;
    const int64_t tn = (static_cast<int64_t>(d.N) + kCols - 1) / kCols, tm = (static_cast<int64_t>(d.M) + kTile - 1) / kTile;
    if (tn * tm >= (int64_t{1} << 31) / kThreads) return PSATTN_EUNSUPPORTED;  // 2^31 threads to a grid
    psattn_ffn_any<E, PKC, QKC, PASS, ACT><<<dim3(static_cast<uint32_t>(tn * tm), d.n_prod), kThreads, 0, s>>>(d, static_cast<int>(tn));
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

template <typename E>
int typed(Pass pass, int act, bool pkc, bool qkc, const Product& d, hipStream_t s) {
    if (pass == kGate) return act == PSATTN_ACT_SILU ? launch<E, true, true, kGate, 0>(d, s) : launch<E, true, true, kGate, 1>(d, s);
    if (pass == kDact) return act == PSATTN_ACT_SILU ? launch<E, true, false, kDact, 0>(d, s) : launch<E, true, false, kDact, 1>(d, s);
    if (pkc && qkc) return launch<E, true, true, kPlain, 0>(d, s);
    if (pkc) return launch<E, true, false, kPlain, 0>(d, s);
    return launch<E, false, false, kPlain, 0>(d, s);
}

}  // namespace

int product_any(int dt, Pass pass, int act, bool pkc, bool qkc, const Product& d, hipStream_t s) {
    return dt == PSATTN_BF16 ? typed<uint16_t>(pass, act, pkc, qkc, d, s) : typed<float>(pass, act, pkc, qkc, d, s);
}

}  // namespace gemm
}  // namespace psattn
