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
    if constexpr (sizeof(E) == 4) {  // dX of more items comes with dW
        if (size == k32) return launch_tiles<E, ASYNC, true, false, kSums, 0, Shape<32, 128, 1, 2, 2>>(d, s);
        return launch_tiles<E, ASYNC, true, false, kSums, 0, Shape<64, 128, 1, 2, 2>>(d, s);
    } else {
        return launch_sized<E, ASYNC, true, false, kSums, 0>(size, d, s);
    }
}

// A piece's two products of dz in one launch, tiles of 256 x 256, or 128 x 128 of fp32: first dX's, whose k is the piece, then dW's, whose k is the items and
// which fill the chip to the end of the launch
template <typename E, bool ASYNC, typename S>
__global__ __launch_bounds__(S::kThreads, S::kWavesToSimd) void psattn_head_grads(Product x, Product w, int x_tiles_m, int x_tiles_n, int w_tiles_m, int w_tiles_n) {
    __shared__ __attribute__((aligned(1024))) char lds[kLds<S>];
    const int n = x_tiles_m * x_tiles_n, first = n * x.n_split, b = blockIdx.x;
    if (b < first) product_tile<E, ASYNC, true, false, kSums, 0, S>(lds, x, x_tiles_m, x_tiles_n, b % n, b / n);
    else product_tile<E, ASYNC, false, false, sizeof(E) == 2 ? kTokens : kPlain, 0, S>(lds, w, w_tiles_m, w_tiles_n, (b - first) % (w_tiles_m * w_tiles_n), (b - first) / (w_tiles_m * w_tiles_n));
}

// dW of few items, a few steps of k: what is written bounds it, and workgroups with one buffer of either operand leave a CU room for four.
// 32 000 x 4 096 bf16 in us, with psattn_ffn_tiles / so: 1 item 88 / 51; a whole step, forward and backward, 99 items 292 / 272, 122 298 / 274,
// 165 345 / 331, 231 381 / 369, 440 the same.  100 014 x 2 752 fp32 of two items 502 / 194.  k ends at the last item: the rows up to a
// whole step are zeros, and fp32 has no MFMAs to spare for them
template <typename E, bool ASYNC, typename S>
__global__ __launch_bounds__(S::kThreads, 4) void psattn_head_outer(Product d, int tiles_m, int tiles_n) {
    constexpr int MB = S::MB, NB = S::NB, kPB = S::BM * 128, kQB = S::BN * 128, kSteps = 4;
    // results leave through LDS: of a wave 32 rows with 16 bytes more each, which spreads them over the banks
    constexpr int kCols = NB * 32, kPitch = kCols * static_cast<int>(sizeof(E)) + 16, kOut = S::kWaves * 32 * kPitch;
    __shared__ __attribute__((aligned(1024))) char lds[kPB + kQB > kOut ? kPB + kQB : kOut];
    char *const ptile = lds, *const qtile = lds + kPB;
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w / S::WN, wn = w % S::WN;
    int tm, tn;
    tile_of(blockIdx.x, tiles_m, tiles_n, tm, tn);
    const int m0 = tm * S::BM, n0 = tn * S::BN;
    Copy<E, false, S::BM, S::kWaves, false, ASYNC> cp;
    Copy<E, false, S::BN, S::kWaves, false, ASYNC> cq;
    cp.set(d.ldp, m0, d.m_load, w, l);
    cq.set(d.ldq, n0, d.n_load, w, l);
    const LaneRead<E, false> lp(l, wm * MB), lq(l, wn * NB);
    constexpr int kP = decltype(cp)::PER, kQ = decltype(cq)::PER;
    const char *pc = static_cast<const char*>(d.p[0]) + m0 * static_cast<int64_t>(sizeof(E)), *qc = static_cast<const char*>(d.q[0]) + n0 * static_cast<int64_t>(sizeof(E));
    int item[MB];  // asked for ahead of the copies
    if constexpr (sizeof(E) == 2) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const int row = m0 + (wm * MB + mb) * 32 + (l & 31);
            item[mb] = d.out[1] && row < d.M ? static_cast<const int32_t*>(d.H)[row] : -1;
        }
    }
    f32x16 acc[NB][MB] = {};
    for (int k = 0; k < d.K; k += kBK<E>) {
        if (k > 0) __syncthreads();
        static_for<0, kP>([&](auto J) { cp.template issue<decltype(J)::value>(pc, ptile, w); });
        static_for<0, kQ>([&](auto J) { cq.template issue<decltype(J)::value>(qc, qtile, w); });
        pc += kBK<E> * d.ldp * static_cast<int64_t>(sizeof(E));
        qc += kBK<E> * d.ldq * static_cast<int64_t>(sizeof(E));
        if constexpr (ASYNC) {
            asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        } else {
            static_for<0, kP>([&](auto J) { cp.template put<decltype(J)::value>(ptile, w, l); });
            static_for<0, kQ>([&](auto J) { cq.template put<decltype(J)::value>(qtile, w, l); });
            __syncthreads();
        }
        static_for<0, kSteps>([&](auto T) {
            constexpr int t = decltype(T)::value;
            if (k + t * (kBK<E> / kSteps) >= d.K) return;  // zeros
            Frag<E> fp[MB], fq[NB];
            static_for<0, NB>([&](auto R) { fq[decltype(R)::value] = read_frag<E, false, decltype(R)::value, t>(qtile, lq); });
            static_for<0, MB>([&](auto R) { fp[decltype(R)::value] = read_frag<E, false, decltype(R)::value, t>(ptile, lp); });
            static_for<0, NB * MB>([&](auto I) {
                constexpr int i = decltype(I)::value;
                acc[i % NB][i / NB] = mfma(fq[i % NB], fp[i / NB], acc[i % NB][i / NB]);
            });
        });
    }
    // A block of 32 rows at a time, so that whole lines leave: 128 bytes of a row to eight lanes.  (From the accumulators 64 bytes of bf16 and
    // 16 of fp32 would leave together.)
    __syncthreads();
    constexpr int EPC = kChunk<E>, kPer = 32 * kCols / EPC / 64;
    char* const mine = lds + w * 32 * kPitch;
    const int nw = n0 + wn * kCols;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int m = m0 + (wm * MB + mb) * 32;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const Chunks x = chunks(acc[nb][mb]);
            if constexpr (sizeof(E) == 2)
                if (item[mb] >= 0) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int n = nw + nb * 32 + 16 * k + 8 * (l >> 5);
                        put_rest(static_cast<uint16_t*>(d.out[1]) + item[mb] * d.ldo + n, x.c[k], d.N - n);
                    }
                }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                char* const to = mine + (l & 31) * kPitch + (nb * 32 + 16 * k + 8 * (l >> 5)) * static_cast<int>(sizeof(E));
                if constexpr (sizeof(E) == 2) {
                    *reinterpret_cast<uint4*>(to) = make_uint4(mma::pack2(x.c[k][0], x.c[k][1]), mma::pack2(x.c[k][2], x.c[k][3]), mma::pack2(x.c[k][4], x.c[k][5]), mma::pack2(x.c[k][6], x.c[k][7]));
                } else {
                    *reinterpret_cast<float4*>(to) = make_float4(x.c[k][0], x.c[k][1], x.c[k][2], x.c[k][3]);
                    *reinterpret_cast<float4*>(to + 16) = make_float4(x.c[k][4], x.c[k][5], x.c[k][6], x.c[k][7]);
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            constexpr int kRow = kCols / EPC;  // chunks of a row
            const int c = j * 64 + l, row = c / kRow, col = c % kRow * EPC, n = nw + col;
            const uint4 u = *reinterpret_cast<const uint4*>(mine + row * kPitch + col * static_cast<int>(sizeof(E)));
            if (m + row >= d.M || n >= d.N) continue;
            E* const to = static_cast<E*>(d.out[0]) + (m + row) * d.ldo + n;
            if (!d.odd) {
                *reinterpret_cast<uint4*>(to) = u;
            } else if (n + EPC <= d.N) {
                *reinterpret_cast<Raw16*>(to) = Raw16{u.x, u.y, u.z, u.w};
            } else {
                union { uint4 u; E e[EPC]; } v{u};
#pragma unroll
                for (int k = 0; k < EPC; ++k)
                    if (n + k < d.N) to[k] = v.e[k];
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename E, bool ASYNC>
int launch_outer(const Product& d, hipStream_t s) {
    using S = Shape<128, 128, 2, 2, 2>;
    const int64_t m = (static_cast<int64_t>(d.M) + S::BM - 1) / S::BM, n = (static_cast<int64_t>(d.N) + S::BN - 1) / S::BN;
    if (m * n >= (int64_t{1} << 31) / S::kThreads) return PSATTN_EUNSUPPORTED;
    psattn_head_outer<E, ASYNC, S><<<static_cast<uint32_t>(m * n), S::kThreads, 0, s>>>(d, static_cast<int>(m), static_cast<int>(n));
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

template <typename E, bool ASYNC>
int launch_grads(const Product& x, const Product& w, hipStream_t s) {
    using S = std::conditional_t<sizeof(E) == 2, Shape<256, 256, 2, 4, 3>, Shape<128, 128, 2, 2, ASYNC ? 3 : 2>>;
    auto tiles = [](int64_t n) { return (n + S::BM - 1) / S::BM; };
    const int64_t xm = tiles(x.M), xn = tiles(x.N), wm = tiles(w.M), wn = tiles(w.N), n = xm * xn * x.n_split + wm * wn * w.n_split;
    if (n >= (int64_t{1} << 31) / S::kThreads) return PSATTN_EUNSUPPORTED;
    psattn_head_grads<E, ASYNC, S><<<static_cast<uint32_t>(n), S::kThreads, 0, s>>>(x, w, static_cast<int>(xm), static_cast<int>(xn), static_cast<int>(wm), static_cast<int>(wn));
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

}  // namespace gemm
}  // namespace psattn
