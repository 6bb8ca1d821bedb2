// The feed-forward block's bf16 products on whole 16-byte groups: tiles of 256 x 256, copied to LDS asynchronously.
//
// Workgroups of eight waves (one to a CU, two waves to a SIMD), 128 m x 64 n to a wave: 128 accumulator registers, six operand
// reads from LDS for eight MFMAs.  64 k at a time in two LDS buffers of 64 KB.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <utility>

#include "psattn.h"
#include "psattn_ffn.h"

namespace psattn {
namespace gemm {
namespace {

using B = uint16_t;

// Which tile a workgroup takes.  Workgroups go to the eight XCDs in turn: each XCD takes a run of tiles, and the run goes through
// kGroup rows of tiles at a time, so that those that run together share their operands in its L2.
constexpr int kGroup = 8;
__device__ __forceinline__ void tile_of(int b, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int n = tiles_m * tiles_n, x = b % 8, q = n / 8, r = n % 8;
    const int t = x * q + min(x, r) + b / 8;
    const int per = kGroup * tiles_n, grp = t / per, in = t - grp * per, rows = min(kGroup, tiles_m - grp * kGroup);
    tm = grp * kGroup + in % rows;
    tn = in / rows;
}

// Copies of one operand's tile, 1024 bytes to a wave instruction: PER instructions for each of NW waves.
template <bool KC, int ROWS, int NW, bool GATE>
struct Copy {
    static constexpr int PER = ROWS * 128 / 1024 / NW;
    uint32_t off[PER];
    // r0: first m or n of the tile, n_rows: how many there are in all.  What lies behind them is read again from the last one: those
    // results are not stored
    __device__ __forceinline__ void set(int64_t ld, int r0, int n_rows, int w, int l) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int q = w * PER + j;
            if constexpr (KC) {
                const int row = q * 8 + (l >> 3);
                const int r = GATE ? (row >> 6) * 32 + (row & 31) : row;
                off[j] = static_cast<uint32_t>(min(r, n_rows - 1 - r0) * ld * 2) + (((l & 7) ^ swizzle<B, true>(row)) << 4);
            } else {
                const int sub = q / (kBK<B> / 4), row = (q % (kBK<B> / 4)) * 4 + (l >> 4);
                const int ch = sub * 16 + ((l & 15) ^ swizzle<B, false>(row));
                off[j] = static_cast<uint32_t>(row * ld * 2) + (min(ch, (n_rows - r0) / 8 - 1) << 4);
            }
        }
    }
    template <int J>
    __device__ __forceinline__ void issue(const char* base, const char* tile, int w) const {
        mma::dma16(base, off[J], mma::lds_addr(tile) + (w * PER + J) * 1024);
    }
};

// Eight neighbouring n of two rows of m each: an accumulator's values after a swap between the half-waves.  Lane l has n = 16 k +
// 8 (l / 32) .. of row l % 32
struct Chunks {
    float c[2][8];
};
__device__ __forceinline__ Chunks chunks(const f32x16& x) {
    Chunks o;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[8 * k + j]), __float_as_uint(x[8 * k + 4 + j]), false, false);
            o.c[k][j] = __uint_as_float(r[0]);
            o.c[k][4 + j] = __uint_as_float(r[1]);
        }
    return o;
}
// Stores a block of 32 x 32, 64 contiguous bytes of 16 rows at a time (rows r and r + 16 trade chunks between 16-lane halves)
__device__ __forceinline__ void store_chunks(B* base, int64_t ld, int rows, int cols, const Chunks& x, int l) {
    uint32_t c[2][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const auto r = __builtin_amdgcn_permlane16_swap(mma::pack2(x.c[0][2 * j], x.c[0][2 * j + 1]), mma::pack2(x.c[1][2 * j], x.c[1][2 * j + 1]), false, false);
        c[0][j] = r[0];
        c[1][j] = r[1];
    }
    const int row = l & 15, col = 16 * ((l >> 4) & 1) + 8 * (l >> 5);
    if (col >= cols) return;
    B* const p = base + row * ld + col;
    if (row < rows) *reinterpret_cast<uint4*>(p) = make_uint4(c[0][0], c[0][1], c[0][2], c[0][3]);
    if (row + 16 < rows) *reinterpret_cast<uint4*>(p + 16 * ld) = make_uint4(c[1][0], c[1][1], c[1][2], c[1][3]);
}
__device__ __forceinline__ void load_chunk(const B* p, float (&x)[8]) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}

template <bool PKC, bool QKC, Pass PASS, int ACT, int BM, int BN, int WM, int WN>
struct Cfg {
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int MB = BM / WM / 32, NB = BN / WN / 32;  // blocks of a wave
    static constexpr int kCols = PASS == kGate ? BN / 2 : BN;   // n of a tile: gate and up share it
    static constexpr int kPBytes = BM * 128, kQBytes = BN * 128;
    static_assert(PASS != kGate || NB == 2, "a wave holds a block of the gate and the same of up");
};

template <bool PKC, bool QKC, Pass PASS, int ACT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void psattn_ffn_tiles(Product d, int tiles_m, int tiles_n) {
    using C = Cfg<PKC, QKC, PASS, ACT, BM, BN, WM, WN>;
    constexpr int MB = C::MB, NB = C::NB, kPB = C::kPBytes, kQB = C::kQBytes, kBk = kBK<B>;
    __shared__ __attribute__((aligned(1024))) char lds[2 * (kPB + kQB)];
    char *const ptile = lds, *const qtile = lds + 2 * kPB;  // two buffers each, so that a read's buffer is in its immediate offset
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w / WN, wn = w % WN;
    const int z = blockIdx.y;
    int tm, tn;
    tile_of(blockIdx.x, tiles_m, tiles_n, tm, tn);
    const int m0 = tm * BM, n0 = tn * C::kCols;
    Copy<PKC, BM, C::kWaves, false> cp;
    Copy<QKC, BN, C::kWaves, PASS == kGate> cq;
    cp.set(d.ldp, m0, d.M, w, l);
    cq.set(d.ldq, n0, d.N, w, l);
    const LaneRead<B, PKC> lp(l, wm * MB);
    const LaneRead<B, QKC> lq(l, wn * NB);
    f32x16 acc[NB][MB] = {};
    Frag<B> fp[2][MB], fq[2][NB];

    const int per_seg = d.K / kBk, total = per_seg * d.n_seg;  // whole tiles
    const int64_t p_row0 = PKC ? m0 * d.ldp : m0, q_row0 = QKC ? n0 * d.ldq : n0;
    const int64_t p_step = (PKC ? kBk : kBk * d.ldp) * 2, q_step = (QKC ? kBk : kBk * d.ldq) * 2;
    auto p_base = [&](int seg) { return static_cast<const char*>(d.p[d.n_prod > 1 ? z : seg]) + p_row0 * 2; };
    auto q_base = [&](int seg) { return static_cast<const char*>(d.q[seg]) + q_row0 * 2; };
    // where the next copies come from
    const char *pc = p_base(0), *qc = q_base(0), *qc2 = PASS == kGate ? q_base(1) : nullptr;
    int left = per_seg;  // tiles of the segment not yet copied
    // of a tile: PER copies of P, then those of Q
    constexpr int kP = Copy<PKC, BM, C::kWaves, false>::PER, kQ = Copy<QKC, BN, C::kWaves, PASS == kGate>::PER, kCopies = kP + kQ;
    auto copy = [&](auto J, auto BUF) {
        constexpr int j = decltype(J)::value, buf = decltype(BUF)::value;
        if constexpr (j < kP) {
            cp.template issue<j>(pc, ptile + buf * kPB, w);
        } else {
            const char* base = qc;
            if constexpr (PASS == kGate) base = (((w * kQ + j - kP) * 8) >> 5) & 1 ? qc2 : qc;
            cq.template issue<j - kP>(base, qtile + buf * kQB, w);
        }
    };
    auto advance = [&] {
        pc += p_step;
        qc += q_step;
        if constexpr (PASS == kGate) qc2 += q_step;
        if (--left == 0 && d.n_seg > 1) {
            pc = p_base(1);
            qc = q_base(1);
        }
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    auto read = [&](auto R, auto SET, auto BUF, auto T) {  // the R-th operand of step T
        constexpr int r = decltype(R)::value, set = decltype(SET)::value, buf = decltype(BUF)::value, t = decltype(T)::value;
        if constexpr (r < NB) fq[set][r] = read_frag<B, QKC, r, t>(qtile + buf * kQB, lq);
        else fp[set][r - NB] = read_frag<B, PKC, r - NB, t>(ptile + buf * kPB, lp);
    };
    constexpr int kSteps = 4, kReads = MB + NB, kSlots = MB * NB;
    // One tile.  Its first step's operands are in registers; those of a step are read while the one before is multiplied.  Ahead
    // of the last step all waves have read their last operands of this tile and the next tile has arrived: the barrier
    // stands there, behind it the next tile's first operands are read and the buffer is filled again.
    auto tile = [&](auto BUF, bool more) {
        constexpr int buf = decltype(BUF)::value;
        static_for<0, kSteps>([&](auto T) {
            constexpr int t = decltype(T)::value, set = t & 1;
            if constexpr (t == kSteps - 1) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            static_for<0, kSlots>([&](auto S) {
                constexpr int s = decltype(S)::value;
                if constexpr (s < kReads) {
                    if constexpr (t < kSteps - 1) read(S, std::integral_constant<int, set ^ 1>{}, BUF, std::integral_constant<int, t + 1>{});
                    else read(S, std::integral_constant<int, set ^ 1>{}, std::integral_constant<int, buf ^ 1>{}, I0{});
                }
                if constexpr (t == kSteps - 1)
                    if (more)
                        static_for<0, (kCopies + kSlots - 1) / kSlots>([&](auto X) {
                            constexpr int j = s + decltype(X)::value * kSlots;
                            if constexpr (j < kCopies) copy(std::integral_constant<int, j>{}, BUF);
                        });
                acc[s % NB][s / NB] = mfma(fq[set][s % NB], fp[set][s / NB], acc[s % NB][s / NB]);
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        if (more) advance();
    };
    if (total > 0) {
        static_for<0, kCopies>([&](auto J) { copy(J, I0{}); });
        advance();
        if (total > 1) {
            static_for<0, kCopies>([&](auto J) { copy(J, I1{}); });
            advance();
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kCopies) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        }
        static_for<0, kReads>([&](auto R) { read(R, I0{}, I0{}, I0{}); });
        int i = 0;
        for (; i + 1 < total; i += 2) {
            tile(I0{}, i + 2 < total);
            tile(I1{}, i + 3 < total);
        }
        if (i < total) tile(I0{}, false);
    }
    if (const int rest = per_seg * kBk; rest < d.K) {  // what is left of k, through registers, zeros behind it
        for (int seg = 0; seg < d.n_seg; ++seg) {
            __syncthreads();
            for (int c = threadIdx.x; c < BM * 8; c += C::kThreads)
                *reinterpret_cast<uint4*>(ptile + chunk_off<B, PKC, BM>(c)) = fetch<B, PKC, BM>(c, d.ldp, rest, d.K, m0, d.M, [&](int r) { return std::make_pair(d.p[d.n_prod > 1 ? z : seg], m0 + r); });
            for (int c = threadIdx.x; c < BN * 8; c += C::kThreads)
                *reinterpret_cast<uint4*>(qtile + chunk_off<B, QKC, BN>(c)) = fetch<B, QKC, BN>(c, d.ldq, rest, d.K, n0, d.N, [&](int r) {
                    if constexpr (PASS == kGate) return std::make_pair(d.q[(r >> 5) & 1], n0 + (r >> 6) * 32 + (r & 31));
                    else return std::make_pair(d.q[seg], n0 + r);
                });
            __syncthreads();
            static_for<0, kSteps>([&](auto T) {
                static_for<0, kReads>([&](auto R) { read(R, I0{}, I0{}, T); });
                static_for<0, kSlots>([&](auto S) {
                    constexpr int s = decltype(S)::value;
                    acc[s % NB][s / NB] = mfma(fq[0][s % NB], fp[0][s / NB], acc[s % NB][s / NB]);
                });
            });
        }
    }
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int m = m0 + (wm * MB + mb) * 32, rows = d.M - m;
        if (rows <= 0) break;
        __builtin_amdgcn_sched_barrier(0);  // one block at a time: beside 128 accumulators there is no room for more
        if constexpr (PASS == kGate) {
            const int n = n0 + wn * 32, cols = d.N - n;
            if (cols <= 0) break;
            const int64_t at = m * d.ldo + n;
            f32x16 h;
#pragma unroll
            for (int i = 0; i < 16; ++i) h[i] = act<ACT>(acc[0][mb][i]) * acc[1][mb][i];
            if (d.G) store_chunks(static_cast<B*>(d.G) + at, d.ldo, rows, cols, chunks(acc[0][mb]), l);
            if (d.U) store_chunks(static_cast<B*>(d.U) + at, d.ldo, rows, cols, chunks(acc[1][mb]), l);
            store_chunks(static_cast<B*>(d.H) + at, d.ldo, rows, cols, chunks(h), l);
        } else {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int n = n0 + (wn * NB + nb) * 32, cols = d.N - n;
                if (cols <= 0) break;
                const int64_t at = m * d.ldo + n;
                const Chunks x = chunks(acc[nb][mb]);
                if constexpr (PASS == kPlain) {
                    store_chunks(static_cast<B*>(d.out[d.n_prod > 1 ? z : 0]) + at, d.ldo, rows, cols, x, l);
                } else {
                    Chunks dg, du;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        // rows and columns outside: read from inside, not stored
                        const int64_t from = at + min(l & 31, rows - 1) * d.ldo + min(16 * k + 8 * (l >> 5), cols - 8);
                        float gate[8], up[8];
                        load_chunk(static_cast<const B*>(d.G) + from, gate);
                        load_chunk(static_cast<const B*>(d.U) + from, up);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            float a, da;
                            act_grad<ACT>(gate[j], a, da);
                            dg.c[k][j] = x.c[k][j] * up[j] * da;
                            du.c[k][j] = x.c[k][j] * a;
                        }
                    }
                    store_chunks(static_cast<B*>(d.out[0]) + at, d.ldo, rows, cols, dg, l);
                    store_chunks(static_cast<B*>(d.out[1]) + at, d.ldo, rows, cols, du, l);
                }
            }
        }
    }
}

template <bool PKC, bool QKC, Pass PASS, int ACT, int BM, int BN, int WM, int WN>
int launch(const Product& d, hipStream_t s) {
    using C = Cfg<PKC, QKC, PASS, ACT, BM, BN, WM, WN>;
    const int64_t tn = (static_cast<int64_t>(d.N) + C::kCols - 1) / C::kCols, tm = (static_cast<int64_t>(d.M) + BM - 1) / BM;
    if (tn * tm >= (int64_t{1} << 31) / C::kThreads) return PSATTN_EUNSUPPORTED;  // 2^31 threads to a grid
    psattn_ffn_tiles<PKC, QKC, PASS, ACT, BM, BN, WM, WN><<<dim3(static_cast<uint32_t>(tn * tm), d.n_prod), C::kThreads, 0, s>>>(d, static_cast<int>(tm), static_cast<int>(tn));
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

template <bool PKC, bool QKC, Pass PASS, int ACT>
int sized(const Product& d, hipStream_t s) {
    return launch<PKC, QKC, PASS, ACT, 256, 256, 2, 4>(d, s);
}

bool at16(std::initializer_list<const void*> p) {
    uintptr_t a = 0;
    for (const void* x : p) a |= reinterpret_cast<uintptr_t>(x);
    return a % 16 == 0;
}

}  // namespace

// Every row of P, Q and out a whole number of 16-byte groups on 16-byte boundaries; a tile's copies within 32-bit offsets
bool product_mfma_ok(bool pkc, bool qkc, const Product& d) {
    if (!at16({d.p[0], d.p[1], d.q[0], d.q[1], d.out[0], d.out[1], d.G, d.U, d.H})) return false;
    if (d.ldp % 8 || d.ldq % 8 || d.ldo % 8 || d.N % 8) return false;
    if ((pkc ? d.K : d.M) % 8 || (qkc && d.K % 8)) return false;
    return std::max(d.ldp, d.ldq) * 2 * 256 < (int64_t{1} << 31);
}

int product_mfma(Pass pass, int act, bool pkc, bool qkc, const Product& d, hipStream_t s) {
    if (pass == kGate) return act == PSATTN_ACT_SILU ? sized<true, true, kGate, 0>(d, s) : sized<true, true, kGate, 1>(d, s);
    if (pass == kDact) return act == PSATTN_ACT_SILU ? sized<true, false, kDact, 0>(d, s) : sized<true, false, kDact, 1>(d, s);
    if (pkc && qkc) return sized<true, true, kPlain, 0>(d, s);
    if (pkc) return sized<true, false, kPlain, 0>(d, s);
    return sized<false, false, kPlain, 0>(d, s);
}

}  // namespace gemm
}  // namespace psattn
