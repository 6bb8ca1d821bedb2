// The kernel of the feed-forward block's products (psattn_gemm.h has its tiles and operands), built for bf16 with asynchronous
// copies (psattn_ffn_bf16.hip), for bf16 of any alignment (psattn_ffn_bf16_any.hip) and for fp32 (psattn_ffn_f32.hip).
//
// k goes through LDS buffers, 128 bytes of it (64 bf16, 32 fp32) at a time.  The operands of a step (16 bf16, 8 fp32) are
// read while the step before is multiplied.  Ahead of a tile's last step every wave has read its last operands of it and the
// next tile has arrived: the one barrier of a tile stands there.  Behind it the next tile's first operands are read, so that no
// MFMA waits for LDS, and what follows is asked for.
//   ASYNC       global -> LDS copies, 16-byte groups on 16-byte boundaries.  Q has a third buffer: its copies are asked for a tile earlier than
//               P's, two to a step of either, so that the path to LDS is never without them nor flooded (8 192 tokens, hidden 4 096, inner
//               14 336, forward and backward 7 360 us with two buffers and all copies behind the barrier, 7 085 so; 64 bytes of k in
//               three to five buffers, which reads half lines, 7 320 - 7 410 where two buffers of 128 took 7 120)
//   otherwise   loads into registers (16 bytes from anywhere), written to LDS a tile later, before its barrier; a group that
//               reaches past the end of its row is read from inside it and shifted (same sizes, 10 400 us)
// 256 x 256 to a workgroup of eight waves (one to a CU), 128 m x 64 n to a wave: 128 accumulator registers, six operand reads for eight
// MFMAs; 128 x 128 to four waves (two to a CU); 64 and 32 x 128 to two for few tokens.
//   What bounds the large ones (Y of 8 192 tokens, a tile of k for all workgroups): copies by themselves 1.2 us, 54 GB/s to a CU; MFMAs by
// themselves, on operands that never change and let the clock rise, 1.0; MFMAs and reads without copies 1.3; all of it 1.6 (1.35 PFLOP/s).
#pragma once
#include <hip/hip_runtime.h>

#include <utility>

#include "psattn.h"
#include "psattn_ffn.h"

namespace psattn {
namespace gemm {

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

__device__ __forceinline__ uint4 shift_down(uint4 u, int bits) {  // the chunk as 128 bits
    const uint64_t lo = (static_cast<uint64_t>(u.y) << 32) | u.x, hi = (static_cast<uint64_t>(u.w) << 32) | u.z;
    uint64_t a = lo, b = hi;
    if (bits >= 64) { a = hi >> (bits - 64); b = 0; }
    else if (bits > 0) { a = (lo >> bits) | (hi << (64 - bits)); b = hi >> bits; }
    return make_uint4(static_cast<uint32_t>(a), static_cast<uint32_t>(a >> 32), static_cast<uint32_t>(b), static_cast<uint32_t>(b >> 32));
}

// Copies of one operand's whole tiles: PER chunks of 16 bytes to a lane, 1024 bytes to a wave and instruction.
template <typename E, bool KC, int ROWS, int NW, bool GATE, bool ASYNC>
struct Copy {
    static constexpr int PER = ROWS * 128 / 1024 / NW, EPC = kChunk<E>;
    static constexpr int kBias = ASYNC || KC ? 0 : 16;  // bytes: a chunk may be read from up to one before the tile's first column
    uint32_t off[PER];
    static constexpr int kShifts = sizeof(E) == 2 ? 4 : 1;  // chunks whose shifts, in bits, share a register
    uint32_t shift[ASYNC || KC ? 1 : (PER + kShifts - 1) / kShifts];
    uint4 r[ASYNC ? 1 : PER];
    bool edge, tiny;  // the tile reaches past the rows' ends; rows shorter than a chunk
    int in_row;
    // r0: first m or n of the tile, n_rows: how many there are in all (KS: in a row in memory).  What lies behind them is read again from the
    // last one: those results are not stored
    __device__ __forceinline__ void set(int64_t ld, int r0, int n_rows, int w, int l) {
        edge = !KC && r0 + ROWS > n_rows;
        tiny = !KC && n_rows < EPC;
        in_row = n_rows - r0;
        for (uint32_t& s : shift) s = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int q = w * PER + j;
            if constexpr (KC) {
                const int row = q * 8 + (l >> 3);
                const int at = GATE ? (row >> 6) * 32 + (row & 31) : row;
                off[j] = static_cast<uint32_t>(min(at, n_rows - 1 - r0) * ld * sizeof(E)) + (((l & 7) ^ swizzle<E, true>(row)) << 4);
            } else {
                const int sub = q / (kBK<E> / 4), row = (q % (kBK<E> / 4)) * 4 + (l >> 4);
                const int col = (sub * 16 + ((l & 15) ^ swizzle<E, false>(row))) * EPC;
                int at = min(col, in_row - EPC);
                if constexpr (ASYNC) {
                    at = min(col, in_row / EPC * EPC - EPC);
                } else {
                    shift[j / kShifts] |= static_cast<uint32_t>(col < in_row ? (col - at) * static_cast<int>(sizeof(E)) * 8 : 0) << (8 * (j % kShifts));
                    if (tiny) at = 0;
                }
                off[j] = static_cast<uint32_t>((row * ld + at) * static_cast<int64_t>(sizeof(E)) + kBias);
            }
        }
    }
    template <int J>
    __device__ __forceinline__ void issue(const char* base, char* tile, int w) {
        if constexpr (ASYNC) {
            mma::dma16(base, off[J], mma::lds_addr(tile) + (w * PER + J) * 1024);
        } else if (!KC && tiny) {
            r[J] = load_part(reinterpret_cast<const E*>(base - kBias + off[J]), in_row);
        } else {
            const Raw16 x = *reinterpret_cast<const Raw16*>(base - kBias + off[J]);
            r[J] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
        }
    }
    template <int J>
    __device__ __forceinline__ void put(char* tile, int w, int l) {
        if constexpr (!ASYNC) {
            uint4 u = r[J];
            if constexpr (!KC)
                if (edge && !tiny) {
                    uint32_t s = shift[J / kShifts];
                    if constexpr (kShifts > 1) {
                        asm("" : "+v"(s));  // taken apart ahead of the loop, it would hold four registers there again
                        s = s >> (8 * (J % kShifts)) & 255;
                    }
                    u = shift_down(u, s);
                }
            *reinterpret_cast<uint4*>(tile + (w * PER + J) * 1024 + 16 * l) = u;
        }
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

// eight elements to and from memory; n of them are there
template <bool ALIGNED>
__device__ __forceinline__ void put8(uint16_t* p, const uint32_t (&w)[4], int n) {
    if (n >= 8) {
        if constexpr (ALIGNED) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<Raw16*>(p) = Raw16{w[0], w[1], w[2], w[3]};
    } else if constexpr (!ALIGNED) {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < n) p[j] = static_cast<uint16_t>(w[j >> 1] >> (16 * (j & 1)));
    }
}
__device__ __forceinline__ void put8(float* p, const float (&x)[8], int n) {
    if (n >= 8) {
        *reinterpret_cast<Raw16*>(p) = Raw16{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
        *reinterpret_cast<Raw16*>(p + 4) = Raw16{__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])};
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < n) p[j] = x[j];
    }
}
// eight floats as they come from memory
struct Group {
    float w[8];
    __device__ __forceinline__ void get(const float* p, int n) {
        if (n >= 8) {
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const Raw16 x = *reinterpret_cast<const Raw16*>(p + i);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[i + j] = __uint_as_float(x.w[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = j < n ? p[j] : 0.f;
        }
    }
};

// Stores a block of 32 x 32.  bf16: 64 contiguous bytes of 16 rows at a time (rows r and r + 16 trade chunks between the 16-lane
// halves); fp32: 32 bytes to a lane
template <bool ALIGNED>
__device__ __forceinline__ void store_chunks(uint16_t* base, int64_t ld, int rows, int cols, const Chunks& x, int l) {
    uint32_t c[2][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const auto r = __builtin_amdgcn_permlane16_swap(mma::pack2(x.c[0][2 * j], x.c[0][2 * j + 1]), mma::pack2(x.c[1][2 * j], x.c[1][2 * j + 1]), false, false);
        c[0][j] = r[0];
        c[1][j] = r[1];
    }
    const int row = l & 15, col = 16 * ((l >> 4) & 1) + 8 * (l >> 5);
    uint16_t* const p = base + row * ld + col;
    if (row < rows) put8<ALIGNED>(p, c[0], cols - col);
    if (row + 16 < rows) put8<ALIGNED>(p + 16 * ld, c[1], cols - col);
}
template <bool ALIGNED>
__device__ __forceinline__ void store_chunks(float* base, int64_t ld, int rows, int cols, const Chunks& x, int l) {
    const int row = l & 31, col = 8 * (l >> 5);
    if (row >= rows) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) put8(base + row * ld + 16 * k + col, x.c[k], cols - 16 * k - col);
}

// ... by rows of whole groups or not, which the launch knows
template <bool ASYNC, typename E>
__device__ __forceinline__ void store_out(E* base, int64_t ld, int rows, int cols, const Chunks& x, int l, int odd) {
    if (ASYNC && !odd) store_chunks<true>(base, ld, rows, cols, x, l);
    else store_chunks<false>(base, ld, rows, cols, x, l);
}

template <int BM_, int BN_, int WM_, int WN_, int NBQ_>
struct Shape {  // tile, waves, LDS buffers of Q (of P: two)
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NBQ = NBQ_, kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int MB = BM / WM / 32, NB = BN / WN / 32;  // blocks of a wave
};

template <typename E, bool ASYNC, bool PKC, bool QKC, Pass PASS, int ACT, typename S>
__global__ __launch_bounds__(S::kThreads, 2) void psattn_ffn_tiles(Product d, int tiles_m, int tiles_n) {
    constexpr int MB = S::MB, NB = S::NB, kPB = S::BM * 128, kQB = S::BN * 128, kBk = kBK<E>;
    constexpr int kCols = PASS == kGate ? S::BN / 2 : S::BN;  // n of a tile: gate and up share it
    static_assert(PASS != kGate || NB == 2, "a wave holds a block of the gate and the same of up");
    static_assert(PKC || S::BM % (256 / sizeof(E)) == 0, "whole sub-tiles");
    static_assert(QKC || S::BN % (256 / sizeof(E)) == 0, "whole sub-tiles");
    constexpr int NBQ = S::NBQ;
    static_assert(ASYNC || NBQ == 2, "what goes through registers is one tile ahead");
    __shared__ __attribute__((aligned(1024))) char lds[2 * kPB + NBQ * kQB];
    char *const ptile = lds, *const qtile = lds + 2 * kPB;
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w / S::WN, wn = w % S::WN;
    const int z = blockIdx.y / d.n_split, part = blockIdx.y % d.n_split;  // product, part of its k
    int tm, tn;
    tile_of(blockIdx.x, tiles_m, tiles_n, tm, tn);
    const int m0 = tm * S::BM, n0 = tn * kCols;
    Copy<E, PKC, S::BM, S::kWaves, false, ASYNC> cp;
    Copy<E, QKC, S::BN, S::kWaves, PASS == kGate, ASYNC> cq;
    cp.set(d.ldp, m0, PKC ? d.M : d.m_load, w, l);
    cq.set(d.ldq, n0, QKC ? d.N : d.n_load, w, l);
    const LaneRead<E, PKC> lp(l, wm * MB);
    const LaneRead<E, QKC> lq(l, wn * NB);
    f32x16 acc[NB][MB] = {};
    Frag<E> fp[2][MB], fq[2][NB];

    // whole tiles of k, over both segments; this workgroup's are [first, first + total)
    const int per_seg = d.K / kBk, all = per_seg * d.n_seg;
    const int first = static_cast<int>(static_cast<int64_t>(all) * part / d.n_split), total = static_cast<int>(static_cast<int64_t>(all) * (part + 1) / d.n_split) - first;
    const int64_t p_step = (PKC ? kBk : kBk * d.ldp) * static_cast<int64_t>(sizeof(E)), q_step = (QKC ? kBk : kBk * d.ldq) * static_cast<int64_t>(sizeof(E));
    auto p_base = [&](int seg) { return static_cast<const char*>(d.p[d.n_prod > 1 ? z : seg]) + (PKC ? m0 * d.ldp : m0) * static_cast<int64_t>(sizeof(E)); };
    auto q_base = [&](int seg) { return static_cast<const char*>(d.q[seg]) + (QKC ? n0 * d.ldq : n0) * static_cast<int64_t>(sizeof(E)); };
    // where an operand's next copies come from
    const int seg0 = d.n_seg > 1 && first >= per_seg ? 1 : 0;
    const char *pc = p_base(seg0) + (first - seg0 * per_seg) * p_step, *qc = q_base(seg0) + (first - seg0 * per_seg) * q_step;
    const char* qc2 = PASS == kGate ? q_base(1) + first * q_step : nullptr;
    int p_left = seg0 ? 0 : per_seg - first, q_left = p_left;  // tiles of the first segment not yet asked for
    constexpr int kP = decltype(cp)::PER, kQ = decltype(cq)::PER;
    auto copy_p = [&](auto J, int buf) { cp.template issue<decltype(J)::value>(pc, ptile + buf * kPB, w); };
    auto copy_q = [&](auto J, int buf) {
        const char* base = qc;
        if constexpr (PASS == kGate) base = (((w * kQ + decltype(J)::value) * 8) >> 5) & 1 ? qc2 : qc;
        cq.template issue<decltype(J)::value>(base, qtile + buf * kQB, w);
    };
    auto advance_p = [&] {
        pc += p_step;
        if (--p_left == 0 && d.n_seg > 1) pc = p_base(1);
    };
    auto advance_q = [&] {
        qc += q_step;
        if constexpr (PASS == kGate) qc2 += q_step;
        if (--q_left == 0 && d.n_seg > 1) qc = q_base(1);
    };
    using I0 = std::integral_constant<int, 0>;
    auto read = [&](auto R, auto SET, int pbuf, int qbuf, auto T) {  // the R-th operand of step T
        constexpr int r = decltype(R)::value, set = decltype(SET)::value, t = decltype(T)::value;
        if constexpr (r < NB) fq[set][r] = read_frag<E, QKC, r, t>(qtile + qbuf * kQB, lq);
        else fp[set][r - NB] = read_frag<E, PKC, r - NB, t>(ptile + pbuf * kPB, lp);
    };
    constexpr int kSteps = 4, kReads = MB + NB, kSlots = MB * NB;
    // f for each of [B, E) that stands in MFMA slot S
    auto in_slot = [&](auto S_, auto B_, auto E_, auto&& f) {
        constexpr int s = decltype(S_)::value, b = decltype(B_)::value, n = decltype(E_)::value - b;
        static_for<0, n>([&](auto I) {
            if constexpr (decltype(I)::value * kSlots / n == s) f(std::integral_constant<int, b + decltype(I)::value>{});
        });
    };
    using Reads = std::integral_constant<int, kReads>;
    using Ps = std::integral_constant<int, kP>;
    using Qs = std::integral_constant<int, kQ>;
    using HalfP = std::integral_constant<int, (kP + 1) / 2>;
    using HalfQ = std::integral_constant<int, (kQ + 1) / 2>;
    // One tile; `ahead`: how many there are behind it; q0, q1, q2: the buffers of Q of this tile, of the next one, and the one that is filled
    auto tile = [&](auto BUF, int ahead, int q0, int q1, int q2) {
        constexpr int buf = decltype(BUF)::value;
        static_for<0, kSteps>([&](auto T) {
            constexpr int t = decltype(T)::value, set = t & 1;
            using Set = std::integral_constant<int, set ^ 1>;
            if constexpr (t == kSteps - 1) {
                if constexpr (!ASYNC) {
                    __syncthreads();
                } else if constexpr (NBQ == 2) {
                    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                } else {  // the copies of Q of the tile after the next may be in flight
                    if (ahead >= 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kQ) : "memory");
                    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                }
            }
            static_for<0, kSlots>([&](auto S_) {
                constexpr int s = decltype(S_)::value;
                in_slot(S_, I0{}, Reads{}, [&](auto R) {
                    if constexpr (t < kSteps - 1) read(R, Set{}, buf, q0, std::integral_constant<int, t + 1>{});
                    else read(R, Set{}, buf ^ 1, q1, I0{});
                });
                if constexpr (!ASYNC && t == kSteps - 2) {
                    if (ahead >= 1) {
                        in_slot(S_, I0{}, Ps{}, [&](auto J) { cp.template put<decltype(J)::value>(ptile + (buf ^ 1) * kPB, w, l); });
                        in_slot(S_, I0{}, Qs{}, [&](auto J) { cq.template put<decltype(J)::value>(qtile + q1 * kQB, w, l); });
                    }
                }
                if constexpr (NBQ == 2) {
                    if constexpr (t == kSteps - 1)
                        if (ahead >= 2) {
                            in_slot(S_, I0{}, Ps{}, [&](auto J) { copy_p(J, buf); });
                            in_slot(S_, I0{}, Qs{}, [&](auto J) { copy_q(J, q2); });
                        }
                } else if constexpr (t == kSteps - 1) {
                    if (ahead >= 2) in_slot(S_, I0{}, HalfP{}, [&](auto J) { copy_p(J, buf); });
                } else if constexpr (t == 0) {
                    if (ahead >= 1) in_slot(S_, HalfP{}, Ps{}, [&](auto J) { copy_p(J, buf ^ 1); });
                } else if constexpr (t == 1) {
                    if (ahead >= 2) in_slot(S_, I0{}, HalfQ{}, [&](auto J) { copy_q(J, q2); });
                } else {
                    if (ahead >= 2) in_slot(S_, HalfQ{}, Qs{}, [&](auto J) { copy_q(J, q2); });
                }
                acc[s % NB][s / NB] = mfma(fq[set][s % NB], fp[set][s / NB], acc[s % NB][s / NB]);
                __builtin_amdgcn_sched_barrier(0);
            });
            if constexpr (NBQ == 3 && t == 0) {
                if (ahead >= 1) advance_p();
            } else if constexpr (NBQ == 3 && t == 2) {
                if (ahead >= 2) advance_q();
            } else if constexpr (NBQ == 2 && t == kSteps - 1) {
                if (ahead >= 2) {
                    advance_p();
                    advance_q();
                }
            }
        });
    };
    if (total > 0) {
        static_for<0, kP>([&](auto J) { copy_p(J, 0); });
        static_for<0, kQ>([&](auto J) { copy_q(J, 0); });
        advance_p();
        advance_q();
        if constexpr (!ASYNC) {
            static_for<0, kP>([&](auto J) { cp.template put<decltype(J)::value>(ptile, w, l); });
            static_for<0, kQ>([&](auto J) { cq.template put<decltype(J)::value>(qtile, w, l); });
        }
        if (total > 1) {
            static_for<0, kQ>([&](auto J) { copy_q(J, 1); });
            advance_q();
            static_for<0, NBQ == 3 ? HalfP::value : kP>([&](auto J) { copy_p(J, 1); });
            if constexpr (NBQ == 2) advance_p();
            if constexpr (ASYNC) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kQ + (NBQ == 3 ? HalfP::value : kP)) : "memory");
        } else {
            if constexpr (ASYNC) asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        }
        if constexpr (!ASYNC) __syncthreads();
        static_for<0, kReads>([&](auto R) { read(R, I0{}, 0, 0, I0{}); });
        int ahead = total - 1, q0 = 0, q1 = 1, q2 = NBQ - 1;
        auto turn = [&] {
            if constexpr (NBQ == 3) {
                const int q = q0;
                q0 = q1;
                q1 = q2;
                q2 = q;
            } else {
                q0 ^= 1;
                q1 ^= 1;
            }
            --ahead;
        };
        while (ahead >= 1) {
            tile(std::integral_constant<int, 0>{}, ahead, NBQ == 2 ? 0 : q0, NBQ == 2 ? 1 : q1, NBQ == 2 ? 0 : q2);
            turn();
            tile(std::integral_constant<int, 1>{}, ahead, NBQ == 2 ? 1 : q0, NBQ == 2 ? 0 : q1, NBQ == 2 ? 1 : q2);
            turn();
        }
        if (ahead == 0) tile(std::integral_constant<int, 0>{}, 0, NBQ == 2 ? 0 : q0, NBQ == 2 ? 1 : q1, NBQ == 2 ? 0 : q2);
    }
    // With both operands k-major and through registers the lane is asked for again: kept over the loop, it and what is made of it would spill
    constexpr bool kAskAgain = !ASYNC && !PKC && sizeof(E) == 2;
    int le = l, te = threadIdx.x;
    if constexpr (kAskAgain) {
        le = static_cast<int>(__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0)));
        te = 64 * w + le;
    }
    if (const int rest = per_seg * kBk; rest < d.K && part == d.n_split - 1) {  // what is left of k, zeros behind it
        for (int seg = 0; seg < d.n_seg; ++seg) {
            __syncthreads();
            for (int c = te; c < S::BM * 8; c += S::kThreads)
                *reinterpret_cast<uint4*>(ptile + chunk_off<E, PKC, S::BM>(c)) =
                    fetch<E, PKC, S::BM>(c, d.ldp, rest, d.K, m0, d.M, [&](int r) { return std::make_pair(d.p[d.n_prod > 1 ? z : seg], m0 + r); });
            for (int c = te; c < S::BN * 8; c += S::kThreads)
                *reinterpret_cast<uint4*>(qtile + chunk_off<E, QKC, S::BN>(c)) = fetch<E, QKC, S::BN>(c, d.ldq, rest, d.K, n0, d.N, [&](int r) {
                    if constexpr (PASS == kGate) return std::make_pair(d.q[(r >> 5) & 1], n0 + (r >> 6) * 32 + (r & 31));
                    else return std::make_pair(d.q[seg], n0 + r);
                });
            __syncthreads();
            static_for<0, kSteps>([&](auto T) {
                static_for<0, kReads>([&](auto R) { read(R, I0{}, 0, 0, T); });
                static_for<0, kSlots>([&](auto S_) {
                    constexpr int s = decltype(S_)::value;
                    acc[s % NB][s / NB] = mfma(fq[0][s % NB], fp[0][s / NB], acc[s % NB][s / NB]);
                });
            });
        }
    }
    if (PASS == kDact && d.n_split == 1) {
        // G and U of the wave's next block are asked for before this one's results are made.  Rows outside are read from inside and not
        // stored; so are whole groups of columns, and blocks that have none
        auto place = [&](int i, int& m, int& n, int& rows, int& cols) {
            m = m0 + (wm * MB + i / NB) * 32;
            n = n0 + (wn * NB + i % NB) * 32;
            rows = d.M - m;
            cols = d.N - n;
            return rows > 0 && cols > 0;
        };
        constexpr int kBlocks = MB * NB;
        Group g[2][2], u[2][2];
        auto ask = [&](int i, int set) {
            int m, n, rows, cols;
            if (!place(i, m, n, rows, cols)) return;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int c = min(16 * k + 8 * (le >> 5), (cols - 1) / 8 * 8);
                const int64_t from = (m + min(le & 31, rows - 1)) * d.ld_kept + n + c;
                g[set][k].get(d.G + from, cols - c);
                u[set][k].get(d.U + from, cols - c);
            }
        };
        ask(0, 0);
        static_for<0, kBlocks>([&](auto I) {
            constexpr int i = decltype(I)::value, set = i & 1;
            if constexpr (i + 1 < kBlocks) ask(i + 1, set ^ 1);
            int m, n, rows, cols;
            if (!place(i, m, n, rows, cols)) return;
            const Chunks x = chunks(acc[i % NB][i / NB]);
            Chunks dg, du;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float a, da;
                    act_grad<E, ACT>(g[set][k].w[j], a, da);
                    dg.c[k][j] = x.c[k][j] * u[set][k].w[j] * da;
                    du.c[k][j] = x.c[k][j] * a;
                }
            }
            const int64_t at = m * d.ldo + n;
            store_out<ASYNC>(static_cast<E*>(d.out[0]) + at, d.ldo, rows, cols, dg, le, d.odd);
            store_out<ASYNC>(static_cast<E*>(d.out[1]) + at, d.ldo, rows, cols, du, le, d.odd);
            __builtin_amdgcn_sched_barrier(0);
        });
        return;
    }
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int m = m0 + (wm * MB + mb) * 32, rows = d.M - m;
        if (rows <= 0) break;
        __builtin_amdgcn_sched_barrier(0);  // one block at a time: beside 128 accumulators there is no room for more
        if (d.n_split > 1) {  // this part's sums, as they are: kGate [part][gate, up], else [part][product] of M x ld_part
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int which = PASS == kGate ? nb : z, n = n0 + (PASS == kGate ? wn : wn * NB + nb) * 32, cols = d.N - n;
                if (cols <= 0) break;
                const int64_t at = ((static_cast<int64_t>(part) * (PASS == kGate ? 2 : d.n_prod) + which) * d.M + m) * d.ld_part + n;
                store_chunks<true>(d.parts + at, d.ld_part, rows, cols, chunks(acc[nb][mb]), le);
            }
        } else if constexpr (PASS == kGate) {
            const int n = n0 + wn * 32, cols = d.N - n;
            if (cols <= 0) break;
            const int64_t at = m * d.ldo + n;
            f32x16 h;
#pragma unroll
            for (int i = 0; i < 16; ++i) h[i] = act<E, ACT>(acc[0][mb][i]) * acc[1][mb][i];
            if (d.G) store_chunks<false>(d.G + at, d.ldo, rows, cols, chunks(acc[0][mb]), le);
            if (d.U) store_chunks<false>(d.U + at, d.ldo, rows, cols, chunks(acc[1][mb]), le);
            store_out<ASYNC>(static_cast<E*>(d.H) + at, d.ldo, rows, cols, chunks(h), le, d.odd);
        } else if constexpr (PASS == kPlain) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int n = n0 + (wn * NB + nb) * 32, cols = d.N - n;
                if (cols <= 0) break;
                store_out<ASYNC>(static_cast<E*>(d.out[d.n_prod > 1 ? z : 0]) + m * d.ldo + n, d.ldo, rows, cols, chunks(acc[nb][mb]), le, d.odd);
            }
        }
    }
}

template <typename E, bool ASYNC, bool PKC, bool QKC, Pass PASS, int ACT, typename S>
int launch_tiles(const Product& d, hipStream_t s) {
    constexpr int kCols = PASS == kGate ? S::BN / 2 : S::BN;
    const int64_t tn = (static_cast<int64_t>(d.N) + kCols - 1) / kCols, tm = (static_cast<int64_t>(d.M) + S::BM - 1) / S::BM;
    if (tn * tm >= (int64_t{1} << 31) / S::kThreads) return PSATTN_EUNSUPPORTED;  // 2^31 threads to a grid
    psattn_ffn_tiles<E, ASYNC, PKC, QKC, PASS, ACT, S><<<dim3(static_cast<uint32_t>(tn * tm), d.n_prod * d.n_split), S::kThreads, 0, s>>>(d, static_cast<int>(tm), static_cast<int>(tn));
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

template <typename E, bool ASYNC, bool PKC, bool QKC, Pass PASS, int ACT>
int launch_sized(TileSize size, const Product& d, hipStream_t s) {
    if constexpr (PKC) {
        if (size == k32) return launch_tiles<E, ASYNC, PKC, QKC, PASS, ACT, Shape<32, 128, 1, 2, 2>>(d, s);
        if (size == k64) return launch_tiles<E, ASYNC, PKC, QKC, PASS, ACT, Shape<64, 128, 1, 2, 2>>(d, s);
    }
    if (size == k256) return launch_tiles<E, ASYNC, PKC, QKC, PASS, ACT, Shape<256, 256, 2, 4, ASYNC ? 3 : 2>>(d, s);
    return launch_tiles<E, ASYNC, PKC, QKC, PASS, ACT, Shape<128, 128, 2, 2, ASYNC ? 3 : 2>>(d, s);
}

template <typename E, bool ASYNC>
int launch_product(Pass pass, int act, bool pkc, bool qkc, TileSize size, const Product& d, hipStream_t s) {
    if (pass == kGate) return act == PSATTN_ACT_SILU ? launch_sized<E, ASYNC, true, true, kGate, 0>(size, d, s) : launch_sized<E, ASYNC, true, true, kGate, 1>(size, d, s);
    if (pass == kDact) return act == PSATTN_ACT_SILU ? launch_sized<E, ASYNC, true, false, kDact, 0>(size, d, s) : launch_sized<E, ASYNC, true, false, kDact, 1>(size, d, s);
    if (pkc && qkc) return launch_sized<E, ASYNC, true, true, kPlain, 0>(size, d, s);
    if (pkc) return launch_sized<E, ASYNC, true, false, kPlain, 0>(size, d, s);
    return launch_sized<E, ASYNC, false, false, kPlain, 0>(size, d, s);
}

}  // namespace gemm
}  // namespace psattn
