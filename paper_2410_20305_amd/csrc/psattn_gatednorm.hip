// RMS norms before and after a part of a block, fused with its gate and residual scale, forward and backward.
//   N = B rb w_post, rb = 1 / sqrt(mean(B^2) + eps)                (N = B without w_post)
//   S = res X + g o N, rounded to the element type (the residual stream is held in it, and the backward reads it; S = X without B)
//   Y = S rs w_pre, rs = 1 / sqrt(mean(S^2) + eps)
// Backward, with bh = B rb, sh = S rs, q = dY w_pre, gw = g w_post:
//   t = dS + rs q,  m = mean(q sh),  ds = t - rs m sh;  dX = res ds;  dB = rb (ds gw - bh mean(ds gw bh))
//   dw_pre = sum_rows dY sh;  with C = sum_rows ds bh (of gates for all rows):  dw_post = g C, dg = w_post C
//                             with gates for each row:  dw_post = sum_rows g ds bh, dg = w_post ds bh
// mean(ds gw bh) = mean(t gw bh) - rs m mean(sh gw bh): the three sums of a row are taken together, in one pass over it.
//
// Bound by HBM: each row is read once and stays in registers (16 bytes to a lane and load) between its sums and its result, in fp32.
// 65 536 rows of 8 192 bf16 with a gate for each: forward 920 us (5.8 TB/s), backward 1 616 (5.3); 8 334 of 4 096 with one for all 52 and 90.
// The sums run over the lanes in a tree of a fixed shape: a row's bits do not depend on the other rows.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "psattn.h"
#include "psattn_rows.h"

namespace {

using namespace psattn::rows;

template <typename E>
struct Args {
    int32_t n_rows, hidden;
    float eps, res;
    const E *X, *B, *w_post, *gate, *w_pre;
    int32_t gate_step;  // elements from one row's gate to the next: hidden, or 0
    E *S, *Y;
    float *rstd_b, *rstd_s;
    // backward
    const E *dY, *dS;
    E *dX, *dB, *dgate;  // dgate: of gates for each row
    float *part, *row_m;
};

// Groups p of a row whose lanes take PER each: the first PER / 2 of them lie inside of it (`sized`), but for what lane 0 has before its start,
// so that only the first and those of the second half have an edge, on one side
template <bool WHOLE, int PER>
__device__ __forceinline__ u32x4 settled_at(const u32x4& x, int p, int down) {
    if (WHOLE || (PER > 1 && p > 0 && p < PER / 2)) return x;
    if (PER == 1) return settled<WHOLE>(x, down);
    return settled<WHOLE>(x, p == 0 ? min(down, 0) : max(down, 0));
}
template <bool WHOLE, int PER, typename E>
__device__ __forceinline__ void store_at(E* row, int p, int c, int hidden, const float (&x)[kVec<E>]) {
    if constexpr (WHOLE || PER == 1) {
        store<WHOLE>(row, c, hidden, x);
    } else if (p > 0 && p < PER / 2) {
        reinterpret_cast<Raw*>(row + c)->u = pack<E>(x);
    } else if (p == 0 ? c >= 0 : c + kVec<E> <= hidden) {
        reinterpret_cast<Raw*>(row + c)->u = pack<E>(x);
    } else {
#pragma unroll
        for (int j = 0; j < kVec<E>; ++j)
            if (p == 0 ? c + j >= 0 : c + j < hidden) store1(row + c + j, x[j]);
    }
}

// whether the lanes reach over a row that starts anywhere behind a 16-byte boundary: its groups are taken on such boundaries then.  Where they
// do not quite, groups off a boundary cost less than twice the lanes (20 000 rows of 4 095 bf16, forward and backward: 512 lanes 677 us, 256 389)
template <typename E>
__device__ __forceinline__ bool shifts(int hidden, int lanes, int per) {
    return hidden + kVec<E> - 1 <= lanes * per * kVec<E>;
}

template <typename E, int LANES, int PER, bool WHOLE>
__global__ __launch_bounds__(kThreads<LANES>, LANES * PER == 2048 ? 8 : 1) void psattn_gn_fwd(Args<E> a) {
    constexpr int V = kVec<E>, kAt = kThreads<LANES> / LANES;
    __shared__ float sm[2][16];
    const int row = blockIdx.x * kAt + threadIdx.x / LANES, lane = threadIdx.x % LANES, hidden = a.hidden;
    if (row >= a.n_rows) return;
    const size_t at = static_cast<size_t>(row) * hidden;
    const int from = lane * V - (WHOLE || !shifts<E>(hidden, LANES, PER) ? 0 : misalignment(a.X + at));  // this lane's first column
    u32x4 xr[PER], br[PER], gr[PER], wr[PER];
    Place pl[PER];
    const E* const gate = a.gate ? a.gate + static_cast<size_t>(row) * a.gate_step : nullptr;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        pl[p] = place<WHOLE, E>(from + p * LANES * V, hidden);
        xr[p] = raw<WHOLE>(a.X + at, pl[p], hidden);
        if (a.B) br[p] = raw<WHOLE>(a.B + at, pl[p], hidden);
        if (gate) gr[p] = raw<WHOLE>(gate, pl[p], hidden);
        if (a.w_post) wr[p] = raw<WHOLE>(a.w_post, pl[p], hidden);
    }
    float rb = 1.f;
    if (a.w_post) {
        float sq[1] = {0.f};
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            float b[V];
            unpack(settled<WHOLE>(br[p], pl[p].down), b);
#pragma unroll
            for (int j = 0; j < V; ++j) sq[0] += b[j] * b[j];
        }
        group_sum<LANES>(sq, sm[0]);
        rb = 1.f / sqrtf(sq[0] / hidden + a.eps);
    }
    float x[PER][V], sq[1] = {0.f};
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        unpack(settled<WHOLE>(xr[p], pl[p].down), x[p]);
        if (a.B) {
            float b[V], f[V];
            unpack(settled<WHOLE>(br[p], pl[p].down), b);
            if (a.w_post) {
                unpack(settled<WHOLE>(wr[p], pl[p].down), f);
#pragma unroll
                for (int j = 0; j < V; ++j) b[j] *= rb * f[j];
            }
            if (gate) {
                unpack(settled<WHOLE>(gr[p], pl[p].down), f);
#pragma unroll
                for (int j = 0; j < V; ++j) b[j] *= f[j];
            }
#pragma unroll
            for (int j = 0; j < V; ++j) x[p][j] = hold(fmaf(a.res, x[p][j], b[j]), a.X);
            store<WHOLE>(a.S + at, from + p * LANES * V, hidden, x[p]);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sq[0] += x[p][j] * x[p][j];
    }
    group_sum<LANES>(sq, sm[1]);
    const float rs = 1.f / sqrtf(sq[0] / hidden + a.eps);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        float w[V];
        unpack(settled<WHOLE>(raw<WHOLE>(a.w_pre, pl[p], hidden), pl[p].down), w);
#pragma unroll
        for (int j = 0; j < V; ++j) x[p][j] *= rs * w[j];
        store<WHOLE>(a.Y + at, from + p * LANES * V, hidden, x[p]);
    }
    if (lane == 0) {
        if (a.w_post) a.rstd_b[row] = rb;
        a.rstd_s[row] = rs;
    }
}

// Backward.  A workgroup takes the rows from blockIdx.x on, gridDim.x apart, and keeps its lanes' columns of dw_pre and C in registers;
// they go to part[workgroup] at its end and are joined by psattn_gn_weights (rows that share a workgroup add up in LDS first).
// Rows stay in the registers as they came and are unpacked twice, with room for the next row's loads while one is summed.  ALL: a gate
// for each row; else w_post and gate are one factor for all rows.  What there is not stands there as zeros or ones, without branches, and
// what the sums have unpacked is unpacked again for the results: kept, it spilled (65 536 x 8 192, a gate for each row: 3 670 us).
//   Rows of 32 columns to a lane keep the columns' sums in LDS, each lane its own (20 000 rows of 16 384 bf16, forward and backward: in a second pass
// over the rows 2 113 us, so 1 528).
template <typename E, int LANES, int PER, bool WHOLE, bool ALL>
__global__ __launch_bounds__(kThreads<LANES>) void psattn_gn_bwd(Args<E> a) {
    constexpr int V = kVec<E>, kAt = kThreads<LANES> / LANES;  // rows at a time
    constexpr bool kInLds = PER * V >= 32;
    __shared__ float4 columns[kInLds ? 2 * PER * (V / 4) * LANES : 1];  // [dw_pre, C][group][four of V][lane]
    __shared__ float sm[2][48];
    __shared__ float add[kAt > 1 ? kAt * LANES * PER * V : 1];
    const int lane = threadIdx.x % LANES, hidden = a.hidden, n_rows = a.n_rows;
    // rows of a wave and more are known to be: their addresses are scalar
    const int own = kAt == 1 ? 0 : LANES == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : static_cast<int>(threadIdx.x) / LANES;
    float sums[2][kInLds ? 1 : PER][V] = {};
    auto slot = [&](int which, int p, int q) -> float4& { return columns[((which * PER + p) * (V / 4) + q) * LANES + lane]; };
    if constexpr (kInLds) {
#pragma unroll
        for (int i = 0; i < 2 * PER * (V / 4); ++i) columns[i * LANES + lane] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    auto collect = [&](int which, int p, const float (&x)[V]) {  // a lane's own columns
        if constexpr (kInLds) {
#pragma unroll
            for (int q = 0; q < V / 4; ++q) {
                float4& to = slot(which, p, q);
                float4 s = to;
                s.x += x[4 * q], s.y += x[4 * q + 1], s.z += x[4 * q + 2], s.w += x[4 * q + 3];
                to = s;
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) sums[which][p][j] += x[j];
        }
    };
    constexpr bool kAhead = PER <= 2 && (WHOLE || !ALL || PER * V < 16);  // the next row's loads, where there are registers for them
    const int step = gridDim.x * kAt;
    int row = blockIdx.x * kAt + own;
    // this lane's first column: the same for all its rows, whose misalignment has to be
    const int from = lane * V - (WHOLE || !shifts<E>(hidden, LANES, PER) || (step % V != 0 && hidden % V != 0) || row >= n_rows ? 0 : misalignment(a.S + static_cast<size_t>(row) * hidden));
    // The weights' groups stay in registers, and with one factor for all rows so does its product of w_post and gate, in fp32.  Of rows of four
    // groups to a lane they are asked for again each time
    constexpr bool kKeep = PER <= 2;
    Place pl[PER];
    u32x4 w_pre[kKeep ? PER : 1], w_post[kKeep ? PER : 1];
    float both[kKeep && !ALL ? PER : 1][V];
    auto weight = [&](const E* w, int p) { return settled_at<WHOLE, PER>(raw<WHOLE>(w, pl[p], hidden), p, pl[p].down); };
    auto post = [&](int p) {
        float one[V];
#pragma unroll
        for (int j = 0; j < V; ++j) one[j] = 1.f;
        return a.w_post ? weight(a.w_post, p) : pack<E>(one);
    };
    auto times_gate = [&](int p, float (&f)[V]) {
        if (!a.gate) return;
        float g[V];
        unpack(weight(a.gate, p), g);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] *= g[j];
    };
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        pl[p] = place<WHOLE, E>(from + p * LANES * V, hidden);
        if constexpr (kKeep) {
            w_pre[p] = weight(a.w_pre, p);
            w_post[p] = post(p);
            if constexpr (!ALL) {
                unpack(w_post[p], both[p]);
                times_gate(p, both[p]);
            }
        }
    }
    struct Row {
        u32x4 s[PER], b[PER], dy[PER], ds[PER], g[ALL ? PER : 1];
        float rs, rb;
    } now = {}, next = {};
    auto fetch = [&](int r, Row& x) {
        const size_t at = static_cast<size_t>(r) * hidden;
        x.rs = a.rstd_s[r];
        x.rb = a.w_post ? a.rstd_b[r] : 1.f;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            x.s[p] = raw<WHOLE>(a.S + at, pl[p], hidden);
            x.dy[p] = raw<WHOLE>(a.dY + at, pl[p], hidden);
            if (a.B) x.b[p] = raw<WHOLE>(a.B + at, pl[p], hidden);
            if (a.dS) x.ds[p] = raw<WHOLE>(a.dS + at, pl[p], hidden);
            if constexpr (ALL) x.g[p] = raw<WHOLE>(a.gate + at, pl[p], hidden);
        }
    };
    if (kAhead && row < n_rows) fetch(row, now);
    for (int turn = 0; row < n_rows; row += step, turn ^= 1) {
        if constexpr (!kAhead) fetch(row, now);
        else if (row + step < n_rows) fetch(row + step, next);
        // a lane's values of one group; outside of the row s, b, dy and t are zeros
        float s[V], b[V], dy[V], t[V], g[V], f[V];
        auto unpacked = [&](int p, float (&q)[V]) {
            unpack(now.s[p], s);
            unpack(now.b[p], b);
            unpack(now.dy[p], dy);
            unpack(now.ds[p], t);
            if constexpr (ALL) unpack(now.g[p], g);
            if constexpr (kKeep) {
                unpack(w_pre[p], q);
                if constexpr (ALL) unpack(w_post[p], f);
            } else {
                unpack(weight(a.w_pre, p), q);
                unpack(post(p), f);
                if constexpr (!ALL) times_gate(p, f);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if constexpr (kKeep && !ALL) f[j] = both[p][j];
                q[j] *= dy[j];
                s[j] *= now.rs;
                b[j] *= now.rb;
                t[j] = fmaf(now.rs, q[j], t[j]);
            }
        };
        float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            float q[V], dw[V];
            if constexpr (!WHOLE) {
                const int down = pl[p].down;
                now.s[p] = settled_at<WHOLE, PER>(now.s[p], p, down);
                now.b[p] = settled_at<WHOLE, PER>(now.b[p], p, down);
                now.dy[p] = settled_at<WHOLE, PER>(now.dy[p], p, down);
                now.ds[p] = settled_at<WHOLE, PER>(now.ds[p], p, down);
                if constexpr (ALL) now.g[p] = settled_at<WHOLE, PER>(now.g[p], p, down);
            }
            unpacked(p, q);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                dw[j] = dy[j] * s[j];
                const float fb = (ALL ? g[j] * f[j] : f[j]) * b[j];
                sum[0] += q[j] * s[j];
                sum[1] += t[j] * fb;
                sum[2] += s[j] * fb;
            }
            collect(0, p, dw);
            __builtin_amdgcn_sched_barrier(0);
        }
        group_sum<LANES>(sum, sm[turn]);
        // what was unpacked for the sums is not kept for the results: the compiler would, and has no registers for it
#pragma unroll
        for (int p = 0; p < PER; ++p) asm volatile("" : "+v"(now.s[p]), "+v"(now.b[p]), "+v"(now.dy[p]), "+v"(now.ds[p]));
        if constexpr (ALL)
#pragma unroll
            for (int p = 0; p < PER; ++p) asm volatile("" : "+v"(now.g[p]));
        if constexpr (kKeep)
#pragma unroll
            for (int p = 0; p < PER; ++p) asm volatile("" : "+v"(w_pre[p]), "+v"(w_post[p]));
        const float m = now.rs * (sum[0] / hidden), mb = a.w_post ? (sum[1] - m * sum[2]) / hidden : 0.f, res = a.B ? a.res : 1.f;
        const size_t at = static_cast<size_t>(row) * hidden;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int c = from + p * LANES * V;
            float o[V];
            unpacked(p, o);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                t[j] = fmaf(-m, s[j], t[j]);
                o[j] = res * t[j];
            }
            store_at<WHOLE, PER>(a.dX + at, p, c, hidden, o);
            if (a.B) {
                float dc[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float tb = t[j] * b[j];
                    dc[j] = ALL ? g[j] * tb : tb;
                    o[j] = now.rb * (t[j] * (ALL ? g[j] * f[j] : f[j]) - b[j] * mb);
                    if constexpr (ALL) t[j] = f[j] * tb;
                }
                collect(1, p, dc);
                store_at<WHOLE, PER>(a.dB + at, p, c, hidden, o);
                if constexpr (ALL) store_at<WHOLE, PER>(a.dgate + at, p, c, hidden, t);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (kAhead) now = next;
    }
    float* const mine = a.part + 2 * static_cast<size_t>(blockIdx.x) * hidden;
    auto value = [&](int which, int p, int j) {
        if constexpr (kInLds) return reinterpret_cast<const float*>(&slot(which, p, j / 4))[j % 4];
        else return sums[which][p][j];
    };
    auto out = [&](float* to, int which) {
        float* const at = kAt > 1 ? add + own * LANES * PER * V : to;  // rows that share the workgroup: by column, then added up
        if constexpr (kAt > 1) __syncthreads();
#pragma unroll
        for (int p = 0; p < PER; ++p)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = from + p * LANES * V + j;
                if (c >= 0 && c < hidden) at[c] = value(which, p, j);
            }
        if constexpr (kAt > 1) {
            __syncthreads();
            for (int c = threadIdx.x; c < hidden; c += kThreads<LANES>) {
                float t = 0.f;
#pragma unroll
                for (int o = 0; o < kAt; ++o) t += add[o * LANES * PER * V + c];
                to[c] = t;
            }
        }
    };
    out(mine, 0);
    if (a.B) out(mine + hidden, 1);
}

// The weights' gradients from the workgroups' parts: 64 columns to a workgroup, sixteen lanes to a column; the first `hidden` are dw_pre,
// the others C
template <typename E>
__global__ __launch_bounds__(1024) void psattn_gn_weights(int n_parts, int hidden, const float* part, E* dw_pre, E* dw_post, E* dgate, const E* w_post, const E* gate) {
    __shared__ float sm[16][65];
    const int c = threadIdx.x & 63, k = threadIdx.x >> 6;
    const int64_t i = blockIdx.x * 64 + c, width = 2 * static_cast<int64_t>(hidden);
    const bool there = i < (dw_post || dgate ? width : hidden);
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (there) {
        int p = k;
        for (; p + 48 < n_parts; p += 64)
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] += part[(p + 16 * u) * width + i];
        for (; p < n_parts; p += 16) v[0] += part[p * width + i];
    }
    sm[k][c] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    if (k > 0 || !there) return;
    float t = 0.f;
#pragma unroll
    for (int o = 0; o < 16; ++o) t += sm[o][c];
    if (i < hidden) {
        store1(dw_pre + i, t);
    } else {
        const int64_t at = i - hidden;
        if (dw_post) store1(dw_post + at, gate ? to_f32(gate[at]) * t : t);
        if (dgate) store1(dgate + at, w_post ? to_f32(w_post[at]) * t : t);
    }
}

// ---- rows too wide for registers: read again for each step
template <typename E>
__global__ __launch_bounds__(1024) void psattn_gn_fwd_wide(Args<E> a) {
    constexpr int V = kVec<E>, kStep = 1024 * V;
    __shared__ float sm[2][16];
    const int hidden = a.hidden;
    const size_t at = static_cast<size_t>(blockIdx.x) * hidden;
    const E* const gate = a.gate ? a.gate + static_cast<size_t>(blockIdx.x) * a.gate_step : nullptr;
    const E* x = a.X + at;
    float rb = 1.f, sq[1] = {0.f};
    if (a.w_post) {
        for (int c = threadIdx.x * V; c < hidden; c += kStep) {
            float b[V];
            load<false>(a.B + at, c, hidden, b);
#pragma unroll
            for (int j = 0; j < V; ++j) sq[0] += b[j] * b[j];
        }
        group_sum<1024>(sq, sm[0]);
        rb = 1.f / sqrtf(sq[0] / hidden + a.eps);
        sq[0] = 0.f;
    }
    for (int c = threadIdx.x * V; c < hidden; c += kStep) {
        float v[V];
        load<false>(x, c, hidden, v);
        if (a.B) {
            float b[V], f[V];
            load<false>(a.B + at, c, hidden, b);
            if (a.w_post) {
                load<false>(a.w_post, c, hidden, f);
#pragma unroll
                for (int j = 0; j < V; ++j) b[j] *= rb * f[j];
            }
            if (gate) {
                load<false>(gate, c, hidden, f);
#pragma unroll
                for (int j = 0; j < V; ++j) b[j] *= f[j];
            }
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = hold(fmaf(a.res, v[j], b[j]), x);
            store<false>(a.S + at, c, hidden, v);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sq[0] += v[j] * v[j];
    }
    if (a.B) x = a.S + at;  // each lane reads back what it wrote
    group_sum<1024>(sq, sm[1]);
    const float rs = 1.f / sqrtf(sq[0] / hidden + a.eps);
    for (int c = threadIdx.x * V; c < hidden; c += kStep) {
        float v[V], w[V];
        load<false>(x, c, hidden, v);
        load<false>(a.w_pre, c, hidden, w);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] *= rs * w[j];
        store<false>(a.Y + at, c, hidden, v);
    }
    if (threadIdx.x == 0) {
        if (a.w_post) a.rstd_b[blockIdx.x] = rb;
        a.rstd_s[blockIdx.x] = rs;
    }
}

// A lane's values of one group of a row, and what comes of them
template <int V>
struct Group {
    float s[V], b[V], dy[V], t[V], g[V], wp[V];  // t: dS, then dS + rs q; g: gate; wp: w_post
};

// what the backward of one row reads at columns c ..
template <typename E>
__device__ __forceinline__ void group_at(const Args<E>& a, int row, float rs, float rb, int c, Group<kVec<E>>& x, float (&q)[kVec<E>]) {
    constexpr int V = kVec<E>;
    const size_t at = static_cast<size_t>(row) * a.hidden;
    load<false>(a.S + at, c, a.hidden, x.s);
    load<false>(a.dY + at, c, a.hidden, x.dy);
    load<false>(a.w_pre, c, a.hidden, q);
    if (a.dS) load<false>(a.dS + at, c, a.hidden, x.t);
    if (a.B) load<false>(a.B + at, c, a.hidden, x.b);
    if (a.gate) load<false>(a.gate + static_cast<size_t>(row) * a.gate_step, c, a.hidden, x.g);
    if (a.w_post) load<false>(a.w_post, c, a.hidden, x.wp);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        q[j] *= x.dy[j];
        x.s[j] *= rs;
        x.t[j] = fmaf(rs, q[j], a.dS ? x.t[j] : 0.f);
        x.b[j] = a.B ? x.b[j] * rb : 0.f;
        if (!a.gate) x.g[j] = 1.f;
        if (!a.w_post) x.wp[j] = 1.f;
    }
}

// Rows that are read twice, the second time from the caches: a row to a workgroup of 1 024.  COLUMNS: rows from blockIdx.x on, gridDim.x apart, of 16 384 columns at most, whose sums stand in LDS, each
// lane's own, and go to part[workgroup] at the end.  Else psattn_gn_columns makes them in a pass over
// the rows of its own (20 000 rows of 10 001 bf16 with a gate for each 1 673 us, 1 266 by LDS; 10 000 of 10 000 fp32 1 129, 759)
constexpr int kColumns = 16384;
template <typename E, bool COLUMNS>
__global__ __launch_bounds__(1024) void psattn_gn_bwd_wide(Args<E> a) {
    constexpr int V = kVec<E>, kStep = 1024 * V;
    __shared__ float sm[2][48];
    __shared__ float4 columns[COLUMNS ? 2 * kColumns / 4 : 1];  // [dw_pre, C][group][four of V][lane]
    const int hidden = a.hidden, step = gridDim.x;
    const bool shift = COLUMNS && hidden + V - 1 <= kColumns && (step % V == 0 || hidden % V == 0);  // all rows of this workgroup start alike
    const int from = static_cast<int>(threadIdx.x) * V - (shift ? misalignment(a.S + static_cast<size_t>(blockIdx.x) * hidden) : 0);
    auto slot = [&](int which, int c, int q) -> float4& { return columns[((which * (kColumns / kStep) + (c - from) / kStep) * (V / 4) + q) * 1024 + threadIdx.x]; };
    if constexpr (COLUMNS) {
#pragma unroll
        for (int i = 0; i < 2 * kColumns / 4096; ++i) columns[i * 1024 + threadIdx.x] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    auto collect = [&](int which, int c, const float (&x)[V]) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            float4& to = slot(which, c, q);
            float4 s = to;
            s.x += x[4 * q], s.y += x[4 * q + 1], s.z += x[4 * q + 2], s.w += x[4 * q + 3];
            to = s;
        }
    };
    Group<V> x;
    float q[V], o[V];
    int turn = 0;
    for (int row = blockIdx.x; row < a.n_rows; row += step, turn ^= 1) {
        const size_t at = static_cast<size_t>(row) * hidden;
        const float rs = a.rstd_s[row], rb = a.w_post ? a.rstd_b[row] : 1.f;
        float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll 1
        for (int c = from; c < hidden; c += kStep) {
            group_at(a, row, rs, rb, c, x, q);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float gwb = x.g[j] * x.wp[j] * x.b[j];
                sum[0] += q[j] * x.s[j];
                sum[1] += x.t[j] * gwb;
                sum[2] += x.s[j] * gwb;
                o[j] = x.dy[j] * x.s[j];
            }
            if constexpr (COLUMNS) collect(0, c, o);
        }
        group_sum<1024>(sum, sm[turn]);
        const float m = rs * (sum[0] / hidden), mb = (sum[1] - m * sum[2]) / hidden;
#pragma unroll 1
        for (int c = from; c < hidden; c += kStep) {
            group_at(a, row, rs, rb, c, x, q);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x.t[j] = fmaf(-m, x.s[j], x.t[j]);
                o[j] = a.B ? a.res * x.t[j] : x.t[j];
            }
            store<false>(a.dX + at, c, hidden, o);
            if (!a.B) continue;
            if constexpr (COLUMNS) {
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = (a.gate_step ? x.g[j] : 1.f) * (x.t[j] * x.b[j]);
                collect(1, c, o);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = x.t[j] * (x.g[j] * x.wp[j]);
                o[j] = a.w_post ? rb * (d - x.b[j] * mb) : d;
            }
            store<false>(a.dB + at, c, hidden, o);
            if (!a.dgate) continue;
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = x.wp[j] * (x.t[j] * x.b[j]);
            store<false>(a.dgate + at, c, hidden, o);
        }
        if (!COLUMNS && threadIdx.x == 0) a.row_m[row] = m;
    }
    if constexpr (COLUMNS) {
        float* const mine = a.part + 2 * static_cast<size_t>(blockIdx.x) * hidden;
        for (int c = from; c < hidden; c += kStep)
            for (int which = 0; which < (a.B ? 2 : 1); ++which)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (c + j >= 0 && c + j < hidden) mine[which * hidden + c + j] = reinterpret_cast<const float*>(&slot(which, c, j / 4))[j % 4];
    }
}

// part[y]: sums of kVec columns to a lane over rows y, y + gridDim.y, ...
template <typename E>
__global__ __launch_bounds__(256) void psattn_gn_columns(Args<E> a) {
    constexpr int V = kVec<E>;
    const int step = gridDim.y, hidden = a.hidden;
    const bool same = step % V == 0 || hidden % V == 0;  // all rows of this workgroup start alike
    const int c = (blockIdx.x * 256 + threadIdx.x) * V - (same ? misalignment(a.S + static_cast<size_t>(blockIdx.y) * hidden) : 0);
    if (c >= hidden) return;
    float w[V] = {}, k[V] = {};
    for (int r = blockIdx.y; r < a.n_rows; r += step) {
        Group<V> x;
        float q[V];
        const float m = a.row_m[r];
        group_at(a, r, a.rstd_s[r], a.w_post ? a.rstd_b[r] : 1.f, c, x, q);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            w[j] += x.dy[j] * x.s[j];
            const float t = fmaf(-m, x.s[j], x.t[j]) * x.b[j];
            k[j] += a.gate_step ? x.g[j] * t : t;
        }
    }
    float* const mine = a.part + 2 * static_cast<size_t>(blockIdx.y) * hidden;
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (c + j >= 0 && c + j < hidden) {
            mine[c + j] = w[j];
            mine[hidden + c + j] = k[j];
        }
}

// ---- which kernel: rows of up to 32 groups of 16 bytes are sixteen lanes', of up to 128 a wave's, wider ones a workgroup's
template <typename E, bool BWD, typename F>
bool sized(int hidden, bool all, F&& f) {
    using std::integral_constant;
    auto go = [&](auto lanes, auto per) { return f(lanes, per), true; };
    const int64_t g = (static_cast<int64_t>(hidden) + kVec<E> - 1) / kVec<E>;
    constexpr int kWidest = 4 * 8 / kVec<E>;  // groups of a lane: 32 columns
    using One = integral_constant<int, 1>;
    using Two = integral_constant<int, 2>;
    if (g <= 16) return go(integral_constant<int, 16>{}, One{});
    if (g <= 32) return go(integral_constant<int, 16>{}, Two{});
    if (g <= 64) return go(integral_constant<int, 64>{}, One{});
    if (g <= 128) return go(integral_constant<int, 64>{}, Two{});
    if (g <= 256) return go(integral_constant<int, 256>{}, One{});
    if (g <= 512) return go(integral_constant<int, 256>{}, Two{});
    if (g <= 1024) return go(integral_constant<int, 512>{}, Two{});
    if constexpr (BWD) {
        // bf16 off a boundary, and fp32 of eight groups to a lane, have no registers for a row: spilled / read twice, the backward of 20 000 rows of
        // 10 001 bf16 with a gate for each 1 896 / 1 266 us, of 10 000 rows of 10 000 fp32 1 018 / 759
        if (g <= 2048 && (all || sizeof(E) == 4)) return go(integral_constant<int, 512>{}, integral_constant<int, 4>{});
    } else {
        if (g <= 2048) return go(integral_constant<int, 1024>{}, Two{});
        if (g <= 512 * kWidest) return go(integral_constant<int, 1024>{}, integral_constant<int, kWidest / 2>{});
    }
    return false;
}

// Workgroups of the backward, each with a part of the columns' sums: as many as the chip has room for at once, 512 of 256 threads or 256 of
// 512, and 1 024 where rows are many.  A few more than fit wait for a second turn (8 334 rows of 4 096 bf16, forward and backward: 256
// workgroups 158 us, 320 the same, 512 147, 520 180, 1 024 159; 3 000 rows of 8 192: 256 106, 512 118, 1 024 151)
constexpr int kManyRows = 26 * 1024;
int n_parts(int32_t n_rows, int lanes) { return std::max(1, std::min(n_rows, n_rows >= kManyRows ? 1024 : lanes >= 512 ? 256 : 512)); }

// ... that a workspace has room for.  Rows wider than 16 384 have their columns summed apart, in fewer parts the wider they are
int most_parts(int32_t n_rows, int32_t hidden) {
    const int cols = (hidden + 2047) / 2048;  // of bf16
    return hidden <= 16384 ? n_parts(n_rows, 256) : std::min(n_parts(n_rows, 256), std::max(8, 2048 / cols / 8 * 8));
}

bool bad_shape(int32_t dt, int32_t n_rows, int32_t hidden) { return (dt != PSATTN_F32 && dt != PSATTN_BF16) || n_rows < 0 || hidden <= 0; }

template <typename E>
void fwd(const Args<E>& a, hipStream_t s) {
    const bool all = whole<E>(a.hidden, {a.X, a.B, a.w_post, a.gate, a.w_pre, a.S, a.Y});
    const bool done = sized<E, false>(a.hidden, all, [&](auto lanes, auto per) {
        constexpr int L = decltype(lanes)::value, PER = decltype(per)::value, kAt = kThreads<L> / L;
        auto go = [&](auto kernel) { kernel<<<(a.n_rows + kAt - 1) / kAt, kThreads<L>, 0, s>>>(a); };
        all ? go(psattn_gn_fwd<E, L, PER, true>) : go(psattn_gn_fwd<E, L, PER, false>);
    });
    if (!done) psattn_gn_fwd_wide<E><<<a.n_rows, 1024, 0, s>>>(a);
}

template <typename E>
void bwd(Args<E> a, bool vector_gate, void* dw_pre, void* dw_post, void* dgate, hipStream_t s) {
    int np = a.n_rows > 0 ? n_parts(a.n_rows, 256) : 0;
    if (a.n_rows > 0) {
        const bool all = whole<E>(a.hidden, {a.S, a.B, a.w_post, a.gate, a.w_pre, a.dY, a.dS, a.dX, a.dB, a.dgate});
        const bool done = sized<E, true>(a.hidden, all, [&](auto lanes, auto per) {
            constexpr int L = decltype(lanes)::value, PER = decltype(per)::value, kAt = kThreads<L> / L;
            np = std::min(n_parts(a.n_rows, L), (a.n_rows + kAt - 1) / kAt);
            if (np > 8) np -= np % 8;  // a workgroup's rows start alike
            auto go = [&](auto kernel) { kernel<<<np, kThreads<L>, 0, s>>>(a); };
            if constexpr (PER == 4 && sizeof(E) == 2) a.gate_step ? go(psattn_gn_bwd<E, L, PER, true, true>) : go(psattn_gn_bwd<E, L, PER, true, false>);  // `sized`
            else if (a.gate_step) all ? go(psattn_gn_bwd<E, L, PER, true, true>) : go(psattn_gn_bwd<E, L, PER, false, true>);
            else all ? go(psattn_gn_bwd<E, L, PER, true, false>) : go(psattn_gn_bwd<E, L, PER, false, false>);
        });
        if (!done && a.hidden <= kColumns) {
            np = std::min(a.n_rows, 256);  // one to a CU, whose LDS the sums fill
            if (np > 8) np -= np % 8;
            psattn_gn_bwd_wide<E, true><<<np, 1024, 0, s>>>(a);
        } else if (!done) {
            psattn_gn_bwd_wide<E, false><<<a.n_rows, 1024, 0, s>>>(a);
            const int cols = (a.hidden + kVec<E> - 1 + 256 * kVec<E> - 1) / (256 * kVec<E>);
            np = std::min(np, std::max(8, 2048 / cols / 8 * 8));  // eight workgroups to a CU
            psattn_gn_columns<E><<<dim3(cols, np), 256, 0, s>>>(a);
        }
    }
    E* const to_gate = vector_gate ? static_cast<E*>(dgate) : nullptr;
    psattn_gn_weights<E><<<((dw_post || to_gate ? 2 : 1) * a.hidden + 63) / 64, 1024, 0, s>>>(np, a.hidden, a.part, static_cast<E*>(dw_pre), static_cast<E*>(dw_post), to_gate,
                                                                                                np ? a.w_post : nullptr, np && vector_gate ? a.gate : nullptr);
}

// grids of at most 2^31 threads: a row to 1 024 of them, or 64 columns of the sums
constexpr int32_t kMostRows = (1 << 21) - 1, kMostHidden = 1 << 24;

template <typename E>
Args<E> make(int32_t n_rows, int32_t hidden, const void* B, const void* w_post, const void* gate, int32_t gate_rows, const void* w_pre, float* rstd_b, float* rstd_s) {
    Args<E> a{};
    a.n_rows = n_rows;
    a.hidden = hidden;
    a.B = static_cast<const E*>(B);
    a.w_post = static_cast<const E*>(w_post);
    a.gate = static_cast<const E*>(gate);
    a.gate_step = gate && gate_rows > 1 ? hidden : 0;
    a.w_pre = static_cast<const E*>(w_pre);
    a.rstd_b = rstd_b;
    a.rstd_s = rstd_s;
    return a;
}

// gates: none, one row for all, or as many rows as there are
bool bad_gate(const void* gate, int32_t gate_rows, int32_t n_rows) { return gate ? gate_rows != 1 && gate_rows != n_rows : gate_rows != 0; }

}  // namespace

extern "C" {

int psattn_gatednorm_fwd(int32_t dt, int32_t n_rows, int32_t hidden, float eps, float res_scale, const void* X, const void* B, const void* w_post, const void* gate,
                         int32_t gate_rows, const void* w_pre, void* S, void* Y, float* rstd_b, float* rstd_s, void* hip_stream) {
    if (bad_shape(dt, n_rows, hidden) || !(eps >= 0.f) || std::isinf(eps) || !std::isfinite(res_scale)) return PSATTN_EINVAL;
    if (n_rows == 0) return PSATTN_OK;
    if (!X || !w_pre || !Y || !rstd_s || bad_gate(gate, gate_rows, n_rows)) return PSATTN_EINVAL;
    if ((!B) != (!S) || (!B && (w_post || gate)) || (w_post && !rstd_b)) return PSATTN_EINVAL;
    if (n_rows > kMostRows || hidden > kMostHidden) return PSATTN_EUNSUPPORTED;
    auto go = [&](auto elem) {
        using E = decltype(elem);
        Args<E> a = make<E>(n_rows, hidden, B, w_post, gate, gate_rows, w_pre, rstd_b, rstd_s);
        a.eps = eps;
        a.res = res_scale;
        a.X = static_cast<const E*>(X);
        a.S = static_cast<E*>(S);
        a.Y = static_cast<E*>(Y);
        fwd(a, static_cast<hipStream_t>(hip_stream));
    };
    if (dt == PSATTN_BF16) go(uint16_t{});
    else go(float{});
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

size_t psattn_gatednorm_bwd_workspace_bytes(int32_t n_rows, int32_t hidden) {
    if (n_rows < 0 || hidden <= 0) return 0;
    return align_up(2 * sizeof(float) * static_cast<size_t>(most_parts(n_rows, hidden)) * hidden, 256) + align_up(sizeof(float) * static_cast<size_t>(n_rows), 256) + 256;
}

int psattn_gatednorm_bwd(int32_t dt, int32_t n_rows, int32_t hidden, float res_scale, const void* B, const void* w_post, const void* gate, int32_t gate_rows,
                         const void* w_pre, const void* S, const float* rstd_b, const float* rstd_s, const void* dY, const void* dS, void* dX, void* dB, void* dw_post,
                         void* dgate, void* dw_pre, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (bad_shape(dt, n_rows, hidden) || !std::isfinite(res_scale) || !dw_pre) return PSATTN_EINVAL;
    if (n_rows > 0 && (!S || !w_pre || !rstd_s || !dY || !dX || !workspace || bad_gate(gate, gate_rows, n_rows))) return PSATTN_EINVAL;
    if (n_rows > 0 && ((!B) != (!dB) || (!B && (w_post || gate)) || (w_post && !rstd_b) || (!w_post) != (!dw_post) || (!gate) != (!dgate))) return PSATTN_EINVAL;
    if (n_rows > 0 && workspace_bytes < psattn_gatednorm_bwd_workspace_bytes(n_rows, hidden)) return PSATTN_EINVAL;
    if (n_rows > kMostRows || hidden > kMostHidden) return PSATTN_EUNSUPPORTED;
    auto go = [&](auto elem) {
        using E = decltype(elem);
        Args<E> a = make<E>(n_rows, hidden, B, w_post, gate, gate_rows, w_pre, const_cast<float*>(rstd_b), const_cast<float*>(rstd_s));
        a.res = res_scale;
        a.S = static_cast<E*>(const_cast<void*>(S));
        a.dY = static_cast<const E*>(dY);
        a.dS = static_cast<const E*>(dS);
        a.dX = static_cast<E*>(dX);
        a.dB = static_cast<E*>(dB);
        const bool vector_gate = dgate && (n_rows == 0 ? gate_rows == 1 : a.gate_step == 0);
        a.dgate = vector_gate ? nullptr : static_cast<E*>(dgate);
        a.part = reinterpret_cast<float*>(align_up(reinterpret_cast<uintptr_t>(workspace), 256));
        a.row_m = a.part + align_up(2 * sizeof(float) * static_cast<size_t>(most_parts(n_rows, hidden)) * hidden, 256) / sizeof(float);
        bwd(a, vector_gate, dw_pre, dw_post, dgate, static_cast<hipStream_t>(hip_stream));
    };
    if (dt == PSATTN_BF16) go(uint16_t{});
    else go(float{});
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

}  // extern "C"
