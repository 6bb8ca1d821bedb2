// Layer norm over rows of `hidden` elements, with the residual sum in front of it, forward and backward.
//   S = X + R (rounded to the element type: the residual stream is held in it, and the backward reads it; S = X without R)
//   Y = (S - mean) rstd w + b, rstd = 1 / sqrt(mean((S - mean)^2) + eps)
//   with xh = (S - mean) rstd, q = dY w:  dX = rstd (q - mean(q) - xh mean(q xh)) + dS,  dw = sum_rows dY xh,  db = sum_rows dY
//
// Bound by HBM: each row is read once and stays in registers (16 bytes to a lane and load) between its sums and its result, in fp32.
// The sums run over the lanes in a tree of a fixed shape: a row's bits do not depend on the other rows.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "psattn.h"
#include "psattn_rows.h"

namespace {

using namespace psattn::rows;

__device__ __forceinline__ float hold(float v, const uint16_t*) { return __uint_as_float(psattn::mma::pack2(v, 0.f) << 16); }
__device__ __forceinline__ float hold(float v, const float*) { return v; }

// sums over LANES lanes, the same in each; `sm` (more than a wave): 16 N floats, another place for each call in flight
template <int LANES, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* sm) {
#pragma unroll
    for (int off = (LANES < 64 ? LANES : 64) / 2; off > 0; off >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], off);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) sm[(threadIdx.x >> 6) * N + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = sm[i];
#pragma unroll
            for (int w = 1; w < LANES / 64; ++w) v[i] += sm[w * N + i];
        }
    }
}

// A row to LANES lanes, PER groups of 16 bytes to each.  Rows of a wave and less share a workgroup of 256.
template <int LANES>
constexpr int kThreads = LANES < 256 ? 256 : LANES;

template <typename E, int LANES, int PER, bool WHOLE, bool RES>
__global__ __launch_bounds__(kThreads<LANES>) void psattn_ln_fwd(int n_rows, int hidden, float eps, const E* X, const E* R, const E* w, const E* b, E* S, E* Y,
                                                                 float* mean, float* rstd) {
    constexpr int V = kVec<E>, kAt = kThreads<LANES> / LANES;
    __shared__ float sm[2][16];
    const int row = blockIdx.x * kAt + threadIdx.x / LANES, lane = threadIdx.x % LANES;
    if (row >= n_rows) return;
    const size_t at = static_cast<size_t>(row) * hidden;
    const int from = lane * V - (WHOLE ? 0 : misalignment(X + at));  // this lane's first column
    float x[PER][V];
    float sum[1] = {0.f};
    u32x4 xr[PER], rr[RES ? PER : 1];
    Place pl[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        pl[p] = place<WHOLE, E>(from + p * LANES * V, hidden);
        xr[p] = raw<WHOLE>(X + at, pl[p], hidden);
        if constexpr (RES) rr[p] = raw<WHOLE>(R + at, pl[p], hidden);
    }
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        unpack(settled<WHOLE>(xr[p], pl[p].down), x[p]);
        if constexpr (RES) {
            float r[V];
            unpack(settled<WHOLE>(rr[p], pl[p].down), r);
#pragma unroll
            for (int j = 0; j < V; ++j) x[p][j] = hold(x[p][j] + r[j], X);
            store<WHOLE>(S + at, from + p * LANES * V, hidden, x[p]);
        }
    }
#pragma unroll
    for (int p = 0; p < PER; ++p)
#pragma unroll
        for (int j = 0; j < V; ++j) sum[0] += x[p][j];
    group_sum<LANES>(sum, sm[0]);
    const float mu = sum[0] / hidden;
    float sq[1] = {0.f};
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int c = from + p * LANES * V;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            x[p][j] -= mu;
            if (WHOLE ? c < hidden : c + j >= 0 && c + j < hidden) sq[0] += x[p][j] * x[p][j];
        }
    }
    group_sum<LANES>(sq, sm[1]);
    const float rs = 1.f / sqrtf(sq[0] / hidden + eps);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int c = from + p * LANES * V;
        float wv[V], bv[V] = {};
        unpack(settled<WHOLE>(raw<WHOLE>(w, pl[p], hidden), pl[p].down), wv);
        if (b) unpack(settled<WHOLE>(raw<WHOLE>(b, pl[p], hidden), pl[p].down), bv);
#pragma unroll
        for (int j = 0; j < V; ++j) x[p][j] = x[p][j] * rs * wv[j] + bv[j];
        store<WHOLE>(Y + at, c, hidden, x[p]);
    }
    if (lane == 0) {
        mean[row] = mu;
        rstd[row] = rs;
    }
}

// Backward.  A workgroup takes the rows from blockIdx.x on, gridDim.x apart, and keeps its lanes' columns of dw and db in registers;
// they go to part[workgroup] at its end and are joined by psattn_ln_weights (rows that share a workgroup add up in LDS first).
// Rows stay in the registers as they came and are unpacked twice, which leaves room for the next row's loads while one is
// summed over the lanes (8 334 rows of 4 096 bf16 with dS 105 -> 70 us, 65 536 of 1 024 198 -> 84).
//   Without SUMS a workgroup has one row, and dw and db are left to psattn_ln_columns: 32 columns to a lane and their sums do not
// fit beside a row (20 000 rows of 16 384 bf16, sums in registers and in part spilled 665 - 1 650 us, apart 616).
template <typename E, int LANES, int PER, bool WHOLE, bool SUMS>
__global__ __launch_bounds__(kThreads<LANES>) void psattn_ln_bwd(int n_rows, int hidden, const E* S, const E* w, const float* mean, const float* rstd, const E* dY,
                                                                 const E* dS, E* dX, float* part) {
    constexpr int V = kVec<E>, kAt = kThreads<LANES> / LANES;  // rows at a time
    __shared__ float sm[2][32];
    __shared__ float add[kAt > 1 ? kAt * LANES * PER * V : 1];
    static_assert(SUMS || kAt == 1, "short rows' columns are summed here");
    const int lane = threadIdx.x % LANES, own = threadIdx.x / LANES;
    float dw[PER][V] = {}, db[PER][V] = {};
    u32x4 xr[PER], gr[PER], sr[PER];
    float mu = 0.f, rs = 0.f;
    constexpr bool kAhead = SUMS;
    const int step = gridDim.x * kAt;
    int row = blockIdx.x * kAt + own;
    // this lane's first column: the same for all its rows, whose misalignment has to be
    const int from = lane * V - (WHOLE || (step % V != 0 && hidden % V != 0) || row >= n_rows ? 0 : misalignment(S + static_cast<size_t>(row) * hidden));
    Place pl[PER];
    u32x4 wr[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        pl[p] = place<WHOLE, E>(from + p * LANES * V, hidden);
        wr[p] = settled<WHOLE>(raw<WHOLE>(w, pl[p], hidden), pl[p].down);
    }
    auto fetch = [&](int r, u32x4 (&a)[PER], u32x4 (&b)[PER], u32x4 (&c)[PER], float& m, float& q) {
        const size_t at = static_cast<size_t>(r) * hidden;
        m = mean[r];
        q = rstd[r];
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            a[p] = raw<WHOLE>(S + at, pl[p], hidden);
            b[p] = raw<WHOLE>(dY + at, pl[p], hidden);
            if (dS) c[p] = raw<WHOLE>(dS + at, pl[p], hidden);
        }
    };
    if (kAhead && row < n_rows) fetch(row, xr, gr, sr, mu, rs);
    for (int turn = 0; row < n_rows; row += step, turn ^= 1) {
        u32x4 xn[PER], gn[PER], sn[PER];
        float mn = 0.f, qn = 0.f;
        if constexpr (!kAhead) fetch(row, xr, gr, sr, mu, rs);
        else if (row + step < n_rows) fetch(row + step, xn, gn, sn, mn, qn);
        float s[2] = {0.f, 0.f};
        // behind the row's end dY and w are zeros
        auto unpacked = [&](int p, float (&x)[V], float (&g)[V], float (&wv)[V]) {
            unpack(settled<WHOLE>(xr[p], pl[p].down), x);
            unpack(settled<WHOLE>(gr[p], pl[p].down), g);
            unpack(wr[p], wv);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = (x[j] - mu) * rs;
        };
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            float x[V], g[V], wv[V];
            unpacked(p, x, g, wv);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if constexpr (SUMS) {
                    dw[p][j] += g[j] * x[j];
                    db[p][j] += g[j];
                }
                g[j] *= wv[j];
                s[0] += g[j];
                s[1] += g[j] * x[j];
            }
        }
        group_sum<LANES>(s, sm[turn]);
        const float m1 = s[0] / hidden, m2 = s[1] / hidden;
        const size_t at = static_cast<size_t>(row) * hidden;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            float x[V], g[V], wv[V], o[V] = {};
            unpacked(p, x, g, wv);
            if (dS) unpack(settled<WHOLE>(sr[p], pl[p].down), o);
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] += rs * (g[j] * wv[j] - m1 - x[j] * m2);
            store<WHOLE>(dX + at, from + p * LANES * V, hidden, o);
        }
        if constexpr (!SUMS) return;  // its one row: nothing is kept for another
        if constexpr (kAhead) {
#pragma unroll
            for (int p = 0; p < PER; ++p) { xr[p] = xn[p]; gr[p] = gn[p]; sr[p] = sn[p]; }
            mu = mn;
            rs = qn;
        }
    }
    if constexpr (!SUMS) return;
    float* const mine = part + 2 * static_cast<size_t>(blockIdx.x) * hidden;
    auto out = [&](float* to, const float (&v)[PER][V]) {
        float* const at = kAt > 1 ? add + own * LANES * PER * V : to;  // rows that share the workgroup: by column, then added up
        if constexpr (kAt > 1) {
            __syncthreads();
        }
#pragma unroll
        for (int p = 0; p < PER; ++p)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = from + p * LANES * V + j;
                if (c >= 0 && c < hidden) at[c] = v[p][j];
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
    out(mine, dw);
    out(mine + hidden, db);
}

// dw and db from the workgroups' parts: 64 of their 2 hidden columns to a workgroup, sixteen lanes to a column
__global__ __launch_bounds__(1024) void psattn_ln_weights(int n_parts, int hidden, const float* part, void* dw, void* db, int bf16) {
    __shared__ float sm[16][65];
    const int c = threadIdx.x & 63, k = threadIdx.x >> 6;
    const int64_t i = blockIdx.x * 64 + c, width = 2 * static_cast<int64_t>(hidden);
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (i < width) {
        int p = k;
        for (; p + 48 < n_parts; p += 64)
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] += part[(p + 16 * u) * width + i];
        for (; p < n_parts; p += 16) v[0] += part[p * width + i];
    }
    sm[k][c] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    if (k > 0 || i >= width) return;
    float t = 0.f;
#pragma unroll
    for (int o = 0; o < 16; ++o) t += sm[o][c];
    void* const to = i < hidden ? dw : db;
    const int64_t at = i < hidden ? i : i - hidden;
    if (!to) return;
    if (bf16) store1(static_cast<uint16_t*>(to) + at, t);
    else store1(static_cast<float*>(to) + at, t);
}

// ---- rows too wide for registers: read again for each step
template <typename E>
__global__ __launch_bounds__(1024) void psattn_ln_fwd_wide(int hidden, float eps, const E* X, const E* R, const E* w, const E* b, E* S, E* Y, float* mean,
                                                           float* rstd) {
    constexpr int V = kVec<E>, kStep = 1024 * V;
    __shared__ float sm[2][16];
    const size_t at = static_cast<size_t>(blockIdx.x) * hidden;
    const E* x = X + at;
    float sum[1] = {0.f}, sq[1] = {0.f};
    for (int c = threadIdx.x * V; c < hidden; c += kStep) {
        float v[V];
        load<false>(x, c, hidden, v);
        if (R) {
            float r[V];
            load<false>(R + at, c, hidden, r);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = hold(v[j] + r[j], x);
            store<false>(S + at, c, hidden, v);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sum[0] += v[j];
    }
    if (R) x = S + at;  // each lane reads back what it wrote
    group_sum<1024>(sum, sm[0]);
    const float mu = sum[0] / hidden;
    for (int c = threadIdx.x * V; c < hidden; c += kStep) {
        float v[V];
        load<false>(x, c, hidden, v);
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (c + j < hidden) sq[0] += (v[j] - mu) * (v[j] - mu);
    }
    group_sum<1024>(sq, sm[1]);
    const float rs = 1.f / sqrtf(sq[0] / hidden + eps);
    for (int c = threadIdx.x * V; c < hidden; c += kStep) {
        float v[V], wv[V], bv[V] = {};
        load<false>(x, c, hidden, v);
        load<false>(w, c, hidden, wv);
        if (b) load<false>(b, c, hidden, bv);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (v[j] - mu) * rs * wv[j] + bv[j];
        store<false>(Y + at, c, hidden, v);
    }
    if (threadIdx.x == 0) {
        mean[blockIdx.x] = mu;
        rstd[blockIdx.x] = rs;
    }
}

template <typename E>
__global__ __launch_bounds__(1024) void psattn_ln_bwd_wide(int hidden, const E* S, const E* w, const float* mean, const float* rstd, const E* dY, const E* dS, E* dX) {
    constexpr int V = kVec<E>, kStep = 1024 * V;
    __shared__ float sm[32];
    const size_t at = static_cast<size_t>(blockIdx.x) * hidden;
    const float mu = mean[blockIdx.x], rs = rstd[blockIdx.x];
    float s[2] = {0.f, 0.f};
    for (int c = threadIdx.x * V; c < hidden; c += kStep) {
        float x[V], g[V], wv[V];
        load<false>(S + at, c, hidden, x);
        load<false>(dY + at, c, hidden, g);
        load<false>(w, c, hidden, wv);
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (c + j < hidden) {
                s[0] += g[j] * wv[j];
                s[1] += g[j] * wv[j] * ((x[j] - mu) * rs);
            }
    }
    group_sum<1024>(s, sm);
    const float m1 = s[0] / hidden, m2 = s[1] / hidden;
    for (int c = threadIdx.x * V; c < hidden; c += kStep) {
        float x[V], g[V], wv[V], o[V] = {};
        load<false>(S + at, c, hidden, x);
        load<false>(dY + at, c, hidden, g);
        load<false>(w, c, hidden, wv);
        if (dS) load<false>(dS + at, c, hidden, o);
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] += rs * (g[j] * wv[j] - m1 - (x[j] - mu) * rs * m2);
        store<false>(dX + at, c, hidden, o);
    }
}

// part[y]: sums of kVec columns to a lane over rows y, y + gridDim.y, ...
template <typename E>
__global__ __launch_bounds__(256) void psattn_ln_columns(int n_rows, int hidden, const E* S, const float* mean, const float* rstd, const E* dY, float* part) {
    constexpr int V = kVec<E>, kAtOnce = 4;
    const int step = gridDim.y;
    const bool same = step % V == 0 || hidden % V == 0;  // all rows of this workgroup start alike
    const int c = (blockIdx.x * 256 + threadIdx.x) * V - (same ? misalignment(S + static_cast<size_t>(blockIdx.y) * hidden) : 0);
    if (c >= hidden) return;
    const Place pl = place<false, E>(c, hidden);
    float w[V] = {}, b[V] = {};
    auto add = [&](const u32x4& s, const u32x4& d, float mu, float rs) {
        float x[V], g[V];
        unpack(settled<false>(s, pl.down), x);
        unpack(settled<false>(d, pl.down), g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            w[j] += g[j] * ((x[j] - mu) * rs);
            b[j] += g[j];
        }
    };
    int r = blockIdx.y;
    for (; r + (kAtOnce - 1) * step < n_rows; r += kAtOnce * step) {
        u32x4 s[kAtOnce], d[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const size_t at = static_cast<size_t>(r + u * step) * hidden;
            s[u] = raw<false>(S + at, pl, hidden);
            d[u] = raw<false>(dY + at, pl, hidden);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) add(s[u], d[u], mean[r + u * step], rstd[r + u * step]);
    }
    for (; r < n_rows; r += step) {
        const size_t at = static_cast<size_t>(r) * hidden;
        add(raw<false>(S + at, pl, hidden), raw<false>(dY + at, pl, hidden), mean[r], rstd[r]);
    }
    float* const mine = part + 2 * static_cast<size_t>(blockIdx.y) * hidden;
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (c + j >= 0 && c + j < hidden) {
            mine[c + j] = w[j];
            mine[hidden + c + j] = b[j];
        }
}

// ---- which kernel.  Rows of up to 32 groups of 16 bytes are sixteen lanes' (of 64, half or more would have nothing to do: 65 536 rows
// of 256 bf16 with R forward 40 us, 27 with sixteen), of up to 128 a wave's, wider ones a workgroup's.
template <typename E, bool BWD, typename F>
bool sized(int hidden, bool all, F&& f) {
    using std::integral_constant;
    auto go = [&](auto lanes, auto per) { return f(lanes, per), true; };
    const int64_t g = (static_cast<int64_t>(hidden) + kVec<E> - 1) / kVec<E> + (all ? 0 : 1);  // rows that start off a boundary reach into one more
    constexpr int kWidest = 4 * 8 / kVec<E>;  // groups of a lane: 32 columns
    using One = integral_constant<int, 1>;
    using Two = integral_constant<int, 2>;
    if (g <= 16) return go(integral_constant<int, 16>{}, One{});
    if (g <= 32) return go(integral_constant<int, 16>{}, Two{});
    if (g <= 64) return go(integral_constant<int, 64>{}, One{});
    if (g <= 128) return go(integral_constant<int, 64>{}, Two{});
    if (g <= 256) return go(integral_constant<int, 256>{}, One{});
    if (g <= 512) return go(integral_constant<int, 256>{}, Two{});
    if (g <= 768 && (all || !BWD)) return go(integral_constant<int, 256>{}, integral_constant<int, 3>{});  // ... at 1.7 TB/s instead of 2.1 where rows start anywhere
    if (g <= 1024) return go(integral_constant<int, 512>{}, Two{});
    if constexpr (BWD) {
        if (g <= 2048) return go(integral_constant<int, 512>{}, integral_constant<int, 4>{});
        if (g <= 512 * kWidest) return go(integral_constant<int, 512>{}, integral_constant<int, kWidest>{});
    } else {
        if (g <= 2048) return go(integral_constant<int, 1024>{}, Two{});
        if (g <= 512 * kWidest) return go(integral_constant<int, 1024>{}, integral_constant<int, kWidest / 2>{});
    }
    return false;
}

// workgroups of the backward, each with a part of dw and db.  A part is written and read in fp32, and costs as much memory time
// as some five rows of bf16: one for 26 rows, but 256 of them (one to a CU) at least and 1 024 at most
int n_parts(int32_t n_rows) { return std::max(1, std::min({n_rows, 1024, std::max(256, n_rows / 26)})); }

bool bad_shape(int32_t dt, int32_t n_rows, int32_t hidden) { return (dt != PSATTN_F32 && dt != PSATTN_BF16) || n_rows < 0 || hidden <= 0; }

template <typename E>
void fwd(int32_t n_rows, int32_t hidden, float eps, const void* X_, const void* R_, const void* w_, const void* b_, void* S_, void* Y_, float* mean,
         float* rstd, hipStream_t s) {
    const E *X = static_cast<const E*>(X_), *R = static_cast<const E*>(R_), *w = static_cast<const E*>(w_), *b = static_cast<const E*>(b_);
    E *S = static_cast<E*>(S_), *Y = static_cast<E*>(Y_);
    const bool all = whole<E>(hidden, {X, R, w, b, S, Y});
    const bool done = sized<E, false>(hidden, all, [&](auto lanes, auto per) {
        constexpr int L = decltype(lanes)::value, PER = decltype(per)::value, kAt = kThreads<L> / L;
        const int grid = (n_rows + kAt - 1) / kAt;
        auto go = [&](auto kernel) { kernel<<<grid, kThreads<L>, 0, s>>>(n_rows, hidden, eps, X, R, w, b, S, Y, mean, rstd); };
        if (R) all ? go(psattn_ln_fwd<E, L, PER, true, true>) : go(psattn_ln_fwd<E, L, PER, false, true>);
        else all ? go(psattn_ln_fwd<E, L, PER, true, false>) : go(psattn_ln_fwd<E, L, PER, false, false>);
    });
    if (!done) psattn_ln_fwd_wide<E><<<n_rows, 1024, 0, s>>>(hidden, eps, X, R, w, b, S, Y, mean, rstd);
}

template <typename E>
void bwd(int32_t n_rows, int32_t hidden, const void* S_, const void* w_, const float* mean, const float* rstd, const void* dY_, const void* dS_, void* dX_,
         void* dw, void* db, float* part, hipStream_t s) {
    const E *S = static_cast<const E*>(S_), *w = static_cast<const E*>(w_), *dY = static_cast<const E*>(dY_), *dS = static_cast<const E*>(dS_);
    E* dX = static_cast<E*>(dX_);
    int np = n_rows > 0 ? n_parts(n_rows) : 0;
    if (n_rows > 0) {
        const bool all = whole<E>(hidden, {S, w, dY, dS, dX});
        bool sums = false;
        const bool done = sized<E, true>(hidden, all, [&](auto lanes, auto per) {
            constexpr int L = decltype(lanes)::value, PER = decltype(per)::value, kAt = kThreads<L> / L;
            constexpr bool SUMS = PER * kVec<E> < 32;  // up to 1 024 groups of bf16, 2 048 of fp32
            if (SUMS) np = std::min(np, (n_rows + kAt - 1) / kAt);
            if (np > 8) np -= np % 8;  // a workgroup's rows start alike
            sums = SUMS;
            auto go = [&](auto kernel) { kernel<<<SUMS ? np : n_rows, kThreads<L>, 0, s>>>(n_rows, hidden, S, w, mean, rstd, dY, dS, dX, part); };
            if constexpr (L == 256 && PER == 3) go(psattn_ln_bwd<E, L, PER, true, SUMS>);  // whole rows alone: `sized`
            else all ? go(psattn_ln_bwd<E, L, PER, true, SUMS>) : go(psattn_ln_bwd<E, L, PER, false, SUMS>);
        });
        if (!done) psattn_ln_bwd_wide<E><<<n_rows, 1024, 0, s>>>(hidden, S, w, mean, rstd, dY, dS, dX);
        if (!sums) {
            const int cols = (hidden + kVec<E> - 1 + 256 * kVec<E> - 1) / (256 * kVec<E>);
            np = std::min(np, std::max(8, 2048 / cols / 8 * 8));  // eight workgroups to a CU
            psattn_ln_columns<E><<<dim3(cols, np), 256, 0, s>>>(n_rows, hidden, S, mean, rstd, dY, part);
        }
    }
    psattn_ln_weights<<<(2 * hidden + 63) / 64, 1024, 0, s>>>(np, hidden, part, dw, db, sizeof(E) == 2);
}

// grids of at most 2^31 threads: a row to 1 024 of them, or 64 columns of dw and db
constexpr int32_t kMostRows = (1 << 21) - 1, kMostHidden = 1 << 24;

}  // namespace

extern "C" {

int psattn_layernorm_fwd(int32_t dt, int32_t n_rows, int32_t hidden, float eps, const void* X, const void* R, const void* weight, const void* bias,
                         void* S, void* Y, float* mean, float* rstd, void* hip_stream) {
    if (bad_shape(dt, n_rows, hidden) || !(eps >= 0.f) || std::isinf(eps)) return PSATTN_EINVAL;
    if (n_rows == 0) return PSATTN_OK;
    if (!X || !weight || !Y || !mean || !rstd || (!R) != (!S)) return PSATTN_EINVAL;
    if (n_rows > kMostRows || hidden > kMostHidden) return PSATTN_EUNSUPPORTED;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dt == PSATTN_BF16) fwd<uint16_t>(n_rows, hidden, eps, X, R, weight, bias, S, Y, mean, rstd, s);
    else fwd<float>(n_rows, hidden, eps, X, R, weight, bias, S, Y, mean, rstd, s);
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

size_t psattn_layernorm_bwd_workspace_bytes(int32_t n_rows, int32_t hidden) {
    if (n_rows < 0 || hidden <= 0) return 0;
    return align_up(2 * sizeof(float) * static_cast<size_t>(n_parts(n_rows)) * hidden, 256) + 256;
}

int psattn_layernorm_bwd(int32_t dt, int32_t n_rows, int32_t hidden, const void* S, const void* weight, const float* mean, const float* rstd,
                         const void* dY, const void* dS, void* dX, void* dweight, void* dbias, void* workspace, size_t workspace_bytes,
                         void* hip_stream) {
    if (bad_shape(dt, n_rows, hidden) || !dweight) return PSATTN_EINVAL;
    if (n_rows > 0 && (!S || !weight || !mean || !rstd || !dY || !dX || !workspace)) return PSATTN_EINVAL;
    if (n_rows > 0 && workspace_bytes < psattn_layernorm_bwd_workspace_bytes(n_rows, hidden)) return PSATTN_EINVAL;
    if (n_rows > kMostRows || hidden > kMostHidden) return PSATTN_EUNSUPPORTED;
    float* const part = reinterpret_cast<float*>(align_up(reinterpret_cast<uintptr_t>(workspace), 256));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dt == PSATTN_BF16) bwd<uint16_t>(n_rows, hidden, S, weight, mean, rstd, dY, dS, dX, dweight, dbias, part, s);
    else bwd<float>(n_rows, hidden, S, weight, mean, rstd, dY, dS, dX, dweight, dbias, part, s);
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

}  // extern "C"
