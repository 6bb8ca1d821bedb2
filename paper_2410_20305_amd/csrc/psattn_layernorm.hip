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
#include <initializer_list>
#include <type_traits>

#include "psattn.h"
#include "psattn_gemm.h"

namespace {

using psattn::gemm::store1;
using psattn::gemm::to_f32;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

template <typename E>
constexpr int kVec = 16 / static_cast<int>(sizeof(E));

__device__ __forceinline__ void unpack(const u32x4& u, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(u[j] << 16);
        x[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const u32x4& u, float (&x)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(u[j]);
}
template <typename E>
__device__ __forceinline__ u32x4 pack(const float* x) {
    u32x4 u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(E) == 2) u[j] = psattn::mma::pack2(x[2 * j], x[2 * j + 1]);
        else u[j] = __float_as_uint(x[j]);
    }
    return u;
}
struct __attribute__((packed, aligned(2))) Raw {
    u32x4 u;
};

// kVec elements from column c of a row of `hidden`; zeros behind its end.  Rows may start anywhere: a group that is all there is one
// load whatever its address
template <bool WHOLE, typename E>
__device__ __forceinline__ void load(const E* row, int c, int hidden, float (&x)[kVec<E>]) {
    if constexpr (WHOLE) {
        if (c < hidden) unpack(*reinterpret_cast<const u32x4*>(row + c), x);
        else
#pragma unroll
            for (int j = 0; j < kVec<E>; ++j) x[j] = 0.f;
    } else if (c + kVec<E> <= hidden) {
        unpack(reinterpret_cast<const Raw*>(row + c)->u, x);
    } else {
#pragma unroll
        for (int j = 0; j < kVec<E>; ++j) x[j] = c + j < hidden ? to_f32(row[c + j]) : 0.f;
    }
}
template <bool WHOLE, typename E>
__device__ __forceinline__ void store(E* row, int c, int hidden, const float (&x)[kVec<E>]) {
    if constexpr (WHOLE) {
        if (c < hidden) *reinterpret_cast<u32x4*>(row + c) = pack<E>(x);
    } else if (c + kVec<E> <= hidden) {
        reinterpret_cast<Raw*>(row + c)->u = pack<E>(x);
    } else {
#pragma unroll
        for (int j = 0; j < kVec<E>; ++j)
            if (c + j < hidden) store1(row + c + j, x[j]);
    }
}
__device__ __forceinline__ float hold(float v, const uint16_t*) { return __uint_as_float(psattn::mma::pack2(v, 0.f) << 16); }
__device__ __forceinline__ float hold(float v, const float*) { return v; }

// sums over NW waves, the same in every lane; `sm`: N NW floats, another place for each call in flight
template <int NW, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* sm) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], off);
    if constexpr (NW > 1) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) sm[(threadIdx.x >> 6) * N + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = sm[i];
#pragma unroll
            for (int w = 1; w < NW; ++w) v[i] += sm[w * N + i];
        }
    }
}

// A row to a group of NW waves, PER groups of 16 bytes to a lane.  NW = 1: four rows to a workgroup.
template <int NW>
constexpr int kThreads = NW == 1 ? 256 : 64 * NW;

template <typename E, int NW, int PER, bool WHOLE, bool RES>
__global__ __launch_bounds__(kThreads<NW>) void psattn_ln_fwd(int n_rows, int hidden, float eps, const E* X, const E* R, const E* w, const E* b, E* S, E* Y,
                                                              float* mean, float* rstd) {
    constexpr int V = kVec<E>, kLanes = 64 * NW;
    __shared__ float sm[2][NW];
    const int row = NW == 1 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x, lane = threadIdx.x % kLanes;
    if (row >= n_rows) return;
    const size_t at = static_cast<size_t>(row) * hidden;
    float x[PER][V];
    float sum[1] = {0.f};
#pragma unroll
    for (int p = 0; p < PER; ++p) load<WHOLE>(X + at, (p * kLanes + lane) * V, hidden, x[p]);
    if constexpr (RES) {
        float r[PER][V];
#pragma unroll
        for (int p = 0; p < PER; ++p) load<WHOLE>(R + at, (p * kLanes + lane) * V, hidden, r[p]);
#pragma unroll
        for (int p = 0; p < PER; ++p) {
#pragma unroll
            for (int j = 0; j < V; ++j) x[p][j] = hold(x[p][j] + r[p][j], X);
            store<WHOLE>(S + at, (p * kLanes + lane) * V, hidden, x[p]);
        }
    }
#pragma unroll
    for (int p = 0; p < PER; ++p)
#pragma unroll
        for (int j = 0; j < V; ++j) sum[0] += x[p][j];
    group_sum<NW>(sum, sm[0]);
    const float mu = sum[0] / hidden;
    float sq[1] = {0.f};
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int c = (p * kLanes + lane) * V;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            x[p][j] -= mu;
            if (WHOLE ? c < hidden : c + j < hidden) sq[0] += x[p][j] * x[p][j];
        }
    }
    group_sum<NW>(sq, sm[1]);
    const float rs = 1.f / sqrtf(sq[0] / hidden + eps);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int c = (p * kLanes + lane) * V;
        float wv[V], bv[V] = {};
        load<WHOLE>(w, c, hidden, wv);
        if (b) load<WHOLE>(b, c, hidden, bv);
#pragma unroll
        for (int j = 0; j < V; ++j) x[p][j] = x[p][j] * rs * wv[j] + bv[j];
        store<WHOLE>(Y + at, c, hidden, x[p]);
    }
    if (lane == 0) {
        mean[row] = mu;
        rstd[row] = rs;
    }
}

// Backward.  A workgroup takes rows first, first + gridDim.x, ... and keeps its lanes' columns of dw and db in registers; they go to
// part[workgroup] at its end and are joined by psattn_ln_weights.  NW = 1: the four waves take rows of their own and add up in LDS.
template <typename E, int NW, int PER, bool WHOLE>
__global__ __launch_bounds__(kThreads<NW>) void psattn_ln_bwd(int n_rows, int hidden, const E* S, const E* w, const float* mean, const float* rstd, const E* dY,
                                                              const E* dS, E* dX, float* part) {
    constexpr int V = kVec<E>, kLanes = 64 * NW, kAt = NW == 1 ? 4 : 1;  // rows at a time
    __shared__ float sm[2][2 * NW];
    __shared__ float add[NW == 1 ? 3 * 64 * V : 1];
    const int lane = threadIdx.x % kLanes, own = NW == 1 ? threadIdx.x >> 6 : 0;
    float dw[PER][V] = {}, db[PER][V] = {}, wv[PER][V];
#pragma unroll
    for (int p = 0; p < PER; ++p) load<WHOLE>(w, (p * kLanes + lane) * V, hidden, wv[p]);
    int turn = 0;
    for (int row = blockIdx.x * kAt + own; row < n_rows; row += gridDim.x * kAt, turn ^= 1) {
        const size_t at = static_cast<size_t>(row) * hidden;
        const float mu = mean[row], rs = rstd[row];
        float x[PER][V], g[PER][V];
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            load<WHOLE>(S + at, (p * kLanes + lane) * V, hidden, x[p]);
            load<WHOLE>(dY + at, (p * kLanes + lane) * V, hidden, g[p]);
        }
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int p = 0; p < PER; ++p)
#pragma unroll
            for (int j = 0; j < V; ++j) {  // behind the row's end dY and w are zeros
                x[p][j] = (x[p][j] - mu) * rs;
                if constexpr (!WHOLE)
                    if ((p * kLanes + lane) * V + j >= hidden) x[p][j] = 0.f;
                dw[p][j] += g[p][j] * x[p][j];
                db[p][j] += g[p][j];
                g[p][j] *= wv[p][j];
                s[0] += g[p][j];
                s[1] += g[p][j] * x[p][j];
            }
        group_sum<NW>(s, sm[turn]);
        const float m1 = s[0] / hidden, m2 = s[1] / hidden;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int c = (p * kLanes + lane) * V;
            float o[V];
            if (dS) {
                load<WHOLE>(dS + at, c, hidden, o);
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] += rs * (g[p][j] - m1 - x[p][j] * m2);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = rs * (g[p][j] - m1 - x[p][j] * m2);
            }
            store<WHOLE>(dX + at, c, hidden, o);
        }
    }
    float* const mine = part + 2 * static_cast<size_t>(blockIdx.x) * hidden;
    auto out = [&](float* to, const float (&v)[PER][V]) {
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            float t[V];
#pragma unroll
            for (int j = 0; j < V; ++j) t[j] = v[p][j];
            if constexpr (NW == 1) {
                __syncthreads();
                if (own > 0)
#pragma unroll
                    for (int j = 0; j < V; ++j) add[((own - 1) * V + j) * 64 + lane] = t[j];
                __syncthreads();
                if (own > 0) continue;
#pragma unroll
                for (int o = 0; o < 3; ++o)
#pragma unroll
                    for (int j = 0; j < V; ++j) t[j] += add[(o * V + j) * 64 + lane];
            }
            const int c = (p * kLanes + lane) * V;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (c + j < hidden) to[c + j] = t[j];
        }
    };
    out(mine, dw);
    out(mine + hidden, db);
}

// dw and db from the workgroups' parts: 32 columns to a workgroup, eight lanes to a column
__global__ __launch_bounds__(256) void psattn_ln_weights(int n_parts, int hidden, const float* part, void* dw, void* db, int bf16) {
    __shared__ float sm[8][2][33];
    const int c = threadIdx.x & 31, k = threadIdx.x >> 5, i = blockIdx.x * 32 + c;
    float v[2] = {0.f, 0.f};
    if (i < hidden)
        for (int p = k; p < n_parts; p += 8) {
            v[0] += part[2 * static_cast<size_t>(p) * hidden + i];
            v[1] += part[(2 * static_cast<size_t>(p) + 1) * hidden + i];
        }
    sm[k][0][c] = v[0];
    sm[k][1][c] = v[1];
    __syncthreads();
    if (k > 1 || i >= hidden || (k == 1 && !db)) return;
    float t = 0.f;
    for (int o = 0; o < 8; ++o) t += sm[o][k][c];
    void* const to = k == 0 ? dw : db;
    if (bf16) store1(static_cast<uint16_t*>(to) + i, t);
    else store1(static_cast<float*>(to) + i, t);
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
    group_sum<16>(sum, sm[0]);
    const float mu = sum[0] / hidden;
    for (int c = threadIdx.x * V; c < hidden; c += kStep) {
        float v[V];
        load<false>(x, c, hidden, v);
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (c + j < hidden) sq[0] += (v[j] - mu) * (v[j] - mu);
    }
    group_sum<16>(sq, sm[1]);
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
    group_sum<16>(s, sm);
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

// part[y]: sums of one column over rows y, y + gridDim.y, ...
template <typename E>
__global__ __launch_bounds__(256) void psattn_ln_columns(int n_rows, int hidden, const E* S, const float* mean, const float* rstd, const E* dY, float* part) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= hidden) return;
    float w = 0.f, b = 0.f;
    for (int r = blockIdx.y; r < n_rows; r += gridDim.y) {
        const size_t at = static_cast<size_t>(r) * hidden + i;
        const float dy = to_f32(dY[at]);
        w += dy * ((to_f32(S[at]) - mean[r]) * rstd[r]);
        b += dy;
    }
    float* const mine = part + 2 * static_cast<size_t>(blockIdx.y) * hidden;
    mine[i] = w;
    mine[hidden + i] = b;
}

// ---- which kernel.  A row of up to 64 lanes' four loads is a wave's; wider ones a workgroup's, in up to two loads to a lane
// (dw, db and w of a lane's columns live in registers in the backward), up to 1 024 lanes.
constexpr int kMostWaves = 16, kMostPer = 2;
template <typename E>
constexpr int kWidest = 64 * kMostWaves * kMostPer * kVec<E>;

template <typename E, typename F>
bool sized(int hidden, F&& f) {
    auto go = [&](auto nw, auto per) { return f(nw, per), true; };
    const int g = (hidden + kVec<E> - 1) / kVec<E>;  // groups of 16 bytes
    using std::integral_constant;
    if (g <= 64) return go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    if (g <= 128) return go(integral_constant<int, 1>{}, integral_constant<int, 2>{});
    if (g <= 256) return go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    if (g <= 512) return go(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    if (g <= 1024) return go(integral_constant<int, 8>{}, integral_constant<int, 2>{});
    if (g <= 2048) return go(integral_constant<int, 16>{}, integral_constant<int, 2>{});
    return false;
}

// workgroups of the backward, each with a part of dw and db: four to a CU keep enough loads in flight, and their parts are small
// beside what they read; few rows have fewer
int n_parts(int32_t n_rows, int32_t hidden) { return std::max(1, std::min(n_rows, 1024)); }

bool bad_shape(int32_t dt, int32_t n_rows, int32_t hidden) { return (dt != PSATTN_F32 && dt != PSATTN_BF16) || n_rows < 0 || hidden <= 0; }

template <typename E>
bool whole(int32_t hidden, std::initializer_list<const void*> p) {
    uintptr_t a = 0;
    for (const void* x : p) a |= reinterpret_cast<uintptr_t>(x);
    return a % 16 == 0 && hidden % kVec<E> == 0;
}

template <typename E>
void fwd(int32_t n_rows, int32_t hidden, float eps, const void* X_, const void* R_, const void* w_, const void* b_, void* S_, void* Y_, float* mean,
         float* rstd, hipStream_t s) {
    const E *X = static_cast<const E*>(X_), *R = static_cast<const E*>(R_), *w = static_cast<const E*>(w_), *b = static_cast<const E*>(b_);
    E *S = static_cast<E*>(S_), *Y = static_cast<E*>(Y_);
    const bool all = whole<E>(hidden, {X, R, w, b, S, Y});
    const bool done = sized<E>(hidden, [&](auto nw, auto per) {
        constexpr int NW = decltype(nw)::value, PER = decltype(per)::value;
        const int grid = NW == 1 ? (n_rows + 3) / 4 : n_rows;
        auto go = [&](auto kernel) { kernel<<<grid, kThreads<NW>, 0, s>>>(n_rows, hidden, eps, X, R, w, b, S, Y, mean, rstd); };
        if (R) all ? go(psattn_ln_fwd<E, NW, PER, true, true>) : go(psattn_ln_fwd<E, NW, PER, false, true>);
        else all ? go(psattn_ln_fwd<E, NW, PER, true, false>) : go(psattn_ln_fwd<E, NW, PER, false, false>);
    });
    if (!done) psattn_ln_fwd_wide<E><<<n_rows, 1024, 0, s>>>(hidden, eps, X, R, w, b, S, Y, mean, rstd);
}

template <typename E>
void bwd(int32_t n_rows, int32_t hidden, const void* S_, const void* w_, const float* mean, const float* rstd, const void* dY_, const void* dS_, void* dX_,
         void* dw, void* db, float* part, hipStream_t s) {
    const E *S = static_cast<const E*>(S_), *w = static_cast<const E*>(w_), *dY = static_cast<const E*>(dY_), *dS = static_cast<const E*>(dS_);
    E* dX = static_cast<E*>(dX_);
    int np = n_rows > 0 ? n_parts(n_rows, hidden) : 0;
    if (n_rows > 0) {
        const bool all = whole<E>(hidden, {S, w, dY, dS, dX});
        const bool done = sized<E>(hidden, [&](auto nw, auto per) {
            constexpr int NW = decltype(nw)::value, PER = decltype(per)::value;
            if (NW == 1) np = (np + 3) / 4;
            auto go = [&](auto kernel) { kernel<<<np, kThreads<NW>, 0, s>>>(n_rows, hidden, S, w, mean, rstd, dY, dS, dX, part); };
            all ? go(psattn_ln_bwd<E, NW, PER, true>) : go(psattn_ln_bwd<E, NW, PER, false>);
        });
        if (!done) {
            np = std::min(np, 64);
            psattn_ln_bwd_wide<E><<<n_rows, 1024, 0, s>>>(hidden, S, w, mean, rstd, dY, dS, dX);
            psattn_ln_columns<E><<<dim3((hidden + 255) / 256, np), 256, 0, s>>>(n_rows, hidden, S, mean, rstd, dY, part);
        }
    }
    psattn_ln_weights<<<(hidden + 31) / 32, 256, 0, s>>>(np, hidden, part, dw, db, sizeof(E) == 2);
}

// grids of at most 2^31 threads: a row to 1 024 of them
constexpr int32_t kMostRows = (1 << 21) - 1;

}  // namespace

extern "C" {

int psattn_layernorm_fwd(int32_t dt, int32_t n_rows, int32_t hidden, float eps, const void* X, const void* R, const void* weight, const void* bias,
                         void* S, void* Y, float* mean, float* rstd, void* hip_stream) {
    if (bad_shape(dt, n_rows, hidden) || !(eps >= 0.f) || std::isinf(eps)) return PSATTN_EINVAL;
    if (n_rows == 0) return PSATTN_OK;
    if (!X || !weight || !Y || !mean || !rstd || (!R) != (!S)) return PSATTN_EINVAL;
    if (n_rows > kMostRows || hidden > INT32_MAX / 2) return PSATTN_EUNSUPPORTED;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dt == PSATTN_BF16) fwd<uint16_t>(n_rows, hidden, eps, X, R, weight, bias, S, Y, mean, rstd, s);
    else fwd<float>(n_rows, hidden, eps, X, R, weight, bias, S, Y, mean, rstd, s);
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

size_t psattn_layernorm_bwd_workspace_bytes(int32_t n_rows, int32_t hidden) {
    if (n_rows < 0 || hidden <= 0) return 0;
    return align_up(2 * sizeof(float) * static_cast<size_t>(n_parts(n_rows, hidden)) * hidden, 256) + 256;
}

int psattn_layernorm_bwd(int32_t dt, int32_t n_rows, int32_t hidden, const void* S, const void* weight, const float* mean, const float* rstd,
                         const void* dY, const void* dS, void* dX, void* dweight, void* dbias, void* workspace, size_t workspace_bytes,
                         void* hip_stream) {
    if (bad_shape(dt, n_rows, hidden) || !dweight) return PSATTN_EINVAL;
    if (n_rows > 0 && (!S || !weight || !mean || !rstd || !dY || !dX || !workspace)) return PSATTN_EINVAL;
    if (n_rows > 0 && workspace_bytes < psattn_layernorm_bwd_workspace_bytes(n_rows, hidden)) return PSATTN_EINVAL;
    if (n_rows > kMostRows || hidden > INT32_MAX / 2) return PSATTN_EUNSUPPORTED;
    float* const part = reinterpret_cast<float*>(align_up(reinterpret_cast<uintptr_t>(workspace), 256));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dt == PSATTN_BF16) bwd<uint16_t>(n_rows, hidden, S, weight, mean, rstd, dY, dS, dX, dweight, dbias, part, s);
    else bwd<float>(n_rows, hidden, S, weight, mean, rstd, dY, dS, dX, dweight, dbias, part, s);
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

}  // extern "C"
