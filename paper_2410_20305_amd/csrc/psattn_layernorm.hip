// Layer norm over rows of `hidden` elements, with the residual sum in front of it, forward and backward.
//   S = X + R (rounded to the element type: the residual stream is held in it, and the backward reads it; S = X without R)
//   Y = (S - mean) rstd w + b, rstd = 1 / sqrt(mean((S - mean)^2) + eps)
//   with xh = (S - mean) rstd, q = dY w:  dX = rstd (q - mean(q) - xh mean(q xh)) + dS,  dw = sum_rows dY xh,  db = sum_rows dY
#include <hip/hip_runtime.h>

#include <cmath>

#include "psattn.h"
#include "psattn_gemm.h"

namespace {

using psattn::gemm::store1;
using psattn::gemm::to_f32;

constexpr int kThreads = 256;
constexpr int kSumRows = 64;  // rows of a partial sum of dw, db

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// the same in every thread
__device__ inline float block_sum(float v, float* sm) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < kThreads / 64; ++i) v += sm[i];
    return v;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void psattn_ln_fwd(int hidden, float eps, const E* X, const E* R, const E* w, const E* b, E* S, E* Y,
                                                          float* mean, float* rstd) {
    __shared__ float sm[kThreads / 64];
    const size_t at = static_cast<size_t>(blockIdx.x) * hidden;
    const E* x = X + at;
    float sum = 0.f;
    for (int i = threadIdx.x; i < hidden; i += kThreads) {
        float v = to_f32(x[i]);
        if (R) {
            store1(S + at + i, v + to_f32(R[at + i]));
            v = to_f32(S[at + i]);
        }
        sum += v;
    }
    if (R) x = S + at;
    const float mu = block_sum(sum, sm) / hidden;
    float sq = 0.f;
    for (int i = threadIdx.x; i < hidden; i += kThreads) {
        const float v = to_f32(x[i]) - mu;
        sq += v * v;
    }
    const float rs = 1.f / sqrtf(block_sum(sq, sm) / hidden + eps);
    for (int i = threadIdx.x; i < hidden; i += kThreads)
        store1(Y + at + i, (to_f32(x[i]) - mu) * rs * to_f32(w[i]) + (b ? to_f32(b[i]) : 0.f));
    if (threadIdx.x == 0) {
        mean[blockIdx.x] = mu;
        rstd[blockIdx.x] = rs;
    }
}

template <typename E>
__global__ __launch_bounds__(kThreads) void psattn_ln_bwd(int hidden, const E* S, const E* w, const float* mean, const float* rstd, const E* dY,
                                                          const E* dS, E* dX) {
    __shared__ float sm[kThreads / 64];
    const size_t at = static_cast<size_t>(blockIdx.x) * hidden;
    const float mu = mean[blockIdx.x], rs = rstd[blockIdx.x];
    float s1 = 0.f, s2 = 0.f;
    for (int i = threadIdx.x; i < hidden; i += kThreads) {
        const float q = to_f32(dY[at + i]) * to_f32(w[i]);
        s1 += q;
        s2 += q * (to_f32(S[at + i]) - mu) * rs;
    }
    s1 = block_sum(s1, sm) / hidden;
    s2 = block_sum(s2, sm) / hidden;
    for (int i = threadIdx.x; i < hidden; i += kThreads) {
        const float q = to_f32(dY[at + i]) * to_f32(w[i]), xh = (to_f32(S[at + i]) - mu) * rs;
        store1(dX + at + i, rs * (q - s1 - xh * s2) + (dS ? to_f32(dS[at + i]) : 0.f));
    }
}

// part[y][0 / 1][column]: sums over rows y kSumRows ..
template <typename E>
__global__ __launch_bounds__(kThreads) void psattn_ln_weight_parts(int n_rows, int hidden, const E* S, const float* mean, const float* rstd, const E* dY,
                                                                   float* part) {
    const int i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= hidden) return;
    float w = 0.f, b = 0.f;
    const int r0 = blockIdx.y * kSumRows, r1 = min(n_rows, r0 + kSumRows);
    for (int r = r0; r < r1; ++r) {
        const size_t at = static_cast<size_t>(r) * hidden + i;
        const float dy = to_f32(dY[at]);
        w += dy * (to_f32(S[at]) - mean[r]) * rstd[r];
        b += dy;
    }
    part[(2 * static_cast<size_t>(blockIdx.y)) * hidden + i] = w;
    part[(2 * static_cast<size_t>(blockIdx.y) + 1) * hidden + i] = b;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void psattn_ln_weight_join(int n_parts, int hidden, const float* part, E* dw, E* db) {
    const int i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= hidden) return;
    float w = 0.f, b = 0.f;
    for (int p = 0; p < n_parts; ++p) {
        w += part[(2 * static_cast<size_t>(p)) * hidden + i];
        b += part[(2 * static_cast<size_t>(p) + 1) * hidden + i];
    }
    store1(dw + i, w);
    if (db) store1(db + i, b);
}

int n_parts(int n_rows) { return (n_rows + kSumRows - 1) / kSumRows; }

bool bad_shape(int32_t dt, int32_t n_rows, int32_t hidden) { return (dt != PSATTN_F32 && dt != PSATTN_BF16) || n_rows < 0 || hidden <= 0; }

template <typename E>
void fwd(int32_t n_rows, int32_t hidden, float eps, const void* X, const void* R, const void* w, const void* b, void* S, void* Y, float* mean,
         float* rstd, hipStream_t s) {
    psattn_ln_fwd<E><<<n_rows, kThreads, 0, s>>>(hidden, eps, static_cast<const E*>(X), static_cast<const E*>(R), static_cast<const E*>(w),
                                                  static_cast<const E*>(b), static_cast<E*>(S), static_cast<E*>(Y), mean, rstd);
}

template <typename E>
void bwd(int32_t n_rows, int32_t hidden, const void* S, const void* w, const float* mean, const float* rstd, const void* dY, const void* dS, void* dX,
         void* dw, void* db, float* part, hipStream_t s) {
    const E *xs = static_cast<const E*>(S), *dy = static_cast<const E*>(dY);
    const int cols = (hidden + kThreads - 1) / kThreads, np = n_parts(n_rows);
    if (n_rows > 0) {
        psattn_ln_bwd<E><<<n_rows, kThreads, 0, s>>>(hidden, xs, static_cast<const E*>(w), mean, rstd, dy, static_cast<const E*>(dS), static_cast<E*>(dX));
        psattn_ln_weight_parts<E><<<dim3(cols, np), kThreads, 0, s>>>(n_rows, hidden, xs, mean, rstd, dy, part);
    }
    psattn_ln_weight_join<E><<<cols, kThreads, 0, s>>>(np, hidden, part, static_cast<E*>(dw), static_cast<E*>(db));
}

}  // namespace

extern "C" {

int psattn_layernorm_fwd(int32_t dt, int32_t n_rows, int32_t hidden, float eps, const void* X, const void* R, const void* weight, const void* bias,
                         void* S, void* Y, float* mean, float* rstd, void* hip_stream) {
    if (bad_shape(dt, n_rows, hidden) || !(eps >= 0.f) || std::isinf(eps)) return PSATTN_EINVAL;
    if (n_rows == 0) return PSATTN_OK;
    if (!X || !weight || !Y || !mean || !rstd || (!R) != (!S)) return PSATTN_EINVAL;
    if (n_rows >= (1 << 23)) return PSATTN_EUNSUPPORTED;
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
    if (n_rows >= (1 << 22)) return PSATTN_EUNSUPPORTED;
    float* const part = reinterpret_cast<float*>(align_up(reinterpret_cast<uintptr_t>(workspace), 256));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dt == PSATTN_BF16) bwd<uint16_t>(n_rows, hidden, S, weight, mean, rstd, dY, dS, dX, dweight, dbias, part, s);
    else bwd<float>(n_rows, hidden, S, weight, mean, rstd, dY, dS, dX, dweight, dbias, part, s);
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

}  // extern "C"
