// The vocabulary head without kept logits: log-probabilities of responses from hidden rows X and the vocabulary matrix W, forward and
// backward (paper Section 2.1, Eq. 1: the loss needs log pi(y | x) of every completion).
//   items i: a row r_i that predicts token y_i of response j_i;  z_iv = X[r_i] . W[v],  lse_i = log sum_v exp z_iv
//   forward:   log pi_j = sum over i of j of (z_{i, y_i} - lse_i)
//   backward:  dz_iv = d_j (1[v = y_i] - exp(z_iv - lse_i));  dX[r] = sum over i of r of dz_i W,  dW = dz^T X
//
// Logits of a packed batch are larger than everything else in a step (65 536 rows of 128 000 bf16: 16.8 GB, and their gradient again).  Here they
// exist as accumulators of the matrix product alone: its epilogue leaves a maximum and a sum of exponentials of every tile's part of a
// row, and the target's logit.  The backward makes them again, a piece of the vocabulary at a time, and turns them into dz in the
// epilogue; dz of a piece (in the element type, rounded once, from fp32) is the operand of the two other products: dW's rows of
// the piece, written at once, and dX's sums over the pieces in fp32.  Only rows that predict something take part: prompts, most of the
// tokens, do not.  A prompt's last row predicts the first token of every response and takes part once for each.
//
// Bound by the matrix cores (four products of 2 items vocab hidden operations in a training step, one of them to make the logits again), for few rows by
// reading W.  Every sum has a fixed order, and none is made by atomics.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "psattn_head.h"
#include "psattn_logprob.h"
#include "psattn_rows.h"

namespace {

using namespace psattn::gemm;
namespace rows = psattn::rows;

constexpr int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
constexpr int64_t up64(int64_t n) { return (n + 63) / 64 * 64; }  // a step of k of bf16, two of fp32
size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
size_t elem_bytes(int32_t dt) { return dt == PSATTN_BF16 ? 2 : 4; }
// of psattn_head_rows: a lane to 16 bytes, up to four waves
int row_threads(int32_t dt, int64_t hidden) { return static_cast<int>(std::min<int64_t>(256, up64(cdiv(hidden, dt == PSATTN_BF16 ? 8 : 4)))); }

// ---- items, numbered response by response: which row and which token are the i-th's.  (Tables of them would be most of a plan: with, without 2.2 and
// 0.95 ms for 2^20 tokens of 512 samples, 136 and 66 us for 65 536 of 64.)
struct Items {
    int32_t n_resp;
    const int32_t *ptr, *resp_first, *resp_prev;  // a plan's
};
// The last response that starts at item i or ahead of it (empty ones have no item), by a whole wave, 256 places at a time.  9 812 items of 96 responses
// and 512 columns, forward's and backward's rows: by halves, seven loads one after the other, in workgroups of 256 12.8 and 16.9 us; so, in as many waves
// as a row has work for, 7.1 and 7.8
__device__ __forceinline__ int response_of(const Items& t, int i) {
    const int l = threadIdx.x & 63;
    int first = 0, n = t.n_resp;
    while (n > 1) {
        const int step = (n - 1) / 256 + 1;
        bool ahead[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int at = (q * 64 + l) * step;
            ahead[q] = at < n && t.ptr[first + at] <= i;
        }
        int k = -1;  // they ascend
#pragma unroll
        for (int q = 0; q < 4; ++q) k += __builtin_popcountll(__builtin_amdgcn_ballot_w64(ahead[q]));
        first += k * step;
        n = min(step, n - k * step);
    }
    return first;
}

// ---- the items' rows, made whole: one workgroup to a row.  Without a token of the vocabulary, or with a weight of 0, an item has no gradient, and its
// row is zeros there: what is not finite in it would reach all of dW by dz = 0.
// BWD: up to `again` the rows stand there once more (for the second part of dz), and behind them, in dz too, rows of zeros, so that dW's
// k is whole steps.  item_of: all -1.  item_row: an item's row, or ~row where an earlier one has the same
template <typename E, bool BWD>
__global__ __launch_bounds__(256) void psattn_head_rows(int n_items, int again, Items items, int32_t* item_row, const int32_t* token_ids, int vocab, int hidden, const E* X, const float* row_lse, const float* d_logp, E* out,
                                                        int32_t* target, float* lse, float* weight, float* at_token, int32_t* item_of, E* dz, int64_t ldz) {
    constexpr int V = rows::kVec<E>;
    const int64_t at = blockIdx.x, ld = (hidden + 7) / 8 * 8;
    if (BWD && item_of)
        for (int64_t v = at * blockDim.x + threadIdx.x; v < vocab; v += gridDim.x * blockDim.x) item_of[v] = -1;
    if (BWD && at >= again) {
        const rows::u32x4 zero = {0, 0, 0, 0};
        for (int64_t c = threadIdx.x * V; c < ld; c += blockDim.x * V) *reinterpret_cast<rows::u32x4*>(out + at * ld + c) = zero;
        for (int64_t c = threadIdx.x * V; c < ldz; c += blockDim.x * V) *reinterpret_cast<rows::u32x4*>(dz + at * ldz + c) = zero;
        return;
    }
    const int i = static_cast<int>(at < n_items ? at : at - n_items), j = response_of(items, i);
    const int prev = items.resp_prev[j], u = i - items.ptr[j] + (prev < 0 ? 1 : 0), first = items.resp_first[j];
    const int row = u == 0 ? prev : first + u - 1, id = token_ids[first + u];
    const bool known = id >= 0 && id < vocab;
    const float d_j = BWD ? d_logp[j] : 0.f, d = known ? d_j : 0.f;
    // an earlier item of this row: the last one, of the response ahead or, behind empty ones, another
    const bool again_row = !BWD && u == 0 && i > 0 && items.resp_prev[items.ptr[j - 1] < i ? j - 1 : response_of(items, i - 1)] == prev;
    if (threadIdx.x == 0 && at < n_items) {
        target[i] = known ? id : -1;
        if constexpr (BWD) {
            lse[i] = known ? row_lse[row] : 0.f;
            weight[i] = d;
            at_token[i] = 0.f;
        } else {
            item_row[i] = again_row ? ~row : row;
        }
    }
    const E* const x = X + static_cast<int64_t>(row) * hidden;
    for (int c = threadIdx.x * V; c < ld; c += blockDim.x * V) {
        rows::u32x4 u = {0, 0, 0, 0};
        if (c < hidden) {
            const auto p = rows::place<false, E>(c, hidden);
            u = rows::settled<false>(rows::raw<false>(x, p, hidden), p.down);
        }
        if (BWD && d == 0.f) u = rows::u32x4{0, 0, 0, 0};
        *reinterpret_cast<rows::u32x4*>(out + at * ld + c) = u;
    }
}

// ---- logits whose tiles are too few for the chip: their products' parts of k, [part][item][ld], joined here
// four logits from column c on; what is behind the last is -inf
__device__ __forceinline__ void joined(const float* parts, int64_t step, int n_parts, int c, int cols, float (&z)[4]) {
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    int p = 0;
    auto add = [&](auto COUNT) {  // loads together, sums in order
        constexpr int n = decltype(COUNT)::value;
        float4 u[n];
#pragma unroll
        for (int k = 0; k < n; ++k) u[k] = *reinterpret_cast<const float4*>(parts + (p + k) * step + c);
#pragma unroll
        for (int k = 0; k < n; ++k) sum.x += u[k].x, sum.y += u[k].y, sum.z += u[k].z, sum.w += u[k].w;
        p += n;
    };
    while (p + 8 <= n_parts) add(std::integral_constant<int, 8>{});
    while (p < n_parts) add(std::integral_constant<int, 1>{});
    z[0] = sum.x;
    z[1] = c + 1 < cols ? sum.y : -INFINITY;
    z[2] = c + 2 < cols ? sum.z : -INFINITY;
    z[3] = c + 3 < cols ? sum.w : -INFINITY;
}

// an item to a workgroup: its log-sum-exp and its token's log-probability
__global__ __launch_bounds__(1024) void psattn_head_parts_lse(int n_items, int n_parts, int cols, int64_t ld, const float* parts, const int32_t* item_row, const int32_t* target,
                                                              float* row_lse, float* item_logp) {
    __shared__ float2 sm[16];
    __shared__ float hit;
    const int i = blockIdx.x, t = target[i];
    const float* const z0 = parts + static_cast<int64_t>(i) * ld;
    float m = -INFINITY, s = 0.f;
    auto merge = [&](float m2, float s2) {
        const float mn = fmaxf(m, m2), ref = mn == -INFINITY ? 0.f : mn;
        s = s * expf(m - ref) + s2 * expf(m2 - ref);
        m = mn;
    };
    for (int c = threadIdx.x * 4; c < cols; c += 4096) {
        float z[4];
        joined(z0, n_items * ld, n_parts, c, cols, z);
        const float mx = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), ref = mx == -INFINITY ? 0.f : mx;
        merge(mx, (expf(z[0] - ref) + expf(z[1] - ref)) + (expf(z[2] - ref) + expf(z[3] - ref)));
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + k == t) hit = z[k];
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) merge(__shfl_xor(m, off), __shfl_xor(s, off));
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = make_float2(m, s);
    __syncthreads();
    if (threadIdx.x > 0) return;
    for (int w = 1; w < 16; ++w) merge(sm[w].x, sm[w].y);
    const float ls = logf(s);
    if (const int r = item_row[i]; r >= 0) row_lse[r] = m + ls;
    item_logp[i] = t >= 0 ? (hit - m) - ls : 0.f;
}

// dz of an item, 1 024 columns to a workgroup.  bf16: what its rounding leaves, or its value at the item's token apart, where that is asked for
template <typename E>
__global__ __launch_bounds__(256) void psattn_head_parts_dz(int n_items, int n_parts, int first, int cols, int64_t ld, const float* parts, const int32_t* target, const float* lse,
                                                            const float* weight, E* dz, E* rest, float* at_token, int32_t* item_of, int64_t ldz) {
    const int64_t i = blockIdx.y;
    const int c = (blockIdx.x * 256 + threadIdx.x) * 4, t = target[i] - first;
    if (c >= cols) return;
    const float l = lse[i], w = weight[i];
    float z[4];
    joined(parts + i * ld, n_items * ld, n_parts, c, cols, z);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (c + k >= cols) break;
        const float p = expf(z[k] - l), x = w == 0.f ? 0.f : w * (c + k == t ? 1.f - p : -p);
        const bool apart = at_token && c + k == t;
        rows::store1(dz + i * ldz + c + k, apart ? 0.f : x);
        if (rest) rows::store1(rest + i * ldz + c + k, x - rows::hold(x, dz));
        if (apart) {
            at_token[i] = x;
            __hip_atomic_store(item_of + target[i], static_cast<int32_t>(i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // other items' too
        }
    }
}

// ---- joins the tiles' parts of an item's row, L lanes to an item; the result is lane 0's.  sm: [L][256 / L]
struct Sum {
    float m, s;  // maximum, sum of exp(z - m)
    __device__ __forceinline__ void merge(float m2, float s2) {
        const float mn = fmaxf(m, m2), ref = mn == -INFINITY ? 0.f : mn;
        s = s * expf(m - ref) + s2 * expf(m2 - ref);
        m = mn;
    }
};
template <int L>
__device__ __forceinline__ Sum join_item(int n_items, int n_parts, const float2* part, int i, int k, int o, float2* sm) {
    constexpr int AT = 256 / L, kAtOnce = 4;
    Sum x{-INFINITY, 0.f};
    if (i < n_items) {
        int p = k;
        for (; p + (kAtOnce - 1) * L < n_parts; p += kAtOnce * L) {
            float2 y[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) y[u] = part[static_cast<int64_t>(p + u * L) * n_items + i];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) x.merge(y[u].x, y[u].y);
        }
        for (; p < n_parts; p += L) {
            const float2 y = part[static_cast<int64_t>(p) * n_items + i];
            x.merge(y.x, y.y);
        }
    }
    sm[k * AT + o] = make_float2(x.m, x.s);
    __syncthreads();
#pragma unroll 1
    for (int n = L / 2; n > 0; n >>= 1) {
        if (k < n) {
            x.merge(sm[(k + n) * AT + o].x, sm[(k + n) * AT + o].y);
            sm[k * AT + o] = make_float2(x.m, x.s);
        }
        __syncthreads();
    }
    return x;
}

// AT items to a workgroup.  log pi of an item as (logit - max) - log(sum), which keeps its accuracy where the token is almost certain
template <int AT>
__global__ __launch_bounds__(256) void psattn_head_join(int n_items, int n_parts, const float2* part, const int32_t* item_row, const int32_t* target, const float* hit,
                                                        float* row_lse, float* item_logp) {
    __shared__ float2 sm[256];
    const int k = threadIdx.x / AT, o = threadIdx.x % AT, i = blockIdx.x * AT + o;
    const Sum x = join_item<256 / AT>(n_items, n_parts, part, i, k, o, sm);
    if (k > 0 || i >= n_items) return;
    const float ls = logf(x.s);
    if (const int r = item_row[i]; r >= 0) row_lse[r] = x.m + ls;
    item_logp[i] = target[i] >= 0 ? (hit[i] - x.m) - ls : 0.f;
}

// ... of few items, a response to a workgroup, and their sum: a launch less
__global__ __launch_bounds__(256) void psattn_head_join_few(int n_items, int n_parts, const float2* part, const int32_t* item_row, const int32_t* item_ptr,
                                                            const int32_t* target, const float* hit, float* row_lse, float* resp_logp) {
    __shared__ float2 sm[256];
    const int j = blockIdx.x, k = threadIdx.x;
    float logp = 0.f;
    for (int i = item_ptr[j]; i < item_ptr[j + 1]; ++i) {
        const Sum x = join_item<256>(n_items, n_parts, part, i, k, 0, sm);
        const float ls = logf(x.s);
        if (const int r = item_row[i]; k == 0 && r >= 0) row_lse[r] = x.m + ls;
        logp += target[i] >= 0 ? (hit[i] - x.m) - ls : 0.f;
        __syncthreads();
    }
    if (k == 0) resp_logp[j] = logp;
}

__global__ __launch_bounds__(256) void psattn_head_responses(int first, const int32_t* item_ptr, const float* item_logp, float* resp_logp) {
    __shared__ float sm[4];
    const int j = first + static_cast<int>(blockIdx.x), end = item_ptr[j + 1];
    float v = 0.f;
    for (int i = item_ptr[j] + static_cast<int>(threadIdx.x); i < end; i += 256) v += item_logp[i];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) resp_logp[j] = (sm[0] + sm[1]) + (sm[2] + sm[3]);
}

// ---- bf16: dz at an item's own token.  It is most of its row's weight, and its rounding error would be that of all columns of dX and of the
// token's row of dW alike: it stays in fp32, out of the products, and joins their results here.  (99 items, gradients against 64 bits: dX 2.4e-3
// in the products, 1.66e-3 apart, which is its own rounding; dW 2.34e-3 and 1.66e-3.)  The row of a frequent token is a small difference of two
// large parts: what bf16 leaves of the products' part joins it too (columns of mean 1/3, probabilities up to 0.2, equal weights, a row of dW off
// by, without that / with it: 9 812 items 1.7e-2 / 1.5e-3, 1 000 8.8e-3 / 1.9e-3, 99 2.4e-3 / 1.9e-3; 16 384 tokens of 128 000 x 4 096 34.55 / 34.3 ms).
template <typename E>
__device__ __forceinline__ void add_token(float at_token, const E* w, int c, int hidden, float (&x)[4]) {
    if (at_token == 0.f) return;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (c + k < hidden) x[k] = fmaf(at_token, rows::to_f32(w[c + k]), x[k]);
}

// dW[token] += sum of dz X over the items of that token, and what bf16 has left of the products' row, which stands in `rest` by the item that
// item_of names.  That item does it, whichever of them it is: it looks for all of them from the first on, so the sum does not depend on it.  `lanes` * 4
// columns to a workgroup, whose 256 / lanes groups take items in turn; n V / 4 096 steps at most beside the products' n V hidden.
__global__ __launch_bounds__(256) void psattn_head_dw_tokens(int first, int lanes, int col_blocks, int n_items, int hidden, int64_t ld, const int32_t* target, const int32_t* item_of,
                                                             const float* at_token, const uint16_t* x, const uint16_t* rest, uint16_t* dW) {
    constexpr int V = 4, kAtOnce = 8, kFours = 4, kSpan = 1024 * kFours;  // items looked at together: kFours times 4 to a thread
    __shared__ int found[kSpan], count[kFours][4];
    __shared__ float4 sums[256];
    const int i = first + static_cast<int>(blockIdx.x) / col_blocks, token = target[i], mine = static_cast<int>(threadIdx.x) * 4, l = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (token < 0 || item_of[token] != i) return;
    auto same = [&](int base) {  // which of the thread's items are of that token: four bits to each 1 024 of them
        int4 t[kFours];
#pragma unroll
        for (int u = 0; u < kFours; ++u)  // the table's last four are its own: it is of whole 256 bytes
            t[u] = base + 1024 * u + mine < n_items ? *reinterpret_cast<const int4*>(target + base + 1024 * u + mine) : make_int4(-1, -1, -1, -1);
        uint32_t yes = 0;
#pragma unroll
        for (int u = 0; u < kFours; ++u) {
            const int tok[4] = {t[u].x, t[u].y, t[u].z, t[u].w}, at = base + 1024 * u + mine;
#pragma unroll
            for (int k = 0; k < 4; ++k) yes |= tok[k] == token && at + k < n_items ? 1u << (4 * u + k) : 0u;
        }
        return yes;
    };
    const int lane = static_cast<int>(threadIdx.x) & (lanes - 1), group = static_cast<int>(threadIdx.x) / lanes, groups = 256 / lanes;
    const int c = (static_cast<int>(blockIdx.x) % col_blocks * lanes + lane) * V;
    float sum[V] = {};
    for (int base = 0; base < n_items; base += kSpan) {
        const uint32_t yes = same(base);
        if (!__syncthreads_or(yes)) continue;
        int at[kFours] = {}, n = 0;
#pragma unroll
        for (int u = 0; u < kFours; ++u) {
            int all = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint64_t votes = __builtin_amdgcn_ballot_w64(yes >> (4 * u + k) & 1);
                at[u] += __builtin_popcountll(votes & ((uint64_t{1} << l) - 1));
                all += __builtin_popcountll(votes);
            }
            if (l == 0) count[u][wave] = all;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kFours; ++u) {
            at[u] += n;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                at[u] += w < wave ? count[u][w] : 0;
                n += count[u][w];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (yes >> (4 * u + k) & 1) found[at[u]++] = base + 1024 * u + mine + k;
        }
        __syncthreads();
        if (c >= hidden) continue;
        auto add = [&](int k, auto COUNT) {  // loads together, sums in order
            constexpr int m = decltype(COUNT)::value;
            uint2 u[m];
            float w[m];
#pragma unroll
            for (int q = 0; q < m; ++q) {
                const int64_t item = found[k + q * groups];
                u[q] = *reinterpret_cast<const uint2*>(x + item * ld + c);
                w[q] = at_token[item];
            }
#pragma unroll
            for (int q = 0; q < m; ++q) {
                if (w[q] == 0.f) continue;
                sum[0] = fmaf(w[q], __uint_as_float(u[q].x << 16), sum[0]);
                sum[1] = fmaf(w[q], __uint_as_float(u[q].x & 0xffff0000u), sum[1]);
                sum[2] = fmaf(w[q], __uint_as_float(u[q].y << 16), sum[2]);
                sum[3] = fmaf(w[q], __uint_as_float(u[q].y & 0xffff0000u), sum[3]);
            }
        };
        int k = group;
        for (; k + (kAtOnce - 1) * groups < n; k += kAtOnce * groups) add(k, std::integral_constant<int, kAtOnce>{});
        for (; k < n; k += groups) add(k, std::integral_constant<int, 1>{});
    }
    if (groups > 1) {
        sums[threadIdx.x] = make_float4(sum[0], sum[1], sum[2], sum[3]);
        __syncthreads();
        if (group) return;
        for (int g = 1; g < groups; ++g) {
            const float4 x = sums[g * lanes + lane];
            sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
        }
    }
    if (c >= hidden) return;
    uint16_t* const to = dW + static_cast<int64_t>(token) * hidden + c;
    rest += static_cast<int64_t>(i) * hidden + c;
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (c + k < hidden) {
            const float x = rows::to_f32(to[k]);  // of one beyond bf16's range nothing is left that would be a number
            rows::store1(to + k, x + (fabsf(x) < INFINITY ? rows::to_f32(rest[k]) + sum[k] : sum[k]));
        }
}

// dW of a piece from its parts, four columns to a lane; item_of and rest as kTokens has them, or null
template <typename E>
__global__ __launch_bounds__(256) void psattn_head_dw_join(int n_parts, int cols, int hidden, int64_t ld, const float* parts, int odd, E* dW, const int32_t* item_of, E* rest) {
    constexpr int V = 4, kAtOnce = 8;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, per = ld / V, row = i / per, step = cols * ld;
    const int c = static_cast<int>(i - row * per) * V;
    if (row >= cols || c >= hidden) return;
    const float* const from = parts + row * ld + c;
    float x[V] = {};
    auto add = [&](int p, auto COUNT) {  // loads together, sums in order
        constexpr int n = decltype(COUNT)::value;
        float4 u[n];
#pragma unroll
        for (int q = 0; q < n; ++q) u[q] = *reinterpret_cast<const float4*>(from + (p + q) * step);
#pragma unroll
        for (int q = 0; q < n; ++q) x[0] += u[q].x, x[1] += u[q].y, x[2] += u[q].z, x[3] += u[q].w;
    };
    int p = 0;
    for (; p + kAtOnce <= n_parts; p += kAtOnce) add(p, std::integral_constant<int, kAtOnce>{});
    for (; p < n_parts; ++p) add(p, std::integral_constant<int, 1>{});
    E* const to = dW + row * hidden + c;
    if (const int item = item_of ? item_of[row] : -1; item >= 0) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (c + k < hidden) rows::store1(rest + static_cast<int64_t>(item) * hidden + c + k, x[k] - rows::hold(x[k], dW));
    }
    if (!odd) {  // rows of whole groups on their boundaries
        if constexpr (sizeof(E) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(psattn::mma::pack2(x[0], x[1]), psattn::mma::pack2(x[2], x[3]));
        else *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]);
        return;
    }
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (c + k < hidden) rows::store1(to + k, x[k]);
}

// ---- dX of token t: the sums of its items, of all parts of each; `again` rows to a part
template <typename E>
__global__ __launch_bounds__(256) void psattn_head_dx(int64_t first, int col_blocks, int hidden, int n_items, int again, int n_parts, int64_t ld, const float* parts, const int32_t* row_desc,
                                                      const int32_t* resp_first, const int32_t* resp_len, const int32_t* resp_prev, const int32_t* samp_ptr,
                                                      const int32_t* item_ptr, const int32_t* target, const float* weight, const float* at_token, const E* W, E* dX) {
    constexpr int V = 4;
    const int64_t block = first + blockIdx.x;
    const int row = static_cast<int>(block / col_blocks), desc = row_desc[row];
    E* const to = dX + static_cast<int64_t>(row) * hidden;
    int r0 = 0, r1 = 0;  // responses with an item of this row
    if (desc >= 0) r0 = desc, r1 = desc + 1;
    else if (desc < -1) r0 = samp_ptr[-2 - desc], r1 = samp_ptr[-1 - desc];
    for (int c = (static_cast<int>(block - static_cast<int64_t>(row) * col_blocks) * 256 + threadIdx.x) * V; c < hidden; c += col_blocks * 256 * V) {
        float x[V] = {};
        for (int j = r0; j < r1; ++j) {
            if (resp_len[j] == 0) continue;
            const int i = item_ptr[j] + (desc >= 0 ? row - resp_first[j] + (resp_prev[j] >= 0 ? 1 : 0) : 0);
            if (weight[i] == 0.f) continue;
            const int64_t step = again * ld;
            for (int64_t row_of = i; row_of < again; row_of += n_items) {  // and its second part's
                const float* from = parts + row_of * ld + c;
                auto add = [&](auto COUNT) {  // loads together, sums in order
                    constexpr int n = decltype(COUNT)::value;
                    float4 u[n];
#pragma unroll
                    for (int p = 0; p < n; ++p) u[p] = *reinterpret_cast<const float4*>(from + p * step);
#pragma unroll
                    for (int p = 0; p < n; ++p) x[0] += u[p].x, x[1] += u[p].y, x[2] += u[p].z, x[3] += u[p].w;
                    from += n * step;
                };
                int p = 0;
                for (; p + 8 <= n_parts; p += 8) add(std::integral_constant<int, 8>{});
                for (; p < n_parts; ++p) add(std::integral_constant<int, 1>{});
            }
            if (at_token) add_token(at_token[i], W + static_cast<int64_t>(target[i]) * hidden, c, hidden, x);
        }
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (c + k < hidden) rows::store1(to + c + k, x[k]);
    }
}

// ... where it has many parts: 256 columns to a workgroup, whose sixteen waves share the parts
template <typename E>
__global__ __launch_bounds__(1024) void psattn_head_dx_parts(int64_t first, int col_blocks, int hidden, int n_items, int again, int n_parts, int64_t ld, const float* parts,
                                                             const int32_t* row_desc, const int32_t* resp_first, const int32_t* resp_len, const int32_t* resp_prev,
                                                             const int32_t* samp_ptr, const int32_t* item_ptr, const int32_t* target, const float* weight, const float* at_token, const E* W, E* dX) {
    constexpr int V = 4, kAtOnce = 4;
    __shared__ float4 sm[16][64];
    const int64_t block = first + blockIdx.x;
    const int row = static_cast<int>(block / col_blocks), desc = row_desc[row], w = threadIdx.x >> 6, l = threadIdx.x & 63;
    const int c = (static_cast<int>(block - static_cast<int64_t>(row) * col_blocks) * 64 + l) * V;
    int r0 = 0, r1 = 0;
    if (desc >= 0) r0 = desc, r1 = desc + 1;
    else if (desc < -1) r0 = samp_ptr[-2 - desc], r1 = samp_ptr[-1 - desc];
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    const int64_t step = again * ld;
    auto add = [&](const float4& u) { x.x += u.x, x.y += u.y, x.z += u.z, x.w += u.w; };
    if (c < hidden)
        for (int j = r0; j < r1; ++j) {
            if (resp_len[j] == 0) continue;
            const int i = item_ptr[j] + (desc >= 0 ? row - resp_first[j] + (resp_prev[j] >= 0 ? 1 : 0) : 0);
            if (weight[i] == 0.f) continue;
            for (int64_t row_of = i; row_of < again; row_of += n_items) {
                const float* const from = parts + row_of * ld + c;
                int p = w;
                for (; p + 16 * (kAtOnce - 1) < n_parts; p += 16 * kAtOnce) {
                    float4 u[kAtOnce];
#pragma unroll
                    for (int k = 0; k < kAtOnce; ++k) u[k] = *reinterpret_cast<const float4*>(from + (p + 16 * k) * step);
#pragma unroll
                    for (int k = 0; k < kAtOnce; ++k) add(u[k]);
                }
                for (; p < n_parts; p += 16) add(*reinterpret_cast<const float4*>(from + p * step));
            }
            if (at_token && w == 0) {
                float y[V] = {x.x, x.y, x.z, x.w};
                add_token(at_token[i], W + static_cast<int64_t>(target[i]) * hidden, c, hidden, y);
                x = make_float4(y[0], y[1], y[2], y[3]);
            }
        }
    sm[w][l] = x;
    __syncthreads();
    if (w > 0 || c >= hidden) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) add(sm[k][l]);
    E* const to = dX + static_cast<int64_t>(row) * hidden + c;
    const float v[V] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (c + k < hidden) rows::store1(to + k, v[k]);
}

// zeros without a memset, which a captured graph would not replay faithfully
__global__ void psattn_head_zero(uint16_t* p, size_t n) {
    for (size_t i = blockIdx.x * static_cast<size_t>(blockDim.x) + threadIdx.x; i < n; i += static_cast<size_t>(gridDim.x) * blockDim.x) p[i] = 0;
}

// n workgroups in grids of at most 2^31 threads
template <typename F>
void in_grids(int64_t n, int threads, F launch) {
    const int64_t most = (int64_t{1} << 31) / threads;
    for (int64_t at = 0; at < n; at += most) launch(at, static_cast<uint32_t>(std::min<int64_t>(n - at, most)));
}

// ---- products
bool at16(std::initializer_list<const void*> p) {
    uintptr_t a = 0;
    for (const void* x : p) a |= reinterpret_cast<uintptr_t>(x);
    return a % 16 == 0;
}

constexpr int64_t kPartBytes = 64 << 20, kPartItems = 4096;  // of logits in parts, at most

// Which tile: few rows take tiles of 32 and 64 rows, whose workgroups share a CU, others what the products' model says
struct Tiling {
    TileSize size;
    int64_t split;  // parts of k
};
Tiling tiling(Move move, int64_t M, int64_t N, int64_t K, bool may_split) {
    static constexpr int bm[] = {32, 64, 128, 256}, bn[] = {128, 128, 128, 256};
    const int64_t steps = K / (move == kFloat ? 32 : 64);
    auto tiles = [&](TileSize t) { return std::max<int64_t>(1, cdiv(M, bm[t]) * cdiv(N, bn[t])); };
    if (M <= 64) {
        const TileSize t = M <= 32 ? k32 : k64;
        return {t, may_split ? std::max<int64_t>(1, std::min((M <= 32 ? 1024 : 768) / tiles(t), steps / 4)) : 1};
    }
    Tiling best{k128, 1};
    double least = 0;
    for (const TileSize t : {k128, k256})
        for (const int64_t split : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 24, 32, 48, 64}) {
            if (split > 1 && (!may_split || steps / split < 4)) break;
            const double us = product_us(move, kPlain, t, tiles(t), steps, split, sizeof(float) * static_cast<double>(M) * static_cast<double>(N));
            if ((t == k128 && split == 1) || us < least) {
                least = us;
                best = {t, split};
            }
        }
    return best;
}
Move moved(int32_t dt) { return dt == PSATTN_BF16 ? kWhole : kFloat; }
// Logits: in parts of k where one workgroup to a tile would leave much of the chip idle and the parts are small beside W.  A whole step in us,
// whole / in parts: 4 items, vocabulary 2 423, hidden 5 632 109 / 65; 2 items, 1 021, 6 592 108 / 54; forward, 3 items, 3 013, 5 321 87 / 27; fp32,
// 224 items, 2 119, 1 577 129 / 48; but 14 items, 22 005 (172 tiles), 1 472 97 / 119
Tiling logits_tiling(int32_t dt, int64_t n_items, int64_t cols, int64_t hidden) {
    const int64_t steps = hidden / (dt == PSATTN_BF16 ? 64 : 32), bytes = 4 * n_items * up8(cols);
    const bool may_split = n_items <= kPartItems && bytes <= kPartBytes;
    Tiling t = tiling(moved(dt), n_items, cols, hidden, may_split);
    if (n_items <= 64) {
        const int64_t tiles = cdiv(cols, 128);
        t.split = tiles >= 128 ? 1 : std::max<int64_t>(1, std::min(512 / tiles, steps / 4));
    }
    t.split = may_split ? std::max<int64_t>(1, std::min(t.split, kPartBytes / std::max<int64_t>(bytes, 1))) : 1;
    return t;
}
size_t part_bytes(const Tiling& t, int64_t n_items, int64_t cols) { return t.split > 1 ? sizeof(float) * t.split * n_items * up8(cols) : 0; }

int head_product(int32_t dt, Pass pass, bool qkc, TileSize size, Product d, hipStream_t s) {
    d.odd = pass == kDlogit && !(at16({d.out[0]}) && d.ldo % 8 == 0 && d.N % 8 == 0);
    const int group = dt == PSATTN_BF16 ? 8 : 4;
    const bool whole = at16({d.p[0], d.q[0]}) && d.ldp % group == 0 && d.ldq % group == 0 && (qkc || d.n_load % group == 0);
    if (dt == PSATTN_BF16) return (whole ? head_product_bf16 : head_product_bf16_any)(pass, qkc, size, d, s);
    return (whole ? head_product_f32_whole : head_product_f32)(pass, qkc, size, d, s);
}

// Few items of bf16: dz as two numbers each, the second what the first one's rounding leaves, as items of their own.  The gradients are as
// exact as their own rounding then.  Of more items dz at their tokens alone is kept exact (psattn_head_dw_tokens)
constexpr int64_t kTwice = 32;
bool dz_apart(int32_t dt, int64_t n_items) { return dt == PSATTN_BF16 && n_items > kTwice; }
int64_t dz_rows(int32_t dt, int64_t n_items) { return dt == PSATTN_BF16 && n_items <= kTwice ? 2 * n_items : n_items; }
// dz of a piece of the vocabulary, whole steps of k for dW, has this much room at most.  A step's rows are then within the 32-bit offsets of
// the products' copies
constexpr int64_t kPieceBytes = int64_t{512} << 20;
int64_t piece_rows(int32_t dt, int64_t n_items, int64_t vocab) {
    const int64_t most = kPieceBytes / static_cast<int64_t>(elem_bytes(dt)) / std::max<int64_t>(up64(dz_rows(dt, n_items)), 64) / 256 * 256;
    if (most >= vocab) return vocab;
    const int64_t n = cdiv(vocab, std::max<int64_t>(most, 256));
    return cdiv(cdiv(vocab, n), 256) * 256;
}
constexpr int kManyParts = 16;
// dX's sums: k is a piece of the vocabulary, in parts where the rows' tiles are few.
// `both`: dX and dW of a piece in one launch, no part of k longer than half of what a CU has to do.  A whole step in us, apart / so: bf16, vocabulary
// 32 000, hidden 4 096, 300 tokens (60 in 100 predicted) 357 / 366, 600 500 / 510, 1 200 825 / 827, 2 400 1 406 / 1 347, 5 000 2 679 / 2 649; 16 384 tokens, 128 000
// the same (the chip's clock falls with what its matrix cores do); fp32, 20 000, 1 024: 300 tokens 506 / 454, 1 200 1 234 / 1 082, 3 000 2 992 / 2 590
struct DxTiling : Tiling {
    bool both;
};
DxTiling dx_tiling(int32_t dt, int64_t n_items, int64_t vocab, int64_t hidden) {
    const int64_t piece = piece_rows(dt, n_items, vocab);
    if (n_items >= (dt == PSATTN_BF16 ? 1024 : 65) && (dt != PSATTN_BF16 || hidden % 8 == 0)) {
        const int64_t k = dt == PSATTN_BF16 ? 64 : 32, side = dt == PSATTN_BF16 ? 256 : 128, slots = dt == PSATTN_BF16 ? 256 : 512;
        const int64_t x_tiles = cdiv(n_items, side) * cdiv(hidden, side), w_tiles = cdiv(piece, side) * cdiv(hidden, side);
        const int64_t x_steps = piece / k, share = (x_tiles * x_steps + w_tiles * (up64(n_items) / k)) / slots;
        return {{dt == PSATTN_BF16 ? k256 : k128, std::max<int64_t>(1, std::min<int64_t>(cdiv(2 * x_steps, std::max<int64_t>(share, 1)), x_steps / 8))}, true};
    }
    return {tiling(moved(dt), dz_rows(dt, n_items), hidden, piece, true), false};
}

// dW of many items and a small vocabulary has few tiles, each with all items for its k: in parts of the items, where a tile alone would take more
// steps of k than a workgroup's share of the launch, joined by psattn_head_dw_join.  Forward and backward in us, whole / in parts: 9 811 items,
// 1 200 x 512 bf16 349 / 235, fp32 984 / 613
int64_t dw_split(int32_t dt, int64_t n_items, int64_t vocab, int64_t hidden) {
    if (n_items < 1024) return 1;
    const int64_t piece = piece_rows(dt, n_items, vocab), k = dt == PSATTN_BF16 ? 64 : 32, side = dt == PSATTN_BF16 ? 256 : 128, slots = dt == PSATTN_BF16 ? 256 : 512;
    const int64_t steps = up64(n_items) / k, tiles = cdiv(piece, side) * cdiv(hidden, side);
    const int64_t beside = dx_tiling(dt, n_items, vocab, hidden).both ? cdiv(n_items, side) * cdiv(hidden, side) * (piece / k) : 0;
    const int64_t share = std::max<int64_t>(8, (beside + tiles * steps) / slots);
    return std::max<int64_t>(1, std::min(steps / share, kPartBytes / (static_cast<int64_t>(sizeof(float)) * piece * up8(hidden))));
}
size_t dw_part_bytes(int64_t split, int64_t piece, int64_t hidden) { return split > 1 ? sizeof(float) * split * piece * up8(hidden) : 0; }

struct Room {
    char* p;
    explicit Room(void* base) : p(reinterpret_cast<char*>(align_up(reinterpret_cast<uintptr_t>(base), 256))) {}
    template <typename T>
    T* take(size_t n) {
        T* const r = reinterpret_cast<T*>(p);
        p += align_up(n * sizeof(T), 256);
        return r;
    }
};

// a plan's tables are on the device that was current when it was made
bool elsewhere(const psattn_lp_plan* plan) {
    int device = -1;
    return hipGetDevice(&device) == hipSuccess && device != plan->device;
}
bool bad_shape(const psattn_lp_plan* plan, int32_t dt, int32_t vocab, int32_t hidden) {
    return !plan || (dt != PSATTN_F32 && dt != PSATTN_BF16) || vocab <= 0 || hidden <= 0;
}
// a tile's copies have 32-bit offsets, and grids stay below 2^31 threads
bool too_large(const psattn_lp_plan* plan, int32_t dt, int64_t vocab, int64_t hidden, bool bwd) {
    const int64_t n = plan->n_items;
    if (hidden * static_cast<int64_t>(elem_bytes(dt)) * 256 >= (int64_t{1} << 31) || n > (int64_t{1} << 23) - 128 || vocab > INT32_MAX - 512) return true;
    auto fits = [](int64_t M, int64_t N, TileSize t) {
        static constexpr int bm[] = {32, 64, 128, 256}, bn[] = {128, 128, 128, 256}, threads[] = {128, 128, 256, 512};
        return cdiv(M, bm[t]) * cdiv(N, bn[t]) < (int64_t{1} << 31) / threads[t];
    };
    if (!bwd) return !fits(n, vocab, logits_tiling(dt, n, vocab, hidden).size);
    const int64_t piece = piece_rows(dt, n, vocab);
    return !fits(n, piece, logits_tiling(dt, n, piece, hidden).size) || !fits(n, hidden, dx_tiling(dt, n, vocab, hidden).size) || !fits(piece, hidden, k128);
}

size_t fwd_bytes(const psattn_lp_plan* plan, int32_t dt, int32_t vocab, int32_t hidden) {
    if (bad_shape(plan, dt, vocab, hidden)) return 0;
    const size_t n = static_cast<size_t>(plan->n_items);
    const size_t parts = std::max(part_bytes(logits_tiling(dt, n, vocab, hidden), n, vocab), n * cdiv(vocab, 128) * sizeof(float2));
    return align_up(n * up8(hidden) * elem_bytes(dt), 256) + align_up(parts, 256) + 4 * align_up(n * 4, 256) + 256;
}
// parts of the logits of a piece, or of the last one, which is smaller
size_t logits_bytes(int32_t dt, int64_t n, int64_t vocab, int64_t piece, int64_t hidden) {
    const int64_t last = vocab - (vocab - 1) / piece * piece;
    return std::max(part_bytes(logits_tiling(dt, n, piece, hidden), n, piece), part_bytes(logits_tiling(dt, n, last, hidden), n, last));
}
size_t bwd_bytes(const psattn_lp_plan* plan, int32_t dt, int32_t vocab, int32_t hidden) {
    if (bad_shape(plan, dt, vocab, hidden)) return 0;
    const size_t n = static_cast<size_t>(plan->n_items);
    const int64_t m = dz_rows(dt, n), piece = piece_rows(dt, n, vocab);
    const size_t sums = m * up8(hidden) * dx_tiling(dt, n, vocab, hidden).split * sizeof(float), parts = logits_bytes(dt, n, vocab, piece, hidden);
    return align_up(up64(m) * up8(hidden) * elem_bytes(dt), 256) + align_up(up64(m) * up8(piece) * elem_bytes(dt), 256) + align_up(sums, 256) + align_up(parts, 256) +
           align_up(dw_part_bytes(dw_split(dt, n, vocab, hidden), piece, hidden), 256) + 4 * align_up(n * 4, 256) + 256 +
           (dz_apart(dt, n) ? align_up(vocab * sizeof(int32_t), 256) : 0);
}

}  // namespace

extern "C" {

size_t psattn_head_logprob_fwd_workspace_bytes(const psattn_lp_plan* plan, int32_t dt, int32_t vocab, int32_t hidden) { return fwd_bytes(plan, dt, vocab, hidden); }

size_t psattn_head_logprob_bwd_workspace_bytes(const psattn_lp_plan* plan, int32_t dt, int32_t vocab, int32_t hidden) { return bwd_bytes(plan, dt, vocab, hidden); }

int psattn_head_logprob_fwd(const psattn_lp_plan* plan, int32_t dt, int32_t vocab, int32_t hidden, const void* X, const void* W, const int32_t* token_ids, float* row_lse,
                            float* resp_logp, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (bad_shape(plan, dt, vocab, hidden)) return PSATTN_EINVAL;
    if (plan->n_resp == 0) return PSATTN_OK;
    if (!X || !W || !token_ids || !row_lse || !resp_logp || !workspace || workspace_bytes < fwd_bytes(plan, dt, vocab, hidden)) return PSATTN_EINVAL;
    if (too_large(plan, dt, vocab, hidden, false)) return PSATTN_EUNSUPPORTED;
    if (elsewhere(plan)) return PSATTN_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const int n = static_cast<int>(plan->n_items);
    Room room(workspace);
    char* const x = room.take<char>(static_cast<size_t>(n) * up8(hidden) * elem_bytes(dt));
    const Tiling tiling = logits_tiling(dt, n, vocab, hidden);
    float2* const part = reinterpret_cast<float2*>(room.take<char>(std::max(part_bytes(tiling, n, vocab), n * cdiv(vocab, 128) * sizeof(float2))));
    int32_t *const target = room.take<int32_t>(n), *const item_row = room.take<int32_t>(n);
    float *const hit = room.take<float>(n), *const logp = room.take<float>(n);
    constexpr int kFewItems = 4;
    if (n > 0) {
        auto gather = [&](auto* to) {
            using E = std::remove_pointer_t<decltype(to)>;
            psattn_head_rows<E, false><<<n, row_threads(dt, hidden), 0, s>>>(n, n, {plan->n_resp, plan->item_ptr, plan->resp_first, plan->resp_prev}, item_row, token_ids, vocab, hidden, static_cast<const E*>(X),
                                                         nullptr, nullptr, to, target, nullptr, nullptr, nullptr, nullptr, nullptr, 0);
        };
        if (dt == PSATTN_BF16) gather(reinterpret_cast<uint16_t*>(x));
        else gather(reinterpret_cast<float*>(x));
        Product z{};
        z.p[0] = x; z.q[0] = W; z.G = reinterpret_cast<float*>(part); z.U = hit; z.H = target;
        z.ldp = up8(hidden); z.ldq = hidden;
        z.M = n; z.N = vocab; z.K = hidden; z.n_seg = z.n_prod = z.n_split = 1;
        int rc;
        if (tiling.split > 1) {
            z.parts = reinterpret_cast<float*>(part); z.ld_part = up8(vocab); z.n_split = static_cast<int32_t>(tiling.split);
            if ((rc = head_product(dt, kSums, true, tiling.size, z, s)) != PSATTN_OK) return rc;
            psattn_head_parts_lse<<<n, 1024, 0, s>>>(n, z.n_split, vocab, z.ld_part, z.parts, item_row, target, row_lse, logp);
        } else {
            if ((rc = head_product(dt, kLse, true, tiling.size, z, s)) != PSATTN_OK) return rc;
            const int parts = static_cast<int>(cdiv(vocab, tiling.size == k256 ? 256 : 128));
            if (n <= kFewItems && plan->n_resp <= kFewItems) {
                psattn_head_join_few<<<plan->n_resp, 256, 0, s>>>(n, parts, part, item_row, plan->item_ptr, target, hit, row_lse, resp_logp);
                return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
            }
            if (n <= 256) psattn_head_join<1><<<n, 256, 0, s>>>(n, parts, part, item_row, target, hit, row_lse, logp);
            else psattn_head_join<16><<<static_cast<uint32_t>(cdiv(n, 16)), 256, 0, s>>>(n, parts, part, item_row, target, hit, row_lse, logp);
        }
    }
    in_grids(plan->n_resp, 256, [&](int64_t at, uint32_t grid) { psattn_head_responses<<<grid, 256, 0, s>>>(static_cast<int>(at), plan->item_ptr, logp, resp_logp); });
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

int psattn_head_logprob_bwd(const psattn_lp_plan* plan, int32_t dt, int32_t vocab, int32_t hidden, const void* X, const void* W, const int32_t* token_ids,
                            const float* row_lse, const float* d_resp_logp, void* dX, void* dW, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (bad_shape(plan, dt, vocab, hidden) || !dW) return PSATTN_EINVAL;
    if (plan->T > 0 && !dX) return PSATTN_EINVAL;
    const int n = static_cast<int>(plan->n_items);
    if (n > 0 && (!X || !W || !token_ids || !row_lse || !d_resp_logp || !workspace || workspace_bytes < bwd_bytes(plan, dt, vocab, hidden))) return PSATTN_EINVAL;
    if (too_large(plan, dt, vocab, hidden, true)) return PSATTN_EUNSUPPORTED;
    if (plan->T > 0 && elsewhere(plan)) return PSATTN_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const size_t e = elem_bytes(dt);
    Room room(workspace);
    const DxTiling dx = dx_tiling(dt, n, vocab, hidden);
    const int parts = static_cast<int>(dx.split);
    const int64_t ld = up8(hidden), piece = piece_rows(dt, n, vocab), ldz = up8(piece);
    const int again = static_cast<int>(dz_rows(dt, n)), n_whole = static_cast<int>(up64(again));
    const bool apart = dz_apart(dt, n);  // dz at the items' tokens
    uint16_t* const rest_w = static_cast<uint16_t*>(dX);  // written last, and an item's row in it free until then: there are no more items than tokens
    float *sums = nullptr, *at_token = nullptr;
    const float* weights = nullptr;
    const int32_t *target = nullptr, *item_of = nullptr;
    const uint16_t* x_rows = nullptr;
    if (n == 0) {  // nothing is predicted: sums over nothing
        psattn_head_zero<<<1024, 256, 0, s>>>(static_cast<uint16_t*>(dW), static_cast<size_t>(vocab) * hidden * e / 2);
    } else {
        char* const x = room.take<char>(static_cast<size_t>(n_whole) * ld * e);
        x_rows = reinterpret_cast<const uint16_t*>(x);
        char* const dz = room.take<char>(static_cast<size_t>(n_whole) * ldz * e);
        sums = room.take<float>(static_cast<size_t>(again) * ld * parts);
        float* const z_parts = reinterpret_cast<float*>(room.take<char>(logits_bytes(dt, n, vocab, piece, hidden)));
        const int64_t w_split = dw_split(dt, n, vocab, hidden);
        float* const w_parts = reinterpret_cast<float*>(room.take<char>(dw_part_bytes(w_split, piece, hidden)));
        char* const rest = again > n ? dz + n * ldz * e : nullptr;
        int32_t* const targets = room.take<int32_t>(n);
        float *const lse = room.take<float>(n), *const weight = room.take<float>(n);
        at_token = room.take<float>(n);
        target = targets;
        weights = weight;
        int32_t* const items = apart ? room.take<int32_t>(vocab) : nullptr;
        item_of = items;
        auto gather = [&](auto* to) {
            using E = std::remove_pointer_t<decltype(to)>;
            psattn_head_rows<E, true><<<n_whole, row_threads(dt, hidden), 0, s>>>(n, again, {plan->n_resp, plan->item_ptr, plan->resp_first, plan->resp_prev}, nullptr, token_ids, vocab, hidden, static_cast<const E*>(X),
                                                              row_lse, d_resp_logp, to, targets, lse, weight, at_token, items, reinterpret_cast<E*>(dz), ldz);
        };
        if (dt == PSATTN_BF16) gather(reinterpret_cast<uint16_t*>(x));
        else gather(reinterpret_cast<float*>(x));
        for (int64_t at = 0; at < vocab; at += piece) {
            const int32_t cols = static_cast<int32_t>(std::min<int64_t>(piece, vocab - at));
            const char* const w = static_cast<const char*>(W) + at * hidden * e;
            int rc;
            Product z{};  // dz
            z.p[0] = x; z.q[0] = w; z.G = lse; z.U = weight; z.H = targets; z.out[0] = dz; z.out[1] = rest; z.parts = apart ? at_token : nullptr; z.item_of = items;
            z.ldp = ld; z.ldq = hidden; z.ldo = ldz;
            z.M = n; z.N = cols; z.K = hidden; z.n_seg = z.n_prod = z.n_split = 1;
            z.n_load = static_cast<int32_t>(at);
            const Tiling tiling = logits_tiling(dt, n, cols, hidden);
            if (tiling.split > 1) {
                z.parts = z_parts; z.ld_part = up8(cols); z.n_split = static_cast<int32_t>(tiling.split);
                if ((rc = head_product(dt, kSums, true, tiling.size, z, s)) != PSATTN_OK) return rc;
                auto go = [&](auto* to) {
                    using E = std::remove_pointer_t<decltype(to)>;
                    psattn_head_parts_dz<E><<<dim3(static_cast<uint32_t>(cdiv(cols, 1024)), n), 256, 0, s>>>(n, z.n_split, static_cast<int>(at), cols, z.ld_part, z_parts, targets, lse,
                                                                                                            weight, to, reinterpret_cast<E*>(rest), apart ? at_token : nullptr, items, ldz);
                };
                if (dt == PSATTN_BF16) go(reinterpret_cast<uint16_t*>(dz));
                else go(reinterpret_cast<float*>(dz));
            } else if ((rc = head_product(dt, kDlogit, true, tiling.size, z, s)) != PSATTN_OK) {
                return rc;
            }
            Product a{};  // dX += dz W
            a.p[0] = dz; a.q[0] = w; a.parts = sums; a.ld_part = ld; a.add = at > 0;
            a.ldp = ldz; a.ldq = hidden;
            a.M = again; a.N = a.n_load = hidden; a.K = cols; a.n_seg = a.n_prod = 1; a.n_split = parts;
            Product g{};  // dW = dz^T X
            g.p[0] = dz; g.q[0] = x; g.out[0] = static_cast<char*>(dW) + at * hidden * e;
            g.ldp = ldz; g.ldq = ld; g.ldo = hidden;
            g.M = cols; g.m_load = static_cast<int32_t>(up8(cols)); g.N = hidden; g.n_load = static_cast<int32_t>(ld); g.K = n_whole; g.n_seg = g.n_prod = 1;
            g.n_split = static_cast<int32_t>(w_split); g.parts = w_parts; g.ld_part = ld;
            if (apart) g.out[1] = rest_w, g.H = items + at;
            g.odd = !(at16({g.out[0]}) && hidden % (dt == PSATTN_BF16 ? 8 : 4) == 0);
            const bool whole = at16({w}) && hidden % (dt == PSATTN_BF16 ? 8 : 4) == 0;
            if (dx.both && (whole || dt != PSATTN_BF16)) {
                rc = (dt == PSATTN_BF16 ? head_grads_bf16 : whole ? head_grads_f32_whole : head_grads_f32)(a, g, s);
            } else if ((rc = head_product(dt, kSums, false, dx.size, a, s)) != PSATTN_OK) {
                return rc;
            } else if (n_whole <= (dt == PSATTN_BF16 ? 256 : 64)) {
                g.K = again;
                rc = (dt == PSATTN_BF16 ? head_outer_bf16 : head_outer_f32)(g, s);
            } else {  // bf16: fp32 takes one way or the other above
                auto us = [&](TileSize t, int64_t side) { return product_us(kWhole, kPlain, t, cdiv(cols, side) * cdiv(hidden, side), n_whole / 64, w_split, 0); };
                rc = head_tokens_bf16(cdiv(cols, 256) * cdiv(hidden, 256) >= 256 || us(k256, 256) < us(k128, 128) ? k256 : k128, g, s);
            }
            if (rc != PSATTN_OK) return rc;
            if (w_split > 1) {  // 1 024 items and more
                const int64_t groups = static_cast<int64_t>(cols) * (ld / 4);
                auto join = [&](auto* to) {
                    using E = std::remove_pointer_t<decltype(to)>;
                    psattn_head_dw_join<E><<<static_cast<uint32_t>(cdiv(groups, 256)), 256, 0, s>>>(static_cast<int>(w_split), cols, hidden, ld, w_parts, g.odd, to, apart ? items + at : nullptr, reinterpret_cast<E*>(rest_w));
                };
                if (dt == PSATTN_BF16) join(static_cast<uint16_t*>(g.out[0]));
                else join(static_cast<float*>(g.out[0]));
            }
        }
    }
    if (apart) {
        int lanes = 4;
        while (lanes < 256 && lanes * 4 < hidden) lanes *= 2;
        const int blocks = static_cast<int>(cdiv(hidden, lanes * 4));
        const int64_t most = ((int64_t{1} << 31) - 1) / 256 / blocks;
        for (int64_t at = 0; at < n; at += most)
            psattn_head_dw_tokens<<<static_cast<uint32_t>(std::min<int64_t>(most, n - at) * blocks), 256, 0, s>>>(static_cast<int>(at), lanes, blocks, n, hidden, ld, target, item_of, at_token,
                                                                                                                          x_rows, rest_w, static_cast<uint16_t*>(dW));
    }
    // a row to a workgroup; where they are few, 1 024 columns of one, or with many parts 256
    const bool many = n <= 64 && parts * (again / std::max(n, 1)) >= kManyParts && plan->T < 4096;
    const int col_blocks = many ? static_cast<int>(cdiv(hidden, 256)) : plan->T < 4096 ? static_cast<int>(cdiv(hidden, 1024)) : 1;
    in_grids(static_cast<int64_t>(plan->T) * col_blocks, many ? 1024 : 256, [&](int64_t at, uint32_t grid) {
        auto go = [&](auto* to) {
            using E = std::remove_pointer_t<decltype(to)>;
            auto kernel = many ? psattn_head_dx_parts<E> : psattn_head_dx<E>;
            kernel<<<grid, many ? 1024 : 256, 0, s>>>(at, col_blocks, hidden, n, again, parts, ld, sums, plan->row_desc, plan->resp_first, plan->resp_len, plan->resp_prev,
                                                     plan->samp_ptr, plan->item_ptr, target, weights, apart ? at_token : nullptr, static_cast<const E*>(W), to);
        };
        if (dt == PSATTN_BF16) go(static_cast<uint16_t*>(dX));
        else go(static_cast<float*>(dX));
    });
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

}  // extern "C"
