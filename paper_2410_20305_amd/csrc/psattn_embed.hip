// Embedding rows by token id, scaled, and the gradient of the table.
//   X[t] = scale W[id_t],  dW[v] = scale sum of dX[t] over the tokens t with id_t = v, in the order of the tokens, in fp32
// A token whose id is not in [0, vocab) (padding) has a row of zeros and gives no gradient.
//
// Both are bound by HBM.  The gradient sorts the tokens by id (stable, so that a row's tokens stay in their order), cuts the sorted
// tokens into pieces of kPiece, whatever ids they have, and adds up runs of one id within a piece: a frequent id is many
// pieces' work and a rare one no workgroup's own.  Runs that reach past a piece leave fp32 sums, which are joined in order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "psattn.h"
#include "psattn_rows.h"

namespace {

using namespace psattn::rows;

constexpr int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int kThreads = 256;

template <typename E, bool WHOLE>
__global__ __launch_bounds__(kThreads) void psattn_embed_rows(int n_tokens, int hidden, int vocab, float scale, const int32_t* ids, const E* W, E* X) {
    constexpr int V = kVec<E>;
    const int groups = (hidden + V - 1) / V, per = (groups + kThreads - 1) / kThreads;  // workgroups of a row
    const int64_t n = static_cast<int64_t>(n_tokens) * per;
    for (int64_t b = blockIdx.x; b < n; b += gridDim.x) {
        const int t = static_cast<int>(b / per), c = (static_cast<int>(b % per) * kThreads + threadIdx.x) * V;
        if (c >= hidden) continue;
        const int id = ids[t];
        float x[V] = {};
        if (id >= 0 && id < vocab) {
            load<WHOLE>(W + static_cast<int64_t>(id) * hidden, c, hidden, x);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] *= scale;
        }
        store<WHOLE>(X + static_cast<int64_t>(t) * hidden, c, hidden, x);
    }
}

// ---- tokens sorted by id
// Up to kRankMost tokens: a token's place is the number of tokens that come before it, counted by four lanes over all keys, which
// fit LDS.  One launch instead of six, and no chain of barriers.
//
// More: passes over the id's digits, least first, each stable: the digit's counts in every block of kBlock tokens, their running sums
// over digits and blocks (by the one workgroup of a kernel of its own), and each token to its place.  Ids outside the table count as
// `vocab`, so that they end up behind all others.
constexpr int kBlock = 2048, kSortThreads = 512, kEach = kBlock / kSortThreads;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;

__device__ __forceinline__ uint32_t key_of(int id, int vocab) { return id >= 0 && id < vocab ? static_cast<uint32_t>(id) : static_cast<uint32_t>(vocab); }

// counts[digit][block]
__global__ __launch_bounds__(kSortThreads) void psattn_embed_count(int n, int vocab, int shift, bool ids_are_keys, const int32_t* ids, uint32_t* counts) {
    __shared__ uint32_t hist[kDigits];
    for (int i = threadIdx.x; i < kDigits; i += kSortThreads) hist[i] = 0;
    __syncthreads();
    const int at = blockIdx.x * kBlock;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int i = at + e * kSortThreads + threadIdx.x;
        if (i < n) atomicAdd(&hist[((ids_are_keys ? static_cast<uint32_t>(ids[i]) : key_of(ids[i], vocab)) >> shift) & (kDigits - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kDigits; i += kSortThreads) counts[static_cast<size_t>(i) * gridDim.x + blockIdx.x] = hist[i];
}

// running sums, in place
__global__ __launch_bounds__(1024) void psattn_embed_scan(int n, uint32_t* counts) {
    __shared__ uint32_t sums[16];
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t base = 0;
    for (int at = 0; at < n; at += 4096) {
        uint32_t v[4], t = 0;
        const int i = at + 4 * threadIdx.x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = i + j < n ? counts[i + j] : 0;
            t += v[j];
        }
        uint32_t run = t;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t u = __shfl_up(run, off);
            if (l >= off) run += u;
        }
        if (l == 63) sums[w] = run;
        __syncthreads();
        uint32_t before = base, all = 0;
        for (int k = 0; k < 16; ++k) {
            if (k < w) before += sums[k];
            all += sums[k];
        }
        uint32_t x = before + run - t;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (i + j < n) counts[i + j] = x;
            x += v[j];
        }
        base += all;
        __syncthreads();
    }
}

// Each token to its place.  Within a block, threads hold neighbouring tokens in turn (round e: tokens e kSortThreads ..), and a
// token's place among those of its digit is the count of earlier rounds and waves plus that of lower lanes.
__global__ __launch_bounds__(kSortThreads) void psattn_embed_place(int n, int vocab, int shift, bool first, const int32_t* ids, const int32_t* tokens,
                                                                   const uint32_t* offsets, int32_t* out_keys, int32_t* out_tokens) {
    constexpr int kWaves = kSortThreads / 64;
    __shared__ uint32_t next[kDigits];             // where the digit's next token goes
    __shared__ uint16_t wave_count[kWaves][kDigits];  // of this round
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6, at = blockIdx.x * kBlock;
    for (int i = threadIdx.x; i < kDigits; i += kSortThreads) next[i] = offsets[static_cast<size_t>(i) * gridDim.x + blockIdx.x];
    for (int e = 0; e < kEach; ++e) {
        for (int i = threadIdx.x; i < kWaves * kDigits; i += kSortThreads) (&wave_count[0][0])[i] = 0;
        __syncthreads();
        const int i = at + e * kSortThreads + threadIdx.x;
        const bool real = i < n;
        const uint32_t key = !real ? 0 : first ? key_of(ids[i], vocab) : static_cast<uint32_t>(ids[i]);
        const uint32_t digit = (key >> shift) & (kDigits - 1);
        // lanes with the same digit
        uint64_t same = __ballot(real);
#pragma unroll
        for (int b = 0; b < kDigitBits; ++b) {
            const uint64_t one = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? one : ~one;
        }
        const int below = __popcll(same & ((1ull << l) - 1));
        if (real && below == 0) wave_count[w][digit] = static_cast<uint16_t>(__popcll(same));
        __syncthreads();
        if (real) {
            uint32_t to = next[digit] + below;
            for (int k = 0; k < w; ++k) to += wave_count[k][digit];
            out_keys[to] = static_cast<int32_t>(key);
            out_tokens[to] = first ? i : tokens[i];
        }
        __syncthreads();
        for (int d = threadIdx.x; d < kDigits; d += kSortThreads) {
            uint32_t t = 0;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) t += wave_count[k][d];
            next[d] += t;
        }
        // the counts are cleared behind the reads above, and `next` is read behind the next round's first barrier
        __syncthreads();
    }
}

constexpr int kRankMost = 4096;

__global__ __launch_bounds__(kThreads) void psattn_embed_rank(int n, int vocab, const int32_t* ids, int32_t* out_keys, int32_t* out_tokens) {
    __shared__ __attribute__((aligned(16))) uint32_t key[kRankMost];
    const int padded = (n + 15) / 16 * 16;
    for (int i = threadIdx.x; i < padded; i += kThreads) key[i] = i < n ? key_of(ids[i], vocab) : 0xffffffffu;  // behind all
    __syncthreads();
    const int t = blockIdx.x * (kThreads / 4) + (threadIdx.x >> 2);
    const uint32_t mine = key[min(t, n - 1)];
    int before = 0;
    for (int i = 4 * (threadIdx.x & 3); i < padded; i += 16) {
        const uint4 k = *reinterpret_cast<const uint4*>(&key[i]);
        before += (k.x < mine || (k.x == mine && i < t)) + (k.y < mine || (k.y == mine && i + 1 < t)) + (k.z < mine || (k.z == mine && i + 2 < t)) +
                  (k.w < mine || (k.w == mine && i + 3 < t));
    }
    before += __shfl_xor(before, 1);
    before += __shfl_xor(before, 2);
    if (t < n && (threadIdx.x & 3) == 0) {
        out_keys[before] = static_cast<int32_t>(mine);
        out_tokens[before] = t;
    }
}

// ---- sums of runs, and zeros for the other rows
constexpr int kPiece = 32, kZeroRows = 16;

// Workgroups up to n_sums: a piece of sorted tokens and kThreads groups of columns.  Sums of the piece's first run, if it came from the
// piece before, and of its last, if it goes on, to edge[piece][0 / 1]; a run that does both to edge[piece][0].  Those behind: kZeroRows
// rows of the table, of which each that has no token (found by bisection) becomes zeros.
template <typename E, bool WHOLE>
__global__ __launch_bounds__(kThreads) void psattn_embed_sum(int n, int vocab, int hidden, float scale, const int32_t* keys, const int32_t* tokens, const E* dX,
                                                             E* dW, float* edge, int n_sums, int column_groups) {
    constexpr int V = kVec<E>;
    __shared__ int32_t key[kPiece + 2], tok[kPiece];
    if (static_cast<int>(blockIdx.x) >= n_sums) {
        const int v0 = (blockIdx.x - n_sums) * kZeroRows;
        if (threadIdx.x < kZeroRows) {
            const int v = v0 + threadIdx.x;
            int lo = 0, hi = n;  // the first sorted token with an id of v and more
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (keys[mid] < v) lo = mid + 1;
                else hi = mid;
            }
            tok[threadIdx.x] = v < vocab && !(lo < n && keys[lo] == v);
        }
        __syncthreads();
        const float z[V] = {};
        for (int r = 0; r < kZeroRows; ++r)
            if (tok[r])
                for (int c = threadIdx.x * V; c < hidden; c += kThreads * V) store<WHOLE>(dW + static_cast<int64_t>(v0 + r) * hidden, c, hidden, z);
        return;
    }
    const int piece = blockIdx.x / column_groups, at = piece * kPiece, m = min(kPiece, n - at);
    for (int i = threadIdx.x; i < m + 2; i += kThreads) {
        const int j = at + i - 1;
        key[i] = j >= 0 && j < n ? keys[j] : -1;
        if (i < m) tok[i] = tokens[at + i];
    }
    __syncthreads();
    const int c = (blockIdx.x % column_groups * kThreads + threadIdx.x) * V;
    if (c >= hidden) return;
    for (int i = 0; i < m;) {
        const int v = key[i + 1];
        if (v >= vocab) return;  // padding, behind all others
        int end = i + 1;
        while (end < m && key[end + 1] == v) ++end;
        float sum[V] = {};
        int j = i;
        for (; j + 4 <= end; j += 4) {
            u32x4 x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = raw<WHOLE>(dX + static_cast<int64_t>(tok[j + u]) * hidden, c, hidden);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float y[V];
                unpack(x[u], y);
#pragma unroll
                for (int k = 0; k < V; ++k) sum[k] += y[k];
            }
        }
        for (; j < end; ++j) {
            float x[V];
            load<WHOLE>(dX + static_cast<int64_t>(tok[j]) * hidden, c, hidden, x);
#pragma unroll
            for (int k = 0; k < V; ++k) sum[k] += x[k];
        }
        const bool before = i == 0 && key[0] == v, behind = end == m && key[m + 1] == v;
        if (before || behind) {
            float* const to = edge + (2 * static_cast<int64_t>(piece) + (before ? 0 : 1)) * hidden + c;
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (WHOLE || c + k < hidden) to[k] = sum[k];
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) sum[k] *= scale;
            store<WHOLE>(dW + static_cast<int64_t>(v) * hidden, c, hidden, sum);
        }
        i = end;
    }
}

// The run that a piece's last token starts and the next pieces go on with: its sums in the order of the pieces
template <typename E>
__global__ __launch_bounds__(kThreads) void psattn_embed_join(int n, int vocab, int hidden, float scale, const int32_t* keys, const float* edge, E* dW) {
    const int p = blockIdx.x, last = p * kPiece + kPiece - 1;
    if (last + 1 >= n) return;
    const int v = keys[last];
    if (v >= vocab || keys[last + 1] != v) return;                   // ends here
    if (keys[p * kPiece] == v && p > 0 && keys[p * kPiece - 1] == v) return;  // started before
    int end = p + 1;  // behind the last piece that the run reaches
    while (end * kPiece < n && keys[end * kPiece] == v) ++end;
    for (int c = threadIdx.x + blockIdx.y * kThreads; c < hidden; c += kThreads * gridDim.y) {
        float sum = edge[(2 * static_cast<int64_t>(p) + 1) * hidden + c];
        int q = p + 1;
        for (; q + 8 <= end; q += 8) {  // loads together, sums in order
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = edge[2 * static_cast<int64_t>(q + u) * hidden + c];
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += x[u];
        }
        for (; q < end; ++q) sum += edge[2 * static_cast<int64_t>(q) * hidden + c];
        store1(dW + static_cast<int64_t>(v) * hidden + c, sum * scale);
    }
}

bool bad_shape(int32_t dt, int32_t n_tokens, int32_t vocab, int32_t hidden, float scale) {
    return (dt != PSATTN_F32 && dt != PSATTN_BF16) || n_tokens < 0 || vocab <= 0 || hidden <= 0 || !std::isfinite(scale);
}

// the backward's workspace
struct Slots {
    int32_t *keys[2], *tokens[2];
    uint32_t* counts;
    float* edge;
    size_t total;
};
Slots carve(int32_t n, int32_t hidden, void* base) {
    Slots s{};
    char *p = reinterpret_cast<char*>(align_up(reinterpret_cast<uintptr_t>(base), 256)), *const p0 = p;
    auto take = [&](size_t bytes) { char* r = p; p += align_up(bytes, 256); return r; };
    for (int i = 0; i < 2; ++i) {
        s.keys[i] = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * n));
        s.tokens[i] = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * n));
    }
    s.counts = reinterpret_cast<uint32_t*>(take(sizeof(uint32_t) * kDigits * cdiv(n, kBlock)));
    s.edge = reinterpret_cast<float*>(take(sizeof(float) * 2 * cdiv(n, kPiece) * hidden));
    s.total = static_cast<size_t>(p - p0) + 256;
    return s;
}

template <typename E>
void rows(int32_t n, int32_t vocab, int32_t hidden, float scale, const int32_t* ids, const void* W, void* X, hipStream_t s) {
    const E* w = static_cast<const E*>(W);
    E* x = static_cast<E*>(X);
    const int64_t blocks = n * cdiv(cdiv(hidden, kVec<E>), kThreads);
    const int grid = static_cast<int>(std::min<int64_t>(blocks, 1 << 20));
    if (whole<E>(hidden, {W, X})) psattn_embed_rows<E, true><<<grid, kThreads, 0, s>>>(n, hidden, vocab, scale, ids, w, x);
    else psattn_embed_rows<E, false><<<grid, kThreads, 0, s>>>(n, hidden, vocab, scale, ids, w, x);
}

template <typename E>
void grad(int32_t n, int32_t vocab, int32_t hidden, float scale, const int32_t* ids, const void* dX_, void* dW_, void* workspace, hipStream_t s) {
    const E* dX = static_cast<const E*>(dX_);
    E* dW = static_cast<E*>(dW_);
    const Slots w = carve(n, hidden, workspace);
    const int32_t *keys = ids, *tokens = nullptr;
    if (n > kRankMost) {
        const int blocks = static_cast<int>(cdiv(n, kBlock));
        int bits = 1;
        while (bits < 31 && (vocab >> bits) != 0) ++bits;  // keys are 0 .. vocab
        for (int shift = 0, turn = 0; shift < bits; shift += kDigitBits, turn ^= 1) {
            psattn_embed_count<<<blocks, kSortThreads, 0, s>>>(n, vocab, shift, shift > 0, keys, w.counts);
            psattn_embed_scan<<<1, 1024, 0, s>>>(kDigits * blocks, w.counts);
            psattn_embed_place<<<blocks, kSortThreads, 0, s>>>(n, vocab, shift, shift == 0, keys, tokens, w.counts, w.keys[turn], w.tokens[turn]);
            keys = w.keys[turn];
            tokens = w.tokens[turn];
        }
    } else if (n > 0) {
        psattn_embed_rank<<<static_cast<uint32_t>(cdiv(n, kThreads / 4)), kThreads, 0, s>>>(n, vocab, ids, w.keys[0], w.tokens[0]);
        keys = w.keys[0];
        tokens = w.tokens[0];
    }
    const int groups = static_cast<int>(cdiv(cdiv(hidden, kVec<E>), kThreads));
    const int64_t sums = cdiv(n, kPiece) * groups, zeros = cdiv(vocab, kZeroRows);
    auto sum = [&](auto kernel) {
        kernel<<<static_cast<uint32_t>(sums + zeros), kThreads, 0, s>>>(n, vocab, hidden, scale, keys, tokens, dX, dW, w.edge, static_cast<int>(sums), groups);
    };
    if (whole<E>(hidden, {dX, dW})) sum(psattn_embed_sum<E, true>);
    else sum(psattn_embed_sum<E, false>);
    if (n > kPiece) psattn_embed_join<E><<<dim3(static_cast<uint32_t>(cdiv(n, kPiece)), static_cast<uint32_t>(std::min<int64_t>(cdiv(hidden, kThreads), 64))), kThreads, 0, s>>>(n, vocab, hidden, scale, keys, w.edge, dW);
}

// grids below 2^31 threads, and table rows found by int
bool too_large(int32_t n_tokens, int32_t vocab, int32_t hidden) {
    return n_tokens > (1 << 24) || hidden > (1 << 23) || cdiv(n_tokens, kPiece) * cdiv(hidden, kThreads) + cdiv(vocab, kZeroRows) >= (1 << 23) || vocab == INT32_MAX;
}

}  // namespace

extern "C" {

int psattn_embed_fwd(int32_t dt, int32_t n_tokens, int32_t vocab, int32_t hidden, float scale, const int32_t* token_ids, const void* W, void* X,
                     void* hip_stream) {
    if (bad_shape(dt, n_tokens, vocab, hidden, scale)) return PSATTN_EINVAL;
    if (n_tokens == 0) return PSATTN_OK;
    if (!token_ids || !W || !X) return PSATTN_EINVAL;
    if (too_large(n_tokens, vocab, hidden)) return PSATTN_EUNSUPPORTED;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dt == PSATTN_BF16) rows<uint16_t>(n_tokens, vocab, hidden, scale, token_ids, W, X, s);
    else rows<float>(n_tokens, vocab, hidden, scale, token_ids, W, X, s);
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

size_t psattn_embed_bwd_workspace_bytes(int32_t dt, int32_t n_tokens, int32_t vocab, int32_t hidden) {
    if (bad_shape(dt, n_tokens, vocab, hidden, 1.f)) return 0;
    return carve(n_tokens, hidden, nullptr).total;
}

int psattn_embed_bwd(int32_t dt, int32_t n_tokens, int32_t vocab, int32_t hidden, float scale, const int32_t* token_ids, const void* dX, void* dW,
                     void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (bad_shape(dt, n_tokens, vocab, hidden, scale) || !dW || (n_tokens > 0 && (!token_ids || !dX))) return PSATTN_EINVAL;
    if (!workspace || workspace_bytes < psattn_embed_bwd_workspace_bytes(dt, n_tokens, vocab, hidden)) return PSATTN_EINVAL;
    if (too_large(n_tokens, vocab, hidden)) return PSATTN_EUNSUPPORTED;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dt == PSATTN_BF16) grad<uint16_t>(n_tokens, vocab, hidden, scale, token_ids, dX, dW, workspace, s);
    else grad<float>(n_tokens, vocab, hidden, scale, token_ids, dX, dW, workspace, s);
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

}  // extern "C"
