// Embedding rows by token id, scaled, and the gradient of the table.
//   X[t] = scale W[id_t],  dW[v] = scale sum of dX[t] over the tokens t with id_t = v, in fp32
// A token whose id is not in [0, vocab) (padding) has a row of zeros and gives no gradient.
//
// Both are bound by HBM.  The gradient sorts the tokens by id (stable, so that a row's tokens stay in their order), cuts the sorted
// tokens into pieces of one size, whatever ids they have, and adds up runs of one id within a piece: a frequent id is many
// pieces' work and a rare one no workgroup's own.  Within a piece a row's tokens are added one by one in their order.  Runs that reach
// past a piece leave fp32 sums, which are joined in an order of their own (psattn_embed_join): ids and sizes decide it, and which
// ids the other tokens have decides where pieces are cut.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "psattn.h"
#include "psattn_rows.h"

namespace {

using namespace psattn::rows;

constexpr int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int kThreads = 256;

// Lanes of a row of `groups` groups of 16 bytes: a power of two up to a workgroup, so that short rows share one
int lanes_log2(int64_t groups) {
    int n = 3;
    while (n < 8 && (int64_t{1} << n) < groups) ++n;
    return n;
}

// AT tokens at a time to each (1 << lanes) lanes
template <typename E, bool WHOLE, int AT>
__global__ __launch_bounds__(kThreads) void psattn_embed_rows(int n_tokens, int hidden, int vocab, float scale, const int32_t* ids, const E* W, E* X, int lanes) {
    constexpr int V = kVec<E>;
    const int l = threadIdx.x & ((1 << lanes) - 1), sub = threadIdx.x >> lanes, at_once = (kThreads >> lanes) * AT;
    const int per = ((hidden + V - 1) / V + (1 << lanes) - 1) >> lanes;  // workgroups of a row
    const int64_t n = (static_cast<int64_t>(n_tokens) + at_once - 1) / at_once * per;
    for (int64_t b = blockIdx.x; b < n; b += gridDim.x) {
        const int t0 = static_cast<int>(b / per) * at_once + sub * AT, c = ((static_cast<int>(b % per) << lanes) + l) * V;
        if (c >= hidden) continue;
        const Place pl = place<WHOLE, E>(c, hidden);
        u32x4 r[AT];
#pragma unroll
        for (int u = 0; u < AT; ++u) {
            const int id = t0 + u < n_tokens ? ids[t0 + u] : -1;
            r[u] = u32x4{0, 0, 0, 0};
            if (id >= 0 && id < vocab) r[u] = raw<WHOLE>(W + static_cast<int64_t>(id) * hidden, pl, hidden);
        }
#pragma unroll
        for (int u = 0; u < AT; ++u) {
            float x[V];
            unpack(settled<WHOLE>(r[u], pl.down), x);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] *= scale;
            if (t0 + u < n_tokens) store<WHOLE>(X + static_cast<int64_t>(t0 + u) * hidden, c, hidden, x);
        }
    }
}

// ---- tokens sorted by id
// Up to kRankMost tokens: a token's place is the number of tokens that come before it, counted by sixteen lanes over all keys, which
// fit LDS: one launch instead of four (2 000 tokens 6 us, 6 000 16, 8 334 28, where the sort below takes 20 whatever their number up to 16 000).
//
// More: passes over the id's digits, least first, each stable: the digits' counts in every block of tokens, then each token to its
// place, for which a workgroup adds up the counts of all blocks itself (at most kMostBlocks; longer inputs have longer blocks).  Ids
// outside the table count as `vocab`, so that they end up behind all others.
constexpr int kSortThreads = 512, kMostBlocks = 128;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
static_assert(kDigits == kSortThreads, "a digit to a thread");

// tokens of a block: two rounds of a workgroup or more
int sort_block(int n) { return std::max(2, (n + kMostBlocks * kSortThreads - 1) / (kMostBlocks * kSortThreads)) * kSortThreads; }

__device__ __forceinline__ uint32_t key_of(int id, int vocab) { return id >= 0 && id < vocab ? static_cast<uint32_t>(id) : static_cast<uint32_t>(vocab); }

// counts[block][digit]
__global__ __launch_bounds__(kSortThreads) void psattn_embed_count(int n, int vocab, int shift, bool first, const int32_t* ids, uint32_t* counts, int block) {
    __shared__ uint32_t hist[kDigits];
    hist[threadIdx.x] = 0;
    __syncthreads();
    const int at = blockIdx.x * block, end = min(n, at + block);
    for (int i = at + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&hist[((first ? key_of(ids[i], vocab) : static_cast<uint32_t>(ids[i])) >> shift) & (kDigits - 1)], 1u);
    __syncthreads();
    counts[blockIdx.x * kDigits + threadIdx.x] = hist[threadIdx.x];
}

// Each token to its place.  Threads hold neighbouring tokens, kSortThreads to a round; a token's place among those of its digit is the
// count of earlier blocks, rounds and waves plus that of lower lanes.
__global__ __launch_bounds__(kSortThreads) void psattn_embed_place(int n, int vocab, int shift, bool first, const int32_t* ids, const int32_t* tokens,
                                                                   const uint32_t* counts, int32_t* out_keys, int32_t* out_tokens, int block) {
    constexpr int kWaves = kSortThreads / 64;
    __shared__ uint32_t next[kDigits];                // where the digit's next token goes
    __shared__ uint16_t wave_count[kWaves][kDigits];  // of this round
    __shared__ uint32_t sums[kWaves];
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6, at = blockIdx.x * block;
    {   // this thread's digit: tokens of smaller ones, and of earlier blocks
        uint32_t all = 0, before = 0;
#pragma unroll 8
        for (int b = 0; b < static_cast<int>(gridDim.x); ++b) {
            const uint32_t c = counts[b * kDigits + threadIdx.x];
            all += c;
            before += b < static_cast<int>(blockIdx.x) ? c : 0;
        }
        uint32_t run = all;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t u = __shfl_up(run, off);
            if (l >= off) run += u;
        }
        if (l == 63) sums[w] = run;
        __syncthreads();
        for (int k = 0; k < w; ++k) before += sums[k];
        next[threadIdx.x] = before + run - all;
    }
    for (int i0 = at; i0 < min(n, at + block); i0 += kSortThreads) {
        for (int i = threadIdx.x; i < kWaves * kDigits; i += kSortThreads) (&wave_count[0][0])[i] = 0;
        __syncthreads();
        const int i = i0 + threadIdx.x;
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
        uint32_t t = 0;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) t += wave_count[k][threadIdx.x];
        next[threadIdx.x] += t;  // read behind the next round's first barrier
        __syncthreads();         // the counts are cleared behind these reads
    }
}

constexpr int kRankMost = 6144;

__global__ __launch_bounds__(kThreads) void psattn_embed_rank(int n, int vocab, const int32_t* ids, int32_t* out_keys, int32_t* out_tokens) {
    __shared__ __attribute__((aligned(16))) uint32_t key[kRankMost];
    const int padded = (n + 63) / 64 * 64;
    for (int i = threadIdx.x; i < padded; i += kThreads) key[i] = i < n ? key_of(ids[i], vocab) : 0xffffffffu;  // behind all
    __syncthreads();
    const int t = blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    const uint32_t mine = key[min(t, n - 1)];
    int before = 0;
#pragma unroll 4
    for (int i = 4 * (threadIdx.x & 15); i < padded; i += 64) {
        const uint4 k = *reinterpret_cast<const uint4*>(&key[i]);
        before += (k.x < mine || (k.x == mine && i < t)) + (k.y < mine || (k.y == mine && i + 1 < t)) + (k.z < mine || (k.z == mine && i + 2 < t)) +
                  (k.w < mine || (k.w == mine && i + 3 < t));
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) before += __shfl_xor(before, off);
    if (t < n && (threadIdx.x & 15) == 0) {
        out_keys[before] = static_cast<int32_t>(mine);
        out_tokens[before] = t;
    }
}

// ---- sums of runs, and zeros for the other rows
// Pieces of 64 tokens leave half as many sums to join as pieces of 32 (65 536 tokens x 8 192: joined in 39 us instead of 79); they
// are taken where as many workgroups remain as keep the chip busy (60 000 x 1 024: summed in 108 us, with pieces of 32 90).
constexpr int kMostPiece = 64, kZeroRows = 16;

int piece_of(int64_t n, int64_t hidden) { return n * hidden >= (int64_t{1} << 28) ? 64 : 32; }
constexpr int64_t edge_ld(int64_t hidden) { return (hidden + 3) / 4 * 4; }

// Workgroups up to n_sums: (1 << lanes) groups of columns of a piece of sorted tokens, up to four pieces where columns are few.  Sums of the piece's first run, if it came from the
// piece before, and of its last, if it goes on, to edge[piece][0 / 1]; a run that does both to edge[piece][0].  Those behind: kZeroRows
// rows of the table, of which each that has no token (found by bisection) becomes zeros.
template <typename E, bool WHOLE>
__global__ __launch_bounds__(kThreads) void psattn_embed_sum(int n, int vocab, int hidden, float scale, const int32_t* keys, const int32_t* tokens, const E* dX,
                                                             E* dW, float* edge, int size, int n_sums, int lanes) {
    constexpr int V = kVec<E>;
    __shared__ int32_t keys_of[kThreads / 64][kMostPiece + 2], tokens_of[kThreads / 64][kMostPiece];
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
            tokens_of[0][threadIdx.x] = v < vocab && !(lo < n && keys[lo] == v);
        }
        __syncthreads();
        const float z[V] = {};
        for (int r = threadIdx.x >> lanes; r < kZeroRows; r += kThreads >> lanes)
            if (tokens_of[0][r])
                for (int c = (threadIdx.x & ((1 << lanes) - 1)) * V; c < hidden; c += V << lanes) store<WHOLE>(dW + static_cast<int64_t>(v0 + r) * hidden, c, hidden, z);
        return;
    }
    const int per = ((hidden + V - 1) / V + (1 << lanes) - 1) >> lanes, l = threadIdx.x & ((1 << lanes) - 1), sub = threadIdx.x >> lanes;
    const int piece = static_cast<int>(blockIdx.x) / per * (kThreads >> lanes) + sub, at = piece * size, m = min(size, n - at);  // m < 1: behind the last
    int32_t *const key = keys_of[sub], *const tok = tokens_of[sub];
    for (int i = l; i < m + 2; i += 1 << lanes) {
        const int j = at + i - 1;
        key[i] = j >= 0 && j < n ? keys[j] : -1;
        if (i < m) tok[i] = tokens[at + i];
    }
    __syncthreads();
    const int c = ((static_cast<int>(blockIdx.x) % per << lanes) + l) * V;
    if (c >= hidden) return;
    const Place pl = place<WHOLE, E>(c, hidden);
    for (int i = 0; i < m;) {
        const int v = key[i + 1];
        if (v >= vocab) return;  // padding, behind all others
        int end = i + 1;
        while (end < m && key[end + 1] == v) ++end;
        float sum[V] = {};
        int j = i;
        for (; j + 8 <= end; j += 8) {
            u32x4 x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = raw<WHOLE>(dX + static_cast<int64_t>(tok[j + u]) * hidden, pl, hidden);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                float y[V];
                unpack(settled<WHOLE>(x[u], pl.down), y);
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
            float* const to = edge + (2 * static_cast<int64_t>(piece) + (before ? 0 : 1)) * static_cast<int64_t>((hidden + 3) / 4 * 4) + c;
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

// The run that a piece's last token starts and the next pieces go on with, 256 columns of it: with q_0, q_1, ... the pieces' sums of it,
// wave w adds q_w, q_(w+4), q_(w+8), ... one by one, and the row is ((wave 0 + wave 1) + wave 2) + wave 3
template <typename E>
__global__ __launch_bounds__(kThreads) void psattn_embed_join(int n, int vocab, int hidden, float scale, const int32_t* keys, const float* edge, E* dW, int size) {
    __shared__ float4 sm[3][64];
    const int p = blockIdx.x, last = p * size + size - 1;
    if (last + 1 >= n) return;
    const int v = keys[last];
    if (v >= vocab || keys[last + 1] != v) return;                    // ends here
    if (p > 0 && keys[p * size - 1] == v) return;                     // started before
    int end = p + 1;  // behind the last piece that the run reaches, by bisection: a chain of loads for each piece would take longer than their sums
    for (int hi = (n + size - 1) / size; end < hi;) {
        const int mid = (end + hi) / 2;
        if (keys[mid * size] == v) end = mid + 1;
        else hi = mid;
    }
    const int64_t ld = (hidden + 3) / 4 * 4;
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6, c = (blockIdx.y * 64 + l) * 4;
    float4 sum = {0.f, 0.f, 0.f, 0.f};
    if (c < hidden) {
        auto part = [&](int q) { return *reinterpret_cast<const float4*>(edge + (2 * static_cast<int64_t>(q) + (q == p ? 1 : 0)) * ld + c); };
        auto add = [&](const float4& x) { sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w; };
        int q = p + w;
        for (; q + 12 < end; q += 16) {  // loads together, sums in order
            const float4 x0 = part(q), x1 = part(q + 4), x2 = part(q + 8), x3 = part(q + 12);
            add(x0);
            add(x1);
            add(x2);
            add(x3);
        }
        for (; q < end; q += 4) add(part(q));
    }
    if (w > 0) sm[w - 1][l] = sum;
    __syncthreads();
    if (w > 0 || c >= hidden) return;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const float4 x = sm[k][l];
        sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
    }
    const float t[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (c + k < hidden) store1(dW + static_cast<int64_t>(v) * hidden + c + k, t[k] * scale);
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
    s.counts = reinterpret_cast<uint32_t*>(take(sizeof(uint32_t) * kDigits * kMostBlocks));
    s.edge = reinterpret_cast<float*>(take(sizeof(float) * 2 * cdiv(n, piece_of(n, hidden)) * edge_ld(hidden)));
    s.total = static_cast<size_t>(p - p0) + 256;
    return s;
}

template <typename E>
void rows(int32_t n, int32_t vocab, int32_t hidden, float scale, const int32_t* ids, const void* W, void* X, hipStream_t s) {
    const E* w = static_cast<const E*>(W);
    E* x = static_cast<E*>(X);
    const int64_t groups = cdiv(hidden, kVec<E>);
    const int lanes = lanes_log2(groups);
    const int64_t per = cdiv(groups, 1 << lanes);
    auto go = [&](auto kernel, int at) {
        kernel<<<static_cast<uint32_t>(std::min<int64_t>(cdiv(n, (kThreads >> lanes) * at) * per, 1 << 20)), kThreads, 0, s>>>(n, hidden, vocab, scale, ids, w, x, lanes);
    };
    const bool all = whole<E>(hidden, {W, X});
    if ((n >> (8 - lanes)) * per >= 4096) all ? go(psattn_embed_rows<E, true, 4>, 4) : go(psattn_embed_rows<E, false, 4>, 4);
    else all ? go(psattn_embed_rows<E, true, 1>, 1) : go(psattn_embed_rows<E, false, 1>, 1);
}

template <typename E>
void grad(int32_t n, int32_t vocab, int32_t hidden, float scale, const int32_t* ids, const void* dX_, void* dW_, void* workspace, hipStream_t s) {
    const E* dX = static_cast<const E*>(dX_);
    E* dW = static_cast<E*>(dW_);
    const Slots w = carve(n, hidden, workspace);
    const int32_t *keys = ids, *tokens = nullptr;
    if (n > kRankMost) {
        const int block = sort_block(n), blocks = static_cast<int>(cdiv(n, block));
        int bits = 1;
        while (bits < 31 && (vocab >> bits) != 0) ++bits;  // keys are 0 .. vocab
        for (int shift = 0, turn = 0; shift < bits; shift += kDigitBits, turn ^= 1) {
            psattn_embed_count<<<blocks, kSortThreads, 0, s>>>(n, vocab, shift, shift == 0, keys, w.counts, block);
            psattn_embed_place<<<blocks, kSortThreads, 0, s>>>(n, vocab, shift, shift == 0, keys, tokens, w.counts, w.keys[turn], w.tokens[turn], block);
            keys = w.keys[turn];
            tokens = w.tokens[turn];
        }
    } else if (n > 0) {
        psattn_embed_rank<<<static_cast<uint32_t>(cdiv(n, kThreads / 16)), kThreads, 0, s>>>(n, vocab, ids, w.keys[0], w.tokens[0]);
        keys = w.keys[0];
        tokens = w.tokens[0];
    }
    const int64_t groups = cdiv(hidden, kVec<E>);
    const int lanes = std::max(6, lanes_log2(groups));  // no more than a workgroup's four waves' pieces: few tokens need the workgroups
    const int size = piece_of(n, hidden);
    const int64_t sums = cdiv(cdiv(n, size), kThreads >> lanes) * cdiv(groups, 1 << lanes), zeros = cdiv(vocab, kZeroRows);
    auto sum = [&](auto kernel) {
        kernel<<<static_cast<uint32_t>(sums + zeros), kThreads, 0, s>>>(n, vocab, hidden, scale, keys, tokens, dX, dW, w.edge, size, static_cast<int>(sums), lanes);
    };
    if (whole<E>(hidden, {dX, dW})) sum(psattn_embed_sum<E, true>);
    else sum(psattn_embed_sum<E, false>);
    if (n > size) psattn_embed_join<E><<<dim3(static_cast<uint32_t>(cdiv(n, size)), static_cast<uint32_t>(cdiv(hidden, 256))), kThreads, 0, s>>>(n, vocab, hidden, scale, keys, w.edge, dW, size);
}

// grids below 2^31 threads, and table rows found by int
bool too_large(int32_t n_tokens, int32_t vocab, int32_t hidden) {
    return n_tokens > (1 << 24) || hidden > (1 << 23) || cdiv(n_tokens, 32) * cdiv(hidden, kThreads) + cdiv(vocab, kZeroRows) >= (1 << 23) || vocab == INT32_MAX;
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
