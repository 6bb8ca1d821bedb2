// Rotary positions on Q and K in memory: any layout, any part of the head, any frequencies, and the transposed turn for gradients.
//   y_a = c x_a - s x_b,  y_b = c x_b + s x_a  for each pair (a, b) of the first rotary_dim dimensions of a head; c, s: the table's
//   cosine and sine (times its amplitude) of the row's position.  Transposed: -s.  The other dimensions are copied.
//
// Bound by HBM (a head's dimensions in and out; the table's rows are shared by all heads and stay in the caches).  A lane's unit is V pairs in two
// chunks of V elements: dimensions i .. and rotary_dim / 2 + i .. (half), or 2 i .. of 2 V (interleaved), so that either layout reads and
// writes whole chunks.  V is the most that sizes and addresses allow, up to 16 bytes.  65 536 tokens of 72 heads of 128 bf16, out of one
// buffer, both ways: 814 us, 5.9 TB/s.
//   A lane takes KH heads of a token: one where chunks have 16 bytes, more where they are smaller, for which cosines, sines and positions are
// most of what it asks for.  KH 1 / 2 / 4, both ways, in us: 65 536 x 72 x 128 bf16 814 / 865 / 874; chunks of 8 bytes (20 000 tokens, 18 heads of 80, 40
// turned) 43.8 / 41.0 / 40.8; of 4 bytes (5 000 tokens, 32 heads of 80, 20 turned) 34.7 / 26.7 / 24.2.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "psattn_mfma_common.h"
#include "psattn_rope.h"
#include "psattn_rows.h"

namespace psattn {
namespace {

struct RopeArgs {
    const float* table;
    const int32_t* positions;
    const void *in[2];
    void* out[2];           // Q, K
    int64_t in_stride[2], out_stride[2];
    int32_t heads[2];
    int32_t n_items, groups;    // tokens x groups of heads
    int32_t dim, rotary, max_positions;
    int32_t n_rot, n_units;     // units of a head: turned, and in all
    float sign;
};

constexpr int kThreads = 256;

template <int BYTES> struct Word;
template <> struct Word<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <> struct Word<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<2> { typedef uint16_t type; };

// V elements
template <typename E, int V>
struct Chunk {
    typedef typename Word<V * static_cast<int>(sizeof(E))>::type W;
    W w;
    __device__ __forceinline__ void load(const E* p) { w = *reinterpret_cast<const W*>(p); }
    __device__ __forceinline__ void store(E* p) const { *reinterpret_cast<W*>(p) = w; }
    __device__ __forceinline__ void get(float (&x)[V]) const {
        struct Es { E e[V]; };
        const Es e = __builtin_bit_cast(Es, w);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = rows::to_f32(e.e[j]);
    }
    __device__ __forceinline__ void set(const float (&x)[V]) {
        struct Es { E e[V]; } e;
        if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int j = 0; j < V; ++j) e.e[j] = x[j];
        } else {
#pragma unroll
            for (int j = 0; j < V; j += 2) {
                const uint32_t two = mma::pack2(x[j], j + 1 < V ? x[j + 1] : 0.f);
                e.e[j] = static_cast<uint16_t>(two);
                if (j + 1 < V) e.e[j + 1] = static_cast<uint16_t>(two >> 16);
            }
        }
        w = __builtin_bit_cast(W, e);
    }
};

template <typename E, int V, bool HALF, int KH, typename Position>
__device__ __forceinline__ void turn_unit(const RopeArgs& r, Position&& position_of) {
    const int slots = kThreads / r.n_units, slot = static_cast<int>(threadIdx.x) / r.n_units, unit = static_cast<int>(threadIdx.x) - slot * r.n_units;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * slots + slot;
    if (slot >= slots || item >= r.n_items) return;
    const int t = static_cast<int>(item) / r.groups, first = static_cast<int>(item) - t * r.groups;
    const int pos = position_of(t);
    const bool turned = unit < r.n_rot, known = pos >= 0 && pos < r.max_positions;
    const int half = r.rotary / 2;
    const int at0 = !turned ? r.rotary + 2 * (unit - r.n_rot) * V : HALF ? unit * V : 2 * unit * V;
    const int at1 = turned && HALF ? half + unit * V : at0 + V;
    const bool two = at1 < r.dim;
    float c[V], s[V];
    if (turned && known) {
        const float* row = r.table + static_cast<int64_t>(pos) * r.rotary + unit * V;
        Chunk<float, V < 4 ? V : 4> x;
#pragma unroll
        for (int j = 0; j < V; j += V < 4 ? V : 4) {
            float y[V < 4 ? V : 4];
            x.load(row + j);
            x.get(y);
#pragma unroll
            for (int k = 0; k < (V < 4 ? V : 4); ++k) c[j + k] = y[k];
            x.load(row + half + j);
            x.get(y);
#pragma unroll
            for (int k = 0; k < (V < 4 ? V : 4); ++k) s[j + k] = r.sign * y[k];
        }
    }
    const int n_heads = r.heads[0] + r.heads[1];
    Chunk<E, V> a[KH], b[KH];
    auto place = [&](int i, bool out) {  // the i-th head of this lane
        const int h = first + i * r.groups, k = h >= r.heads[0] ? 1 : 0;
        return (out ? static_cast<int64_t>(t) * r.out_stride[k] : static_cast<int64_t>(t) * r.in_stride[k]) + (h - (k ? r.heads[0] : 0)) * static_cast<int64_t>(r.dim);
    };
#pragma unroll
    for (int i = 0; i < KH; ++i) {
        a[i].w = {};
        b[i].w = {};
        const int h = first + i * r.groups;
        if (h < n_heads && known) {
            const E* p = static_cast<const E*>(r.in[h >= r.heads[0] ? 1 : 0]) + place(i, false);
            a[i].load(p + at0);
            if (two) b[i].load(p + at1);
        }
    }
#pragma unroll
    for (int i = 0; i < KH; ++i) {
        const int h = first + i * r.groups;
        if (h >= n_heads) break;
        if (turned && known) {
            float x[V], y[V], u[V], v[V];
            a[i].get(x);
            b[i].get(y);
            if constexpr (HALF || V == 1) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    u[j] = x[j], v[j] = y[j];
                    mma::rope_turn<false>(u[j], v[j], c[j], s[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {  // pair j: elements 2 j and 2 j + 1 of the two chunks
                    float p = 2 * j < V ? x[2 * j % V] : y[2 * j % V], q = 2 * j < V ? x[(2 * j + 1) % V] : y[(2 * j + 1) % V];
                    mma::rope_turn<false>(p, q, c[j], s[j]);
                    (2 * j < V ? u : v)[2 * j % V] = p;
                    (2 * j < V ? u : v)[(2 * j + 1) % V] = q;
                }
            }
            a[i].set(u);
            b[i].set(v);
        }
        E* p = static_cast<E*>(r.out[h >= r.heads[0] ? 1 : 0]) + place(i, true);
        a[i].store(p + at0);
        if (two) b[i].store(p + at1);
    }
}

template <typename E, int V, bool HALF, int KH>
__global__ __launch_bounds__(kThreads) void psattn_rope_rows(RopeArgs r) {
    turn_unit<E, V, HALF, KH>(r, [&](int t) { return r.positions[t]; });
}
// positions by the block mask's descriptors
template <typename E, int V, bool HALF, int KH>
__global__ __launch_bounds__(kThreads) void psattn_rope_rows_of_mask(AttnArgs a, RopeArgs r) {
    turn_unit<E, V, HALF, KH>(r, [&](int t) { return mma::rope_position(token(a.meta, t), t); });
}

template <typename E, int V, bool HALF>
int launch(RopeArgs r, const psattn_meta* meta, int32_t n_tokens, hipStream_t s) {
    constexpr int kBytes = V * static_cast<int>(sizeof(E)), KH = kBytes >= 16 ? 1 : kBytes == 8 ? 2 : 4;
    r.n_rot = r.rotary / 2 / V;
    r.n_units = r.n_rot + (r.dim - r.rotary + 2 * V - 1) / (2 * V);
    const int n_heads = r.heads[0] + r.heads[1], slots = kThreads / r.n_units;
    r.groups = (n_heads + KH - 1) / KH;
    const int64_t items = static_cast<int64_t>(n_tokens) * r.groups, grid = (items + slots - 1) / slots;
    if (items > INT32_MAX || grid >= (int64_t{1} << 31) / kThreads) return PSATTN_EUNSUPPORTED;
    r.n_items = static_cast<int32_t>(items);
    if (meta) {
        AttnArgs a{};
        a.meta = meta->dev;
        psattn_rope_rows_of_mask<E, V, HALF, KH><<<static_cast<uint32_t>(grid), kThreads, 0, s>>>(a, r);
    } else {
        psattn_rope_rows<E, V, HALF, KH><<<static_cast<uint32_t>(grid), kThreads, 0, s>>>(r);
    }
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

}  // namespace
}  // namespace psattn

extern "C" {

int psattn_rope_apply(const psattn_rope* rope, int32_t dt, int32_t transposed, int32_t n_tokens, const int32_t* positions, const psattn_meta* meta,
                      int32_t n_q_heads, const void* Q, int64_t q_stride, void* Qr, int64_t qr_stride, int32_t n_kv_heads, const void* K, int64_t k_stride,
                      void* Kr, int64_t kr_stride, void* hip_stream) {
    using namespace psattn;
    if (!rope || (dt != PSATTN_F32 && dt != PSATTN_BF16) || n_tokens < 0 || n_q_heads < 0 || n_kv_heads < 0) return PSATTN_EINVAL;
    if ((positions != nullptr) == (meta != nullptr) && n_tokens > 0) return PSATTN_EINVAL;  // one says where the tokens are
    const int64_t q_row = static_cast<int64_t>(n_q_heads) * rope->head_dim, k_row = static_cast<int64_t>(n_kv_heads) * rope->head_dim;
    if (q_stride < q_row || qr_stride < q_row || k_stride < k_row || kr_stride < k_row) return PSATTN_EINVAL;
    if (n_q_heads > (1 << 20) || n_kv_heads > (1 << 20)) return PSATTN_EUNSUPPORTED;
    if (meta) {
        if (meta->T != n_tokens) return PSATTN_EINVAL;
        if (!meta->on_device) return PSATTN_ENODEVICE;
        if (meta->n_positions > rope->max_positions) return PSATTN_ELIMIT;
    }
    if (n_tokens == 0 || n_q_heads + n_kv_heads == 0) return PSATTN_OK;
    int device = -1;
    if (hipGetDevice(&device) == hipSuccess && device != rope->device) return PSATTN_EINVAL;
    if ((n_q_heads > 0 && (!Q || !Qr)) || (n_kv_heads > 0 && (!K || !Kr))) return PSATTN_EINVAL;
    RopeArgs r{};
    r.table = rope->d_table;
    r.positions = positions;
    r.in[0] = Q, r.in[1] = K, r.out[0] = Qr, r.out[1] = Kr;
    r.in_stride[0] = q_stride, r.in_stride[1] = k_stride, r.out_stride[0] = qr_stride, r.out_stride[1] = kr_stride;
    r.heads[0] = n_q_heads, r.heads[1] = n_kv_heads;
    r.dim = rope->head_dim, r.rotary = rope->rotary_dim, r.max_positions = rope->max_positions;
    r.sign = transposed ? -1.f : 1.f;
    // elements to a chunk: the most that divides what is turned and what is copied, where every chunk is on a boundary of its size
    const int e = dt == PSATTN_BF16 ? 2 : 4;
    auto fits = [&](int v) {
        bool ok = r.rotary / 2 % v == 0 && (r.dim - r.rotary) % v == 0;
        for (int k = 0; k < 2; ++k)
            if (r.heads[k] > 0)
                ok = ok && (reinterpret_cast<uintptr_t>(r.in[k]) | reinterpret_cast<uintptr_t>(r.out[k])) % (v * e) == 0 && (n_tokens == 1 || (r.in_stride[k] % v == 0 && r.out_stride[k] % v == 0));
        return ok;
    };
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    auto sized = [&](auto elem, auto v) {
        using E = decltype(elem);
        constexpr int V = decltype(v)::value;
        return rope->layout == PSATTN_ROPE_HALF ? launch<E, V, true>(r, meta, n_tokens, s) : launch<E, V, false>(r, meta, n_tokens, s);
    };
    using std::integral_constant;
    if (dt == PSATTN_BF16) {
        if (fits(8)) return sized(uint16_t{}, integral_constant<int, 8>{});
        if (fits(4)) return sized(uint16_t{}, integral_constant<int, 4>{});
        if (fits(2)) return sized(uint16_t{}, integral_constant<int, 2>{});
        return sized(uint16_t{}, integral_constant<int, 1>{});
    }
    if (fits(4)) return sized(float{}, integral_constant<int, 4>{});
    if (fits(2)) return sized(float{}, integral_constant<int, 2>{});
    return sized(float{}, integral_constant<int, 1>{});
}

}  // extern "C"
