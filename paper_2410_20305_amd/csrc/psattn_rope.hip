// Rotary position embedding inside the attention op (paper Section 3.1: position ids are set
// so that every response sits where it would sit in the normal paired format, i.e. the
// rejected response restarts right behind the prompt).
//
// Where the rotation happens:
//   Q   in the forward kernel's registers when the query row is loaded (each query row is
//       loaded exactly once); the rotated row is saved for the backward, whose k-major pass
//       streams Q tiles straight from global memory into LDS and cannot rotate them on the way.
//   K   once per layer by the small streaming kernel below: a K row is re-read by every q-tile
//       and q-head that sees it, so rotating it inside the attention kernels would repeat the
//       work dozens of times, and the K tiles travel global -> LDS without passing registers.
//       With grouped-query attention K is 1/G of Q, so this is the cheap half of a RoPE pass.
//   dQ, dK  turned back (gradient w.r.t. the unrotated tensors) in the registers of the dQ and
//       dK/dV kernels just before they are stored.
// No pass over a Q-sized tensor is added; position ids come from the per-token descriptors of
// the block mask, so no position array is stored either.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <new>
#include <vector>

#include "psattn_mfma_common.h"
#include "psattn_rope.h"

namespace psattn {
namespace {
using namespace mma;

// one thread per (token, kv-head, 8 dims below 64): rotates them and their partners above 64
__global__ __launch_bounds__(256) void psattn_rope_k_bf16(AttnArgs a, uint16_t* Kr) {
    const int Hkv = a.Hkv;
    const uint16_t* K = static_cast<const uint16_t*>(a.K);
    const size_t idx = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
    const size_t n = static_cast<size_t>(a.meta.T) * Hkv * 8;
    if (idx >= n) return;
    const int chunk = static_cast<int>(idx & 7);
    const size_t row = idx >> 3;               // token * Hkv + head
    const int t = static_cast<int>(row / Hkv);
    const float* trow = a.rope + static_cast<size_t>(rope_position(token(a.meta, t), t)) * 128;
    Frag8 lo, hi;
    lo.u = *reinterpret_cast<const uint4*>(K + row * 128 + 8 * chunk);
    hi.u = *reinterpret_cast<const uint4*>(K + row * 128 + 64 + 8 * chunk);
    float4 turn[4];
    rope_load8(turn, trow, 8 * chunk);
    rope_frag8(lo, hi, turn);
    *reinterpret_cast<uint4*>(Kr + row * 128 + 8 * chunk) = lo.u;
    *reinterpret_cast<uint4*>(Kr + row * 128 + 64 + 8 * chunk) = hi.u;
}

struct Frequencies {
    double f[kRopeMostDims / 2];
};
// cosines and sines of position * frequency; angles in double, of which a float would lose the low bits at long positions
__global__ __launch_bounds__(256) void psattn_rope_table(Frequencies f, double amplitude, int half, int64_t n, float* table) {
    for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
        const int64_t p = i / half;
        const int k = static_cast<int>(i - p * half);
        const double a = static_cast<double>(p) * f.f[k];
        table[p * 2 * half + k] = static_cast<float>(amplitude * cos(a));
        table[p * 2 * half + half + k] = static_cast<float>(amplitude * sin(a));
    }
}

int check_rope(const psattn_meta* meta, const psattn_rope* rope, int32_t dt, int32_t head_dim) {
    if (!meta || !rope) return PSATTN_EINVAL;
    if (dt != PSATTN_BF16 || head_dim != 128 || rope->head_dim != 128 || rope->rotary_dim != 128 || rope->layout != PSATTN_ROPE_HALF) return PSATTN_EUNSUPPORTED;
    if (!meta->on_device) return PSATTN_ENODEVICE;
    if (meta->n_positions > rope->max_positions) return PSATTN_ELIMIT;
    return PSATTN_OK;
}

}  // namespace

// inv_freq on the host's side; on_device: the table is computed there (131 072 positions of 32 dimensions: 36 ms by the host, 0.3 so), else by
// the host, as psattn_rope_create always has: the two agree but for the last bit of a double ahead of the rounding to float (131 072 positions of 128
// dimensions at two bases: in all of 33 554 432 entries; 157 ms and 0.4)
static int make_rope(int32_t head_dim, int32_t rotary_dim, int32_t layout, const double* inv_freq, double amplitude, int32_t max_positions, bool on_device, void* hip_stream,
              psattn_rope** out) {
    psattn_rope* r = new (std::nothrow) psattn_rope();
    if (!r) return PSATTN_ENOMEM;
    r->head_dim = head_dim;
    r->rotary_dim = rotary_dim;
    r->layout = layout;
    r->max_positions = max_positions;
    const int half = rotary_dim / 2;
    const size_t n = static_cast<size_t>(max_positions) * rotary_dim;
    std::vector<float> host;
    if (!on_device) {
        try {
            host.resize(n);
        } catch (const std::exception&) {  // no memory, or more than a vector may hold
            delete r;
            return PSATTN_ENOMEM;
        }
        // angles in double: a float product position * frequency would lose the low bits of long positions
        for (int32_t p = 0; p < max_positions; ++p)
            for (int i = 0; i < half; ++i) {
                const double a = static_cast<double>(p) * inv_freq[i];
                host[static_cast<size_t>(p) * rotary_dim + i] = static_cast<float>(amplitude * std::cos(a));
                host[static_cast<size_t>(p) * rotary_dim + half + i] = static_cast<float>(amplitude * std::sin(a));
            }
    }
    if (hipGetDevice(&r->device) != hipSuccess || hipMalloc(reinterpret_cast<void**>(&r->d_table), n * sizeof(float)) != hipSuccess) {
        (void)hipGetLastError();
        delete r;
        return PSATTN_ENOMEM;
    }
    // complete on return, for any stream; the host vector dies with this call
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    hipError_t e;
    if (on_device) {
        Frequencies f{};
        std::copy(inv_freq, inv_freq + half, f.f);
        psattn_rope_table<<<2048, 256, 0, s>>>(f, amplitude, half, static_cast<int64_t>(max_positions) * half, r->d_table);
        e = hipGetLastError();
    } else {
        e = hipMemcpyAsync(r->d_table, host.data(), n * sizeof(float), hipMemcpyHostToDevice, s);
    }
    if (e != hipSuccess || hipStreamSynchronize(s) != hipSuccess) {
        (void)hipGetLastError();
        (void)hipFree(r->d_table);
        delete r;
        return PSATTN_EHIP;
    }
    *out = r;
    return PSATTN_OK;
}

}  // namespace psattn

extern "C" {

int psattn_rope_create(int32_t head_dim, float theta, int32_t max_positions, void* hip_stream, psattn_rope** out) {
    if (!out) return PSATTN_EINVAL;
    *out = nullptr;
    if (max_positions <= 0 || !(theta > 0.f)) return PSATTN_EINVAL;
    if (head_dim != 128) return PSATTN_EUNSUPPORTED;
    double inv_freq[64];
    for (int i = 0; i < 64; ++i) inv_freq[i] = std::pow(static_cast<double>(theta), -2.0 * i / head_dim);
    return psattn::make_rope(head_dim, head_dim, PSATTN_ROPE_HALF, inv_freq, 1.0, max_positions, false, hip_stream, out);
}

int psattn_rope_create_layout(int32_t head_dim, int32_t rotary_dim, int32_t layout, const double* inv_freq, double amplitude,
                              int32_t max_positions, void* hip_stream, psattn_rope** out) {
    if (!out) return PSATTN_EINVAL;
    *out = nullptr;
    if (head_dim <= 0 || rotary_dim <= 0 || rotary_dim % 2 != 0 || rotary_dim > head_dim || max_positions <= 0 || !inv_freq) return PSATTN_EINVAL;
    if (layout != PSATTN_ROPE_HALF && layout != PSATTN_ROPE_INTERLEAVED) return PSATTN_EINVAL;
    if (!std::isfinite(amplitude)) return PSATTN_EINVAL;
    if (head_dim > psattn::kRopeMostDims) return PSATTN_EUNSUPPORTED;
    for (int i = 0; i < rotary_dim / 2; ++i)
        if (!std::isfinite(inv_freq[i])) return PSATTN_EINVAL;
    return psattn::make_rope(head_dim, rotary_dim, layout, inv_freq, amplitude, max_positions, true, hip_stream, out);
}

int psattn_rope_frequencies(int32_t rotary_dim, double theta, int32_t scaling, double factor, double original_positions, double low, double high,
                            double* inv_freq) {
    if (!inv_freq || rotary_dim <= 0 || rotary_dim % 2 != 0 || !(theta > 0.0) || std::isinf(theta)) return PSATTN_EINVAL;
    if (scaling < PSATTN_ROPE_PLAIN || scaling > PSATTN_ROPE_PARTS) return PSATTN_EINVAL;
    if (scaling != PSATTN_ROPE_PLAIN && (!(factor > 0.0) || std::isinf(factor))) return PSATTN_EINVAL;
    if (scaling == PSATTN_ROPE_PARTS && (!(original_positions > 0.0) || std::isinf(original_positions) || !(high > low) || std::isinf(low) || std::isinf(high))) return PSATTN_EINVAL;
    const int n = rotary_dim;
    // the lowest frequency is divided by the factor, the highest stays 1: theta^(-(n - 2) / n) falls by factor^(-1)
    const double base = scaling == PSATTN_ROPE_BASE && n > 2 ? theta * std::pow(factor, static_cast<double>(n) / (n - 2)) : theta;
    for (int i = 0; i < n / 2; ++i) {
        double f = std::pow(base, -2.0 * i / n);
        if (scaling == PSATTN_ROPE_LINEAR) f /= factor;
        if (scaling == PSATTN_ROPE_PARTS) {
            const double turns = f * original_positions / 6.283185307179586476925;
            const double keep = std::min(1.0, std::max(0.0, (turns - low) / (high - low)));
            f = keep * f + (1.0 - keep) * f / factor;
        }
        inv_freq[i] = f;
    }
    return PSATTN_OK;
}

int psattn_rope_free(psattn_rope* rope) {
    if (!rope) return PSATTN_OK;
    int rc = PSATTN_OK;
    if (rope->d_table && hipFree(rope->d_table) != hipSuccess) rc = PSATTN_EHIP;
    delete rope;
    return rc;
}

int psattn_rope_k(const psattn_meta* meta, const psattn_rope* rope, int32_t dt, int32_t n_kv_heads, int32_t head_dim,
                  const void* K, void* Kr, void* hip_stream) {
    int rc = psattn::check_rope(meta, rope, dt, head_dim);
    if (rc != PSATTN_OK) return rc;
    if (n_kv_heads <= 0) return PSATTN_EINVAL;
    if (meta->T == 0) return PSATTN_OK;
    if (!K || !Kr) return PSATTN_EINVAL;
    const size_t n = static_cast<size_t>(meta->T) * n_kv_heads * 8;
    const size_t grid = (n + 255) / 256;
    if (grid > 0x7fffffffu) return PSATTN_EUNSUPPORTED;
    psattn::AttnArgs a{};
    a.meta = meta->dev;
    a.Hkv = n_kv_heads; a.K = K; a.rope = rope->d_table;
    psattn::psattn_rope_k_bf16<<<static_cast<unsigned>(grid), 256, 0, static_cast<hipStream_t>(hip_stream)>>>(a, static_cast<uint16_t*>(Kr));
    return hipGetLastError() == hipSuccess ? PSATTN_OK : PSATTN_EHIP;
}

int psattn_fwd_rope(const psattn_meta* meta, const psattn_rope* rope, int32_t dt, int32_t n_q_heads, int32_t n_kv_heads,
                    int32_t head_dim, float scale, const void* Q, const void* K, const void* V, void* O, float* LSE,
                    void* Qr, void* Kr, void* hip_stream) {
    int rc = psattn::check_rope(meta, rope, dt, head_dim);
    if (rc != PSATTN_OK) return rc;
    if (!psattn_uses_mfma(meta, dt, head_dim, scale, 0)) return PSATTN_EUNSUPPORTED;
    if (meta->T > 0 && !Kr) return PSATTN_EINVAL;
    rc = psattn_rope_k(meta, rope, dt, n_kv_heads, head_dim, K, Kr, hip_stream);
    if (rc != PSATTN_OK) return rc;
    return psattn::fwd_checked(meta, dt, n_q_heads, n_kv_heads, head_dim, scale, Q, Kr, V, O, LSE, rope->d_table, Qr,
                               hip_stream);
}

int psattn_bwd_rope(const psattn_meta* meta, const psattn_rope* rope, int32_t dt, int32_t n_q_heads, int32_t n_kv_heads,
                    int32_t head_dim, float scale, const void* Qr, const void* Kr, const void* V, const void* O,
                    const void* dO, const float* LSE, void* dQ, void* dK, void* dV, void* workspace,
                    size_t workspace_bytes, void* hip_stream) {
    const int rc = psattn::check_rope(meta, rope, dt, head_dim);
    if (rc != PSATTN_OK) return rc;
    return psattn::bwd_checked(meta, dt, n_q_heads, n_kv_heads, head_dim, scale, Qr, Kr, V, O, dO, LSE, dQ, dK, dV,
                               workspace, workspace_bytes, hip_stream, rope->d_table);
}

}  // extern "C"
