// Rows of fp32 or bf16 in groups of 16 bytes, whatever address they start at (layer norm, embedding).
#pragma once
#include <algorithm>
#include <initializer_list>

#include "psattn_gemm.h"

namespace psattn {
namespace rows {

using gemm::store1;
using gemm::to_f32;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

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
// 16 bytes from any address of an element
struct __attribute__((packed, aligned(2))) Raw {
    u32x4 u;
};

// kVec elements from column c of a row of `hidden`, zeros outside of it.  Rows may start anywhere: a group is one load whatever its
// address.  One that reaches past an end of its row is read from inside it and shifted when it is used: a lane's groups of all rows
// and tensors share their place, and no wave waits for its two edge lanes' loads by themselves, which took three times as long
// (20 000 rows of 1 003 bf16 with dS, layer norm backward 102 us, 53 by places).  Rows shorter than a group go element by element.
struct Place {
    int at, down;  // first column of the load; bits that the group lies behind it (128 and more: outside)
};
template <bool WHOLE, typename E>
__device__ __forceinline__ Place place(int c, int hidden) {
    constexpr int V = kVec<E>, kBits = 8 * static_cast<int>(sizeof(E));
    if constexpr (WHOLE) return {c, 0};
    if (hidden < V) return {c, 0};
    const int at = min(max(c, 0), hidden - V);
    return {at, min(max(c - at, -V), V) * kBits};
}
template <bool WHOLE, typename E>
__device__ __forceinline__ u32x4 raw(const E* row, const Place& p, int hidden) {
    constexpr int V = kVec<E>, kBits = 8 * static_cast<int>(sizeof(E));
    u32x4 u = {0, 0, 0, 0};
    if constexpr (WHOLE) {
        if (p.at < hidden) u = *reinterpret_cast<const u32x4*>(row + p.at);
    } else if (hidden >= V) {
        u = reinterpret_cast<const Raw*>(row + p.at)->u;
    } else {
        uint64_t lo = 0, hi = 0;
#pragma unroll 1
        for (int j = 0; j < V; ++j) {
            uint64_t v = 0;
            if (p.at + j >= 0 && p.at + j < hidden) {
                if constexpr (sizeof(E) == 2) v = row[p.at + j];
                else v = __float_as_uint(row[p.at + j]);
            }
            const int bit = j * kBits;
            if (bit < 64) lo |= v << bit;
            else hi |= v << (bit - 64);
        }
        u = u32x4{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi), static_cast<uint32_t>(hi >> 32)};
    }
    return u;
}
template <bool WHOLE>
__device__ __forceinline__ u32x4 settled(const u32x4& x, int down) {
    if (WHOLE || down == 0) return x;
    uint64_t lo = (static_cast<uint64_t>(x[1]) << 32) | x[0], hi = (static_cast<uint64_t>(x[3]) << 32) | x[2];
    if (down >= 128 || down <= -128) {
        lo = hi = 0;
    } else if (down > 0) {
        lo = down >= 64 ? hi >> (down - 64) : (lo >> down) | (hi << (64 - down));
        hi = down >= 64 ? 0 : hi >> down;
    } else {
        hi = down <= -64 ? lo << (-down - 64) : (hi << -down) | (lo >> (64 + down));
        lo = down <= -64 ? 0 : lo << -down;
    }
    return u32x4{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi), static_cast<uint32_t>(hi >> 32)};
}
template <bool WHOLE, typename E>
__device__ __forceinline__ void load(const E* row, int c, int hidden, float (&x)[kVec<E>]) {
    const Place p = place<WHOLE, E>(c, hidden);
    unpack(settled<WHOLE>(raw<WHOLE>(row, p, hidden), p.down), x);
}
template <bool WHOLE, typename E>
__device__ __forceinline__ void store(E* row, int c, int hidden, const float (&x)[kVec<E>]) {
    if constexpr (WHOLE) {
        if (c < hidden) *reinterpret_cast<u32x4*>(row + c) = pack<E>(x);
    } else if (c >= 0 && c + kVec<E> <= hidden) {
        reinterpret_cast<Raw*>(row + c)->u = pack<E>(x);
    } else {
#pragma unroll
        for (int j = 0; j < kVec<E>; ++j)
            if (c + j >= 0 && c + j < hidden) store1(row + c + j, x[j]);
    }
}
// elements that a row starts behind a 16-byte boundary
template <typename E>
__device__ __forceinline__ int misalignment(const E* row) {
    return static_cast<int>(reinterpret_cast<uintptr_t>(row) / sizeof(E) % kVec<E>);
}

// rows of `hidden` elements that all start on a 16-byte boundary and are whole groups
template <typename E>
bool whole(int32_t hidden, std::initializer_list<const void*> p) {
    uintptr_t a = 0;
    for (const void* x : p) a |= reinterpret_cast<uintptr_t>(x);
    return a % 16 == 0 && hidden % kVec<E> == 0;
}

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace rows
}  // namespace psattn
