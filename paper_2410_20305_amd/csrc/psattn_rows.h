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
// the same, not yet unpacked
template <bool WHOLE, typename E>
__device__ __forceinline__ u32x4 raw(const E* row, int c, int hidden) {
    if (WHOLE ? c < hidden : c + kVec<E> <= hidden) {
        if constexpr (WHOLE) return *reinterpret_cast<const u32x4*>(row + c);
        else return reinterpret_cast<const Raw*>(row + c)->u;
    }
    u32x4 u = {0, 0, 0, 0};
    if constexpr (!WHOLE) {
#pragma unroll
        for (int j = 0; j < kVec<E>; ++j)
            if (c + j < hidden) {
                if constexpr (sizeof(E) == 2) u[j / 2] |= static_cast<uint32_t>(row[c + j]) << (16 * (j & 1));
                else u[j] = __float_as_uint(row[c + j]);
            }
    }
    return u;
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
