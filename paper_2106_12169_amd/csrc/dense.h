// Dense 16- and 32-bit floating-point operands: one element, or 16 bytes at once, to fp32 and back.
#pragma once
#include "common.h"

#include <climits>
#include <cmath>

namespace apnn {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

inline bool known_type(apnn_dtype t) { return t == APNN_F32 || t == APNN_F16 || t == APNN_BF16; }
inline int size_of(apnn_dtype t) { return t == APNN_F32 ? 4 : 2; }
inline bool aligned_to(const void *p, apnn_dtype t) { return reinterpret_cast<uintptr_t>(p) % static_cast<unsigned>(size_of(t)) == 0; }

// [tokens][heads][D] with element strides: none negative, no address beyond 64 bits, and for a result no two elements in one place.
inline bool strides_fit(int64_t tokens, int64_t heads, int64_t D, int64_t token_stride, int64_t head_stride, bool result)
{
    const int64_t most = INT64_MAX / 16;
    if (token_stride < 0 || head_stride < 0 || (tokens > 1 && token_stride > most / tokens) || (heads > 1 && head_stride > most / heads)) return false;
    if (!result) return true;
    if (heads > 1 && head_stride < D) return false;
    if (tokens > 1 && token_stride < D) return false;
    return tokens <= 1 || heads <= 1 || token_stride >= (heads - 1) * head_stride + D || head_stride >= (tokens - 1) * token_stride + D;
}

// Runs f(T{}) with the element type of `t`.
template <class F> int by_type(apnn_dtype t, F &&f)
{
    switch (t) {
        case APNN_F32: return f(float{});
        case APNN_F16: return f(_Float16{});
        default: return f(__bf16{});
    }
}

// 16 bytes of elements
template <class T> struct alignas(16) Pack16 {
    static constexpr int n = 16 / static_cast<int>(sizeof(T));
    T v[n];
};

// Eight neighbouring elements as fp32, whatever their alignment (one or two 16-byte loads).
template <class T> __device__ __forceinline__ void load8(const T *from, float (&to)[8])
{
    T raw[8];
    __builtin_memcpy(raw, from, sizeof raw);
#pragma unroll
    for (int j = 0; j < 8; ++j) to[j] = static_cast<float>(raw[j]);
}
template <class T> __device__ __forceinline__ void store8(const float (&from)[8], T *to)
{
    T raw[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) raw[j] = static_cast<T>(from[j]);
    __builtin_memcpy(to, raw, sizeof raw);
}

// n / d for 0 <= n, 0 < d: in 32 bits where they do, which takes a third of the instructions.
__device__ __forceinline__ int64_t quotient(int64_t n, int64_t d)
{
    if (((n | d) >> 32) == 0) return static_cast<uint32_t>(n) / static_cast<uint32_t>(d);
    return n / d;
}

}  // namespace apnn
