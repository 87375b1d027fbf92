// Shared by the kernels in which lists of token ids meet dense rows of 32- or 16-bit floats (embedding.hip, distill.hip, logits.hip).
#pragma once

#include <math.h>
#include <type_traits>

#include "spmm_internal.h"

namespace scorch {

typedef _Float16 f16;
typedef __bf16 bf16;

// N elements of type T at the alignment of one: gfx950 takes global loads and stores of up to 16 bytes at any address, so rows of odd
// length or stride need no kernel of their own.
template <typename T, int N> struct Pack {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// N elements from p as floats.
template <typename T, int N> __device__ __forceinline__ void load_floats(const T *p, float (&x)[N]) {
    const typename Pack<T, N>::type v = *reinterpret_cast<const typename Pack<T, N>::type *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)v[i];
}
// The first n < N of them; the others are `rest`.
template <typename T, int N> __device__ __forceinline__ void load_floats_part(const T *p, int n, float rest, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = i < n ? (float)p[i] : rest;
}
// 16 bytes as they are in memory, for values that stay in registers: a vector of 16-bit types is kept as a register per element by the compiler.
typedef uint32_t raw16 __attribute__((ext_vector_type(4)));
typedef uint32_t raw16_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t raw16_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t raw8_at4 __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t raw8_at2 __attribute__((ext_vector_type(2), aligned(2)));
template <typename T> __device__ __forceinline__ raw16 load_raw16(const T *p) {
    return *reinterpret_cast<const std::conditional_t<sizeof(T) == 4, raw16_at4, raw16_at2> *>(p);
}
// The first BYTES, 8 or 16, of them.
template <typename T, int BYTES> __device__ __forceinline__ raw16 load_raw(const T *p) {
    if constexpr (BYTES == 16) return load_raw16(p);
    else {
        typedef std::conditional_t<sizeof(T) == 4, raw8_at4, raw8_at2> at_element;
        const at_element v = *reinterpret_cast<const at_element *>(p);
        return raw16{v[0], v[1], 0, 0};
    }
}
// Element i of them as a float.
template <typename T> __device__ __forceinline__ float element(const raw16 &v, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[i]);
    const uint32_t pair = v[i / 2];
    if constexpr (std::is_same_v<T, bf16>) return __uint_as_float(i % 2 ? pair & 0xffff0000u : pair << 16);
    return (float)__builtin_bit_cast(f16, (uint16_t)(i % 2 ? pair >> 16 : pair));
}

// N floats, rounded to the nearest T (ties to even), the only rounding on the way to a 16-bit result.
template <typename T, int N, bool NT = false> __device__ __forceinline__ void store_floats(T *p, const float (&x)[N]) {
    typename Pack<T, N>::type v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (T)x[i];
    auto *q = reinterpret_cast<typename Pack<T, N>::type *>(p);
    if constexpr (NT) __builtin_nontemporal_store(v, q);
    else *q = v;
}
template <typename T, int N> __device__ __forceinline__ void store_floats_part(T *p, int n, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) p[i] = (T)x[i];
}

// 16 bytes of the wider of two types
template <typename A, typename B> constexpr int kPer16 = 16 / (sizeof(A) > sizeof(B) ? sizeof(A) : sizeof(B));

// A launch has fewer than 2^32 threads in each dimension.
inline bool grid_fits(int64_t blocks, int threads) { return blocks * threads < (1ll << 32); }

template <typename T> struct type_of {
    typedef T type;
};
// Calls f with a type_of<> of the C type; false if `type` names none.
template <typename F> bool with_type(int32_t type, F f) {
    switch (type) {
        case SCORCH_TYPE_F32: f(type_of<float>()); return true;
        case SCORCH_TYPE_BF16: f(type_of<bf16>()); return true;
        case SCORCH_TYPE_F16: f(type_of<f16>()); return true;
        default: return false;
    }
}

}  // namespace scorch
