// Element types of tensors that are not the server's own: 32-bit and 16-bit floating point, and vectors of them.
#pragma once
#include "common.h"

typedef __bf16 bf16_t;
typedef _Float16 f16_t;
template <class T, int W> struct VecOf { typedef T type __attribute__((ext_vector_type(W))); };
template <class T> struct VecOf<T, 1> { typedef T type; };
template <class T, int W> using Vec = typename VecOf<T, W>::type;

// W neighbouring elements, as 32-bit numbers; p starts on W elements (on 16 bytes where those are more)
template <class T, int W>
__device__ __forceinline__ Vec<float, W> load_vec(const T *p) {
    if constexpr (W * sizeof(T) <= 16) {
        const Vec<T, W> x = *reinterpret_cast<const Vec<T, W> *>(p);
        if constexpr (W == 1) return (float)x;
        else return __builtin_convertvector(x, Vec<float, W>);
    } else {                                       // 8 of 32 bits: two accesses
        static_assert(W == 8 && sizeof(T) == 4);
        const Vec<float, 4> a = *reinterpret_cast<const Vec<float, 4> *>(p), b = *reinterpret_cast<const Vec<float, 4> *>(p + 4);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}
// the same the other way: rounded to the nearest, ties to even; what is too large for T becomes infinite
template <class T, int W>
__device__ __forceinline__ void store_vec(T *p, Vec<float, W> v) {
    if constexpr (W * sizeof(T) <= 16) {
        Vec<T, W> x;
        if constexpr (W == 1) x = (T)v;
        else x = __builtin_convertvector(v, Vec<T, W>);
        *reinterpret_cast<Vec<T, W> *>(p) = x;
    } else {
        static_assert(W == 8 && sizeof(T) == 4);
        store_vec<T, 4>(p, __builtin_shufflevector(v, v, 0, 1, 2, 3));
        store_vec<T, 4>(p + 4, __builtin_shufflevector(v, v, 4, 5, 6, 7));
    }
}

inline size_t element_bytes(int32_t type) { return type == PS_F32 ? 4 : 2; }
inline bool is_element_type(int32_t type) { return type == PS_F32 || type == PS_BF16 || type == PS_F16; }
// whether rows of `cols` elements, `stride` elements apart, can be accessed w at a time (on 16 bytes where w elements are more)
inline bool rows_allow(const void *p, int32_t type, int64_t cols, int64_t stride, int w) {
    const size_t want = w * element_bytes(type) < 16 ? w * element_bytes(type) : 16;
    return cols % w == 0 && ((uintptr_t)p % want) == 0 && ((size_t)stride * element_bytes(type)) % want == 0;
}
