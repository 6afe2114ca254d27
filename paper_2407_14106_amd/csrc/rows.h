// 16-byte pieces of feature rows at any width and alignment, for the kernels that
// work on a row in pieces (embedding, dropout).
#pragma once

#include "common.h"

namespace gt {

constexpr int64_t kFarBytes = int64_t(256) << 20;  // the last-level cache: results beyond it are stored past it

// 16 bytes at any element's address (global accesses need no more alignment).
template <typename T>
struct Piece {
    static constexpr int E = 4;
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct Piece<uint16_t> {
    static constexpr int E = 8;
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
};

template <typename T>
__device__ __forceinline__ void load_piece(float (&o)[Piece<T>::E], const T* p) {
    const typename Piece<T>::type x = *reinterpret_cast<const typename Piece<T>::type*>(p);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if constexpr (sizeof(T) == 2) o[2 * t] = bf16lo(x[t]), o[2 * t + 1] = bf16hi(x[t]);
        else o[t] = __uint_as_float(x[t]);
    }
}
template <typename T>
__device__ __forceinline__ void store_piece(T* p, const float (&o)[Piece<T>::E], bool far) {
    typename Piece<T>::type x;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if constexpr (sizeof(T) == 2) x[t] = pack_bf16x2(o[2 * t], o[2 * t + 1]);
        else x[t] = __float_as_uint(o[t]);
    }
    if (far) __builtin_nontemporal_store(x, reinterpret_cast<typename Piece<T>::type*>(p));
    else *reinterpret_cast<typename Piece<T>::type*>(p) = x;
}
template <typename T>
__device__ __forceinline__ float load_one(const T* p) {
    if constexpr (sizeof(T) == 2) return bf16_to_f32(*p);
    else return *p;
}
template <typename T>
__device__ __forceinline__ void store_one(T* p, float v) {
    if constexpr (sizeof(T) == 2) *p = f32_to_bf16(v);
    else *p = v;
}

// An id or a label of either type; ids outside [0, most) are -1.
__device__ __forceinline__ int64_t load_id(const void* p, bool wide, int64_t i, int64_t most) {
    const int64_t v = wide ? static_cast<const int64_t*>(p)[i] : int64_t(static_cast<const int32_t*>(p)[i]);
    return v >= 0 && v < most ? v : -1;
}

}  // namespace gt
