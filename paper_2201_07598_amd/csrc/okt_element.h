// Elements of the operators' tensors: fp32, bf16 or fp16 in memory, fp32 in registers.
#ifndef OKT_ELEMENT_H
#define OKT_ELEMENT_H

#include "okt_device.h"

namespace okt {

typedef float f32x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Eight;
#define OKT_EIGHT(T)                                                                  \
    template <> struct Eight<T> {                                                     \
        typedef T vec __attribute__((ext_vector_type(8)));                            \
        /* the same at the alignment of one element: rows of odd widths start there */ \
        struct __attribute__((packed, aligned(sizeof(T)))) any { vec v; };            \
    };
OKT_EIGHT(float)
OKT_EIGHT(__bf16)
OKT_EIGHT(_Float16)
#undef OKT_EIGHT

// Eight neighbouring elements, wide loads at any alignment of an element.
template <typename T>
__device__ __forceinline__ f32x8 load_eight(const T* p) {
    return __builtin_convertvector(reinterpret_cast<const typename Eight<T>::any*>(p)->v, f32x8);
}

// Rounds to nearest, ties to even, as every store of the operators does.
template <typename T>
__device__ __forceinline__ void store_eight(T* p, f32x8 v) {
    reinterpret_cast<typename Eight<T>::any*>(p)->v = __builtin_convertvector(v, typename Eight<T>::vec);
}

// The first `count` of them; the rest reads as `rest` and is not written.
template <typename T>
__device__ __forceinline__ f32x8 load_some(const T* p, int count, float rest) {
    f32x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < count ? (float)p[i] : rest;
    return v;
}

template <typename T>
__device__ __forceinline__ void store_some(T* p, f32x8 v, int count) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) p[i] = (T)v[i];
}

inline bool known_dtype(int dtype) { return dtype == OKT_F32 || dtype == OKT_BF16 || dtype == OKT_F16; }
inline size_t dtype_bytes(int dtype) { return dtype == OKT_F32 ? 4 : 2; }

}  // namespace okt

#endif
