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

// Eight elements as they lie in memory.
template <typename T>
__device__ __forceinline__ typename Eight<T>::vec raw_eight(const T* p) {
    return reinterpret_cast<const typename Eight<T>::any*>(p)->v;
}

// Drops the first `skip` (1 to 7) of eight elements, moves the rest to the front and puts zeros
// behind.  The ragged end of a row is the last eight elements of the row moved so: a
// load for each element, merged one by one, waits for memory each time.
template <typename T>
__device__ __forceinline__ typename Eight<T>::vec skip_elements(typename Eight<T>::vec v, uint32_t skip) {
    constexpr int WORDS = 2 * sizeof(T), PER = 4 / sizeof(T);          // words, elements of a word
    typedef uint32_t words __attribute__((ext_vector_type(WORDS)));
    words w = __builtin_bit_cast(words, v);
#pragma unroll
    for (int step = 4; step >= PER; step >>= 1)
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const uint32_t from = i + step / PER < WORDS ? w[i + step / PER < WORDS ? i + step / PER : 0] : 0;
            w[i] = skip & step ? from : w[i];
        }
    if (PER == 2) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const uint32_t from = (w[i] >> 16) | (i + 1 < WORDS ? w[i + 1 < WORDS ? i + 1 : 0] << 16 : 0);
            w[i] = skip & 1 ? from : w[i];
        }
    }
    return __builtin_bit_cast(typename Eight<T>::vec, w);
}

// Writes the first `count` (0 to 7) of them, in pieces of four, two and one.
template <typename T>
__device__ __forceinline__ void store_some(T* p, f32x8 v, int count) {
    struct __attribute__((packed, aligned(sizeof(T)))) Four { T v[4]; };
    struct __attribute__((packed, aligned(sizeof(T)))) Two { T v[2]; };
    T e[8];
#pragma unroll
    for (int i = 0; i < 7; ++i) e[i] = (T)v[i];
    if (count & 4) *reinterpret_cast<Four*>(p) = Four{{e[0], e[1], e[2], e[3]}};
    const T a = count & 4 ? e[4] : e[0], b = count & 4 ? e[5] : e[1], c = count & 4 ? e[6] : e[2];
    p += count & 4;
    if (count & 2) *reinterpret_cast<Two*>(p) = Two{{a, b}};
    if (count & 1) p[count & 2] = count & 2 ? c : a;
}

inline bool known_dtype(int dtype) { return dtype == OKT_F32 || dtype == OKT_BF16 || dtype == OKT_F16; }
inline size_t dtype_bytes(int dtype) { return dtype == OKT_F32 ? 4 : 2; }

}  // namespace okt

#endif
