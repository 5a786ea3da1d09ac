// 16-byte pieces of a token matrix's three element types, as floats in
// registers (device code of the token operators).
#pragma once

#include "common.h"

namespace gsmi {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

template <typename T>
struct Piece {
    static constexpr int N = 16 / sizeof(T);       // elements of a 16-byte piece
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
};

// N consecutive elements at p, first as they are in memory (so that several
// loads can be on their way), then as floats.  WHOLE: one 16-byte load (p
// aligned) if any is there; otherwise the first `there` elements one by one.
// Zeros behind.
template <typename T, bool WHOLE>
struct Raw {
    static constexpr int N = Piece<T>::N;
    typename Piece<T>::vec v;

    __device__ __forceinline__ void load(const T* p, int there) {
        v = typename Piece<T>::vec{};
        if (WHOLE) {
            if (there > 0) v = *reinterpret_cast<const typename Piece<T>::vec*>(p);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < there) v[i] = p[i];
        }
    }
    __device__ __forceinline__ void floats(float* f) const {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = (float)v[i];
    }
};

// The way back, rounded to nearest even.
template <typename T, bool WHOLE>
__device__ __forceinline__ void store_piece(T* p, int there, const float* f) {
    constexpr int N = Piece<T>::N;
    if (WHOLE) {
        typename Piece<T>::vec v;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (T)f[i];
        *reinterpret_cast<typename Piece<T>::vec*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < there) p[i] = (T)f[i];
    }
}

}  // namespace gsmi
