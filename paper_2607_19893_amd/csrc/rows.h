// Rows of a token matrix that TPR threads share: their sums and weights, and
// pieces of rows at any alignment of an element (device code of the norms).
#pragma once

#include "vec16.h"

namespace gsmi {

// Sum over the TPR adjacent threads of a row; part: a float a wave in LDS.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* part) {
    if (TPR < GS_WAVE) {
        v = dpp_row_sum(v);
#ifdef __HIP_DEVICE_COMPILE__
        if (TPR == 32) {                       // odd and even rows of 16 swapped between two copies
            const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        }
#endif
        return v;
    }
    v = wave_sum(v);
    if (TPR == GS_WAVE) return v;
    const int w = threadIdx.x / GS_WAVE;
    if (lane_id() == 0) part[w] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < TPR / GS_WAVE; ++i) v += part[i];
    __syncthreads();
    return v;
}

// N weights from column col on (zeros past the row's end).
template <int N, bool WHOLE>
__device__ __forceinline__ void load_weight(const float* weight, int col, int cols, float* w) {
    if (WHOLE) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (col < cols) v = *reinterpret_cast<const float4*>(weight + col + i);
            w[i] = v.x;
            w[i + 1] = v.y;
            w[i + 2] = v.z;
            w[i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = col + i < cols ? weight[col + i] : 0.0f;
    }
}

// N consecutive elements at any multiple of an element's size: one 16-byte load
// or store where all N are there (global memory takes them at any alignment),
// the first `there` one by one where the row ends inside (TAIL: it may), zeros
// behind.  bf16 rows of 1001 columns move as fast so as rows of 1000.
template <typename T, bool TAIL>
struct Span {
    static constexpr int N = Piece<T>::N;
    typedef typename Piece<T>::vec vec;
    typedef vec __attribute__((aligned(sizeof(T)))) loose;
    vec v;

    __device__ __forceinline__ void load(const T* p, int there) {
        v = vec{};
        if (there >= N) {
            v = *reinterpret_cast<const loose*>(p);
        } else if (TAIL) {
#pragma unroll
            for (int i = 0; i < N - 1; ++i)
                if (i < there) v[i] = p[i];
        }
    }
    __device__ __forceinline__ void floats(float* f) const {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = (float)v[i];
    }
    // rounded to nearest even; STREAM: past the caches, for what nobody reads soon
    template <bool STREAM = false>
    static __device__ __forceinline__ void store(T* p, int there, const float* f) {
        vec v;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (T)f[i];
        if (there >= N) {
            if (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<loose*>(p));
            else *reinterpret_cast<loose*>(p) = v;
        } else if (TAIL) {
#pragma unroll
            for (int i = 0; i < N - 1; ++i)
                if (i < there) p[i] = v[i];
        }
    }
};

// N floats from column col on (zeros past the row's end), at any alignment of a float.
template <int N, bool TAIL>
__device__ __forceinline__ void load_floats(const float* p, int col, int cols, float* w) {
    typedef float quad __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        if (col + i + 4 <= cols) {
            const quad v = *reinterpret_cast<const quad*>(p + col + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[i + j] = v[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[i + j] = TAIL && col + i + j < cols ? p[col + i + j] : 0.0f;
        }
    }
}

}  // namespace gsmi
