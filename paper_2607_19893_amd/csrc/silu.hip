// Gated SiLU whose inputs are kept in 8 bits for the gradient, and the gradient.
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace gsmi {

namespace {

// ---------------------------------------------------------------------------
// h = u sigma(u) v.  A thread takes 8 columns of a row, the four threads of a
// quad one block of GS_KEEP_BLOCK columns: its scale is the power of two 2^k,
// k the least with max|u| <= 448 2^k, so u / 2^k is exact in fp32 and the one
// rounding is that to e4m3.  Bound by HBM bytes: 8 and 1/16 an element of two
// 16-bit inputs, forward and (with h again) 10 and 1/16 on the way back.  40,000
// rows of 2048 bf16 columns: 118 us and 142, 5.6 and 5.8 TB/s (some of it stays in
// the last-level cache).
// ---------------------------------------------------------------------------

constexpr int kCols = 8;                       // of a thread
constexpr int kQuad = GS_KEEP_BLOCK / kCols;   // threads of a block
constexpr int kItems = 2;                      // of a thread, in flight together
static_assert(kQuad == 4, "a block is a quad of lanes");

// 8 consecutive elements as floats, at any alignment of an element; zeros behind `there`.
template <typename T, bool TAIL>
struct Eight {
    static constexpr int CH = kCols / Piece<T>::N;
    Span<T, TAIL> s[CH];
    __device__ __forceinline__ void load(const T* p, int there) {
#pragma unroll
        for (int c = 0; c < CH; ++c) s[c].load(p + c * Piece<T>::N, there - c * Piece<T>::N);
    }
    __device__ __forceinline__ void floats(float* f) const {
#pragma unroll
        for (int c = 0; c < CH; ++c) s[c].floats(f + c * Piece<T>::N);
    }
    static __device__ __forceinline__ void store(T* p, int there, const float* f) {
#pragma unroll
        for (int c = 0; c < CH; ++c) Span<T, TAIL>::store(p + c * Piece<T>::N, there - c * Piece<T>::N, f + c * Piece<T>::N);
    }
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 __attribute__((aligned(1))) loose_u32x2;

template <bool TAIL>
__device__ __forceinline__ void store_bytes(uint8_t* p, int there, const uint32_t* b) {
    if (there >= kCols) {
        *reinterpret_cast<loose_u32x2*>(p) = u32x2{b[0], b[1]};
    } else if (TAIL) {
#pragma unroll
        for (int i = 0; i < kCols - 1; ++i)
            if (i < there) p[i] = (uint8_t)(b[i / 4] >> (8 * (i % 4)));
    }
}

template <bool TAIL>
__device__ __forceinline__ u32x2 load_bytes(const uint8_t* p, int there) {
    u32x2 b = {0u, 0u};
    if (there >= kCols) {
        b = *reinterpret_cast<const loose_u32x2*>(p);
    } else if (TAIL) {
#pragma unroll
        for (int i = 0; i < kCols - 1; ++i)
            if (i < there) b[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
    }
    return b;
}

__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, true)));
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xF, 0xF, true)));
}

// 8 values in e4m3 with their block's scale byte k + 127.  NaN and infinities
// become NaN and do not touch the scale.
__device__ __forceinline__ uint32_t eight_bits(const float* f, uint32_t* b) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kCols; ++i) m = fmaxf(m, fabsf(f[i]) < INFINITY ? fabsf(f[i]) : 0.0f);
    m = quad_max(m);
    // m = 1.x 2^(e - 127), 448 = 1.75 2^8
    const int e = (int)(__float_as_uint(m) >> 23), up = (__float_as_uint(m) & 0x7FFFFFu) > 0x600000u;
    const int byte = max(0, e - 8 + up);
    const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);
    float v[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i) v[i] = fabsf(f[i]) < INFINITY ? f[i] * inv : NAN;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int x = 0;
        x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], x, false);
        x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], x, true);
        b[i] = (uint32_t)x;
    }
    return (uint32_t)byte;
}

__device__ __forceinline__ void wide(u32x2 b, uint32_t byte, float* f) {
    // 2^-127 is below the normal numbers
    const float scale = __uint_as_float(byte ? byte << 23 : 0x00400000u);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)b[i], false);
        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)b[i], true);
        f[4 * i] = lo[0] * scale;
        f[4 * i + 1] = lo[1] * scale;
        f[4 * i + 2] = hi[0] * scale;
        f[4 * i + 3] = hi[1] * scale;
    }
}

// sigma(u) = half^2 / (1 + t) with t = exp(-|u|), half = exp(-|u| / 2) where u is
// negative and 1 elsewhere: the halves go to either side of a product, so that it
// keeps its bits down to the least numbers (exp(-|u|) itself is gone at -87).
struct Sigma {
    float half, r, rest;                       // r = 1 / (1 + t); rest = 1 - sigma(u)
    __device__ __forceinline__ explicit Sigma(float u) {
        const float e = __expf(-0.5f * fabsf(u)), t = e * e;
        r = __builtin_amdgcn_rcpf(1.0f + t);
        half = u < 0.0f ? e : 1.0f;
        rest = u < 0.0f ? r : t * r;
    }
};

// Where a thread's item stands: items are rows of `per` threads (whole quads).
struct Place {
    int64_t row;
    int col, there;                            // there <= 0: past the row's or the matrix's end
};

__device__ __forceinline__ Place place(int64_t rows, int cols, int per, float inv_per, int k) {
    const int64_t first = (int64_t)blockIdx.x * (GS_BLOCK * kItems);
    const int64_t row0 = first / per;          // one division of the workgroup
    const int i = (int)(first - row0 * per) + k * GS_BLOCK + (int)threadIdx.x;
    // i < per + 512 < 2^21: the quotient is off by less than half a step of 1 / per
    const int r = (int)(((float)i + 0.5f) * inv_per);
    Place p;
    p.row = row0 + r;
    p.col = (i - r * per) * kCols;
    p.there = p.row < rows ? cols - p.col : 0;
    return p;
}

template <typename T, bool TAIL, bool GATED>
__global__ void __launch_bounds__(GS_BLOCK) k_gated_silu(gs_silu_args a, int per, float inv_per) {
    Place at[kItems];
    Eight<T, TAIL> us[kItems], vs[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        at[k] = place(a.rows, a.cols, per, inv_per, k);
        us[k].load(static_cast<const T*>(a.u) + at[k].row * a.ld_u + at[k].col, at[k].there);
        if (GATED) vs[k].load(static_cast<const T*>(a.v) + at[k].row * a.ld_v + at[k].col, at[k].there);
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int64_t row = at[k].row;
        const int col = at[k].col, there = at[k].there;
        float u[kCols], v[kCols], h[kCols];
        us[k].floats(u);
        if (GATED) vs[k].floats(v);
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            const Sigma s(u[i]);
            h[i] = u[i] * s.r * s.half * (GATED ? s.half * v[i] : s.half);
        }
        if (a.h) Eight<T, TAIL>::store(static_cast<T*>(a.h) + row * a.ld_h + col, there, h);
        if (a.u8) {
            uint32_t b[2], byte = eight_bits(u, b);
            store_bytes<TAIL>(a.u8 + row * a.ld_u8 + col, there, b);
            if (there > 0 && threadIdx.x % kQuad == 0) a.u_scale[row * a.ld_u_scale + col / GS_KEEP_BLOCK] = (uint8_t)byte;
            if (GATED) {
                byte = eight_bits(v, b);
                store_bytes<TAIL>(a.v8 + row * a.ld_v8 + col, there, b);
                if (there > 0 && threadIdx.x % kQuad == 0)
                    a.v_scale[row * a.ld_v_scale + col / GS_KEEP_BLOCK] = (uint8_t)byte;
            }
        }
    }
}

// du = dh v s (1 + u (1 - s)), dv = dh u s, h = u s v again, from what was kept.
template <typename T, bool TAIL, bool GATED>
__global__ void __launch_bounds__(GS_BLOCK) k_gated_silu_bwd(gs_silu_bwd_args a, int per, float inv_per) {
    Place at[kItems];
    Eight<T, TAIL> ds[kItems];
    u32x2 ub[kItems], vb[kItems];
    uint32_t uk[kItems], vk[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        at[k] = place(a.rows, a.cols, per, inv_per, k);
        const int64_t row = at[k].row;
        const int col = at[k].col, there = at[k].there;
        ds[k].load(static_cast<const T*>(a.dh) + row * a.ld_dh + col, there);
        ub[k] = load_bytes<TAIL>(a.u8 + row * a.ld_u8 + col, there);
        uk[k] = there > 0 ? a.u_scale[row * a.ld_u_scale + col / GS_KEEP_BLOCK] : 0;
        if (GATED) {
            vb[k] = load_bytes<TAIL>(a.v8 + row * a.ld_v8 + col, there);
            vk[k] = there > 0 ? a.v_scale[row * a.ld_v_scale + col / GS_KEEP_BLOCK] : 0;
        }
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int64_t row = at[k].row;
        const int col = at[k].col, there = at[k].there;
        float u[kCols], v[kCols], d[kCols], du[kCols], dv[kCols], h[kCols];
        ds[k].floats(d);
        wide(ub[k], uk[k], u);
        if (GATED) wide(vb[k], vk[k], v);
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            const Sigma s(u[i]);
            const float p = u[i] * s.r * s.half;
            du[i] = d[i] * s.half * (GATED ? v[i] : 1.0f) * (s.half * (s.r * fmaf(u[i], s.rest, 1.0f)));
            dv[i] = d[i] * s.half * p;
            h[i] = p * (GATED ? s.half * v[i] : s.half);
        }
        Eight<T, TAIL>::store(static_cast<T*>(a.du) + row * a.ld_du + col, there, du);
        if (GATED) Eight<T, TAIL>::store(static_cast<T*>(a.dv) + row * a.ld_dv + col, there, dv);
        if (a.h) Eight<T, TAIL>::store(static_cast<T*>(a.h) + row * a.ld_h + col, there, h);
    }
}

// A launch holds fewer than 2^32 threads: the rows go in launches of at most 2^23 workgroups.
inline int64_t rows_a_launch(int per) { return ((int64_t)GS_BLOCK * kItems << 23) / per; }

inline char* row_at(const void* p, int64_t bytes) {
    return p ? const_cast<char*>(static_cast<const char*>(p)) + bytes : nullptr;
}

template <typename T>
hipError_t silu_type(const gs_silu_args& all, hipStream_t st) {
    const int per = (int)div_up(all.cols, GS_KEEP_BLOCK) * kQuad;
    const int64_t most = rows_a_launch(per);
    for (int64_t first = 0; first < all.rows; first += most) {
        gs_silu_args a = all;
        a.rows = (int32_t)std::min<int64_t>(most, all.rows - first);
        a.u = row_at(all.u, first * all.ld_u * sizeof(T));
        a.v = row_at(all.v, first * all.ld_v * sizeof(T));
        a.h = row_at(all.h, first * all.ld_h * sizeof(T));
        a.u8 = reinterpret_cast<uint8_t*>(row_at(all.u8, first * all.ld_u8));
        a.v8 = reinterpret_cast<uint8_t*>(row_at(all.v8, first * all.ld_v8));
        a.u_scale = reinterpret_cast<uint8_t*>(row_at(all.u_scale, first * all.ld_u_scale));
        a.v_scale = reinterpret_cast<uint8_t*>(row_at(all.v_scale, first * all.ld_v_scale));
        const uint32_t grid = div_up((uint64_t)a.rows * per, GS_BLOCK * kItems);
        const float inv = 1.0f / (float)per;
        if (a.cols % kCols == 0) {
            if (a.v) k_gated_silu<T, false, true><<<grid, GS_BLOCK, 0, st>>>(a, per, inv);
            else k_gated_silu<T, false, false><<<grid, GS_BLOCK, 0, st>>>(a, per, inv);
        } else {
            if (a.v) k_gated_silu<T, true, true><<<grid, GS_BLOCK, 0, st>>>(a, per, inv);
            else k_gated_silu<T, true, false><<<grid, GS_BLOCK, 0, st>>>(a, per, inv);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t silu_bwd_type(const gs_silu_bwd_args& all, hipStream_t st) {
    const int per = (int)div_up(all.cols, GS_KEEP_BLOCK) * kQuad;
    const int64_t most = rows_a_launch(per);
    for (int64_t first = 0; first < all.rows; first += most) {
        gs_silu_bwd_args a = all;
        a.rows = (int32_t)std::min<int64_t>(most, all.rows - first);
        a.dh = row_at(all.dh, first * all.ld_dh * sizeof(T));
        a.du = row_at(all.du, first * all.ld_du * sizeof(T));
        a.dv = row_at(all.dv, first * all.ld_dv * sizeof(T));
        a.h = row_at(all.h, first * all.ld_h * sizeof(T));
        a.u8 = reinterpret_cast<const uint8_t*>(row_at(all.u8, first * all.ld_u8));
        a.v8 = reinterpret_cast<const uint8_t*>(row_at(all.v8, first * all.ld_v8));
        a.u_scale = reinterpret_cast<const uint8_t*>(row_at(all.u_scale, first * all.ld_u_scale));
        a.v_scale = reinterpret_cast<const uint8_t*>(row_at(all.v_scale, first * all.ld_v_scale));
        const uint32_t grid = div_up((uint64_t)a.rows * per, GS_BLOCK * kItems);
        const float inv = 1.0f / (float)per;
        if (a.cols % kCols == 0) {
            if (a.v8) k_gated_silu_bwd<T, false, true><<<grid, GS_BLOCK, 0, st>>>(a, per, inv);
            else k_gated_silu_bwd<T, false, false><<<grid, GS_BLOCK, 0, st>>>(a, per, inv);
        } else {
            if (a.v8) k_gated_silu_bwd<T, true, true><<<grid, GS_BLOCK, 0, st>>>(a, per, inv);
            else k_gated_silu_bwd<T, true, false><<<grid, GS_BLOCK, 0, st>>>(a, per, inv);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_gated_silu(const gs_silu_args& a, hipStream_t st) {
    if (a.dtype == GS_F32) return silu_type<float>(a, st);
    return a.dtype == GS_BF16 ? silu_type<bf16_t>(a, st) : silu_type<f16_t>(a, st);
}

hipError_t launch_gated_silu_bwd(const gs_silu_bwd_args& a, hipStream_t st) {
    if (a.dtype == GS_F32) return silu_bwd_type<float>(a, st);
    return a.dtype == GS_BF16 ? silu_bwd_type<bf16_t>(a, st) : silu_bwd_type<f16_t>(a, st);
}

}  // namespace gsmi
