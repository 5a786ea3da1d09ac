// Token operators that a row's bytes bound: the root-mean-square norm with the
// residual's addition (into the tokens' type or 8 bits), its gradient, and the
// rotation by position.
#include <cmath>
#include <algorithm>

#include "common.h"
#include "internal.h"
#include "vec16.h"

namespace gsmi {

namespace {

// ---------------------------------------------------------------------------
// Norm.  A row is read once, kept in registers as floats, reduced, and written:
// s = x + residual, y = s w / sqrt(mean s^2 + eps).  Bound by HBM bytes.
// TPR threads share a row: thread t of them owns the 16-byte pieces t, t + TPR,
// ... (E elements in registers).  A wave a row needs no barrier and is taken
// while a row fits 32 elements a lane; longer rows take four.  Rows of up to 256
// columns are taken by the lanes that own one block of GS_NORM_BLOCK columns (16
// or 32), several to a wave: 74,724 fp32 rows of 80 columns into 8 bits took 47
// us with a wave each, whose lanes were two thirds idle, and take 18 so.
//   50,001 bf16 rows of 1536 with a residual into 8 bits and scales: 99 us, 5.5
// TB/s.  Rows that are not whole aligned pieces are loaded an element at a time:
// bf16 rows of 1001 reach 1.2 TB/s where those of 1000 reach 5.7.  7 rows of 1024: 2.6 us, the start of a kernel and one read.
// ---------------------------------------------------------------------------

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

// Maximum over the lanes that own one block of GS_NORM_BLOCK columns: 16 lanes
// of 16-bit pieces, 32 of fp32 pieces (adjacent lanes, a block starts at a
// multiple of its lanes).
template <int LANES>
__device__ __forceinline__ float block_max(float v) {
    // within a row of 16 lanes: pairs, quads, halves mirrored, the row mirrored
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, true)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xF, 0xF, true)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xF, 0xF, true)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xF, 0xF, true)));
#ifdef __HIP_DEVICE_COMPILE__
    if (LANES == 32) {                         // and of two rows: odd and even ones swapped between two copies
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
#endif
    return v;
}

// max|s a w| over a block of GS_NORM_BLOCK columns, N of them a lane, as a float
// and what the largest product lost in its rounding.  a is a power of two.
// The second walk forms its products again: kept, they would take registers.
template <int N>
__device__ __forceinline__ void largest_product(const float* s, float a, const float* w, float& m, float& m_lo) {
    m = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, fabsf(s[i] * a * w[i]));
    m = block_max<GS_NORM_BLOCK / N>(m);
    m_lo = -INFINITY;
    asm volatile("" : "+v"(a));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float p = s[i] * a * w[i], lo = fmaf(s[i] * a, w[i], -p);
        m_lo = fmaxf(m_lo, fabsf(p) == m ? (p < 0.0f ? -lo : lo) : -INFINITY);
    }
    m_lo = block_max<GS_NORM_BLOCK / N>(m_lo);
}

// x w (r + r_lo) rounded to odd in fp32: the exact product cut towards zero,
// its last bit set if anything was cut.  Rounding that to fewer bits gives what
// rounding the exact product would.
__device__ __forceinline__ float odd_product(float x, float w, float r, float r_lo) {
#pragma clang fp contract(off)                 // v is the rounded product wherever it stands
    const float t = x * w, t_lo = fmaf(x, w, -t);
    const float v = t * r, e = fmaf(t, r, -v) + fmaf(t, r_lo, t_lo * r);
    const float hi = v + e, lo = (v - hi) + e;
    int bits = __float_as_int(hi);
    if (lo != 0.0f && (bits & 1) == 0 && hi != 0.0f && fabsf(hi) < INFINITY) bits += (lo > 0.0f) == (hi > 0.0f) ? 1 : -1;
    // infinite or NaN: the parts cannot be told apart, the plain product is right
    return fabsf(v) < INFINITY ? __int_as_float(bits) : v;
}

// N floats in e4m3, rounded to nearest even, the first `there` of them.
template <int N, bool WHOLE>
__device__ __forceinline__ void store_eight(uint8_t* __restrict__ q, int there, const float* v) {
    uint32_t b[N / 4];
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        int x = 0;
        x = __builtin_amdgcn_cvt_pk_fp8_f32(v[i], v[i + 1], x, false);
        x = __builtin_amdgcn_cvt_pk_fp8_f32(v[i + 2], v[i + 3], x, true);
        b[i / 4] = (uint32_t)x;
    }
    if (WHOLE) {
        if (N == 8) *reinterpret_cast<uint2*>(q) = make_uint2(b[0], b[N / 4 - 1]);
        else *reinterpret_cast<uint32_t*>(q) = b[0];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < there) q[i] = (uint8_t)(b[i / 4] >> (8 * (i % 4)));
    }
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

// Five waves a SIMD for 32 16-bit elements a lane: 40,000 bf16 rows of 2048 into 8
// bits 109 us, 113 with the four that the compiler settles for.
template <typename T, bool WHOLE, int TPR, int E>
__global__ void __launch_bounds__(GS_BLOCK, TPR == 64 && E == 32 && sizeof(T) == 2 ? 5 : 1)
    k_rms_norm(gs_norm_args a) {
    constexpr int N = Piece<T>::N, CH = E / N, RPB = GS_BLOCK / TPR;
    __shared__ float part[GS_BLOCK / GS_WAVE];
    const int t = threadIdx.x % TPR;
    const int64_t mine = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    if (TPR >= GS_WAVE && mine >= a.rows) return;          // whole waves
    // rows past the end of a shared wave: the last row's address, no columns
    const int64_t row = mine < a.rows ? mine : a.rows - 1;
    const int cols = mine < a.rows ? a.cols : 0;
    const T* __restrict__ x = static_cast<const T*>(a.x) + row * a.ld_x;
    const T* __restrict__ r = a.residual ? static_cast<const T*>(a.residual) + row * a.ld_residual : nullptr;
    // every load of the row is on its way before the first is used
    Raw<T, WHOLE> xs[CH], rs[CH];
    float s[CH][N], w[CH][N];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + t) * N;
        xs[c].load(x + col, cols - col);
        if (r) rs[c].load(r + col, cols - col);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) load_weight<N, WHOLE>(a.weight, (c * TPR + t) * N, cols, w[c]);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        xs[c].floats(s[c]);
        if (r) {
            float f[N];
            rs[c].floats(f);
#pragma unroll
            for (int i = 0; i < N; ++i) s[c][i] += f[i];
        }
    }
    float ss = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < N; ++i) ss = fmaf(s[c][i], s[c][i], ss);
    ss = row_sum<TPR>(ss, part);
    const float rho = 1.0f / sqrtf(ss / (float)a.cols + a.eps);
    if (a.total) {
        T* __restrict__ o = static_cast<T*>(a.total) + row * a.ld_total;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * TPR + t) * N;
            if (col < cols) store_piece<T, WHOLE>(o + col, cols - col, s[c]);
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + t) * N;
        if (a.y && col < cols) {
            float y[N];
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = s[c][i] * (rho * w[c][i]);
            store_piece<T, WHOLE>(static_cast<T*>(a.y) + row * a.ld_y + col, cols - col, y);
        }
    }
    if (a.q == nullptr) return;
    // 8 bits: y / scale = (s w) * 448 / max|s w|, the row's rho falls out.  The
    // product is carried in two floats and rounded to odd, so that the one
    // rounding to e4m3 that follows is that of the exact value.
    constexpr float kLeast = 1.17549435e-38f;  // of a scale: 2^-126
    bool edge = false;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + t) * N;
        float m, m_lo, q[N];
        largest_product<N>(s[c], 1.0f, w[c], m, m_lo);
        if (col >= cols) continue;           // below: no lane exchange
        const float scale = m * rho / 448.0f, r = 448.0f / m, r_lo = fmaf(-r, m_lo, fmaf(-r, m, 448.0f)) / m;
        edge |= !(m >= 0x1p-60f && m <= 0x1p60f && scale >= kLeast && scale < INFINITY);
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = odd_product(s[c][i], w[c][i], r, r_lo);
        if (col % GS_NORM_BLOCK == 0) a.q_scale[row * a.ld_scale + col / GS_NORM_BLOCK] = scale;
        store_eight<N, WHOLE>(a.q + row * a.ld_q + col, cols - col, q);
    }
    if (!__any(edge)) return;
    // Some block's product or quotient is near an end of fp32's range: the wave's
    // blocks once more.  With rho = f p2, f in [1, 2), the products (s p2) w are
    // y / f; where even they are tiny, up to 2^64 lifts them.  Both are powers of
    // two, so a block that needs no care gets the same bits again.
    const bool finite = rho > 0.0f && rho < INFINITY;
    const float p2 = finite ? __uint_as_float(__float_as_uint(rho) & 0x7F800000u) : 1.0f;
    const float f = finite ? __uint_as_float((__float_as_uint(rho) & 0x007FFFFFu) | 0x3F800000u) : rho;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + t) * N;
        float m, m_lo, some = 0.0f, q[N];      // some: 1 for a product that is not 0, though fp32 may not hold it
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (fabsf(s[c][i]) > 0.0f && fabsf(w[c][i]) > 0.0f) some = 1.0f;
        some = block_max<GS_NORM_BLOCK / N>(some);
        largest_product<N>(s[c], p2, w[c], m, m_lo);
        const float up = m < 0x1p-60f ? fminf(0x1p64f, 0x1p126f / p2) : 1.0f;
        float lift = p2 * up;
        largest_product<N>(s[c], lift, w[c], m, m_lo);
        asm volatile("" : "+v"(lift));         // its products are formed again, not held
        if (col >= cols) continue;           // below: no lane exchange
        float scale = m * f / 448.0f * (1.0f / up), r = 448.0f / m, r_lo = fmaf(-r, m_lo, fmaf(-r, m, 448.0f)) / m;
        if (!(scale >= kLeast)) {              // y of 0 or NaN alone, or a block too small for the quotient
            const bool small = some > 0.0f && finite;
            scale = small ? kLeast : 1.0f;
            r = small ? f * (0x1p126f / up) : f;
            r_lo = 0.0f;
        } else if (scale == INFINITY) {
            r = NAN;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = odd_product(s[c][i] * lift, w[c][i], r, r_lo);
        if (col % GS_NORM_BLOCK == 0) a.q_scale[row * a.ld_scale + col / GS_NORM_BLOCK] = scale;
        store_eight<N, WHOLE>(a.q + row * a.ld_q + col, cols - col, q);
    }
}

// Gradient of the norm: dx = r (g - n mean(g n)) + dtotal with g = dy w, n =
// total r, one read of dy, total and dtotal.  Every workgroup walks rows in
// steps of the grid and keeps dy n of its columns in registers; it writes one
// row of partial sums, and k_norm_dweight adds those in ascending order.
// Bound by HBM bytes: 20,000 fp32 rows of 768: 51 us with the weight's sums, 4.9
// TB/s; 60,000 bf16 rows of 1160: 106 us, 5.2 TB/s.
constexpr int kNormParts = 512;                // two workgroups a compute unit

inline int norm_parts(int32_t rows, int rpb) {
    const int64_t b = ((int64_t)rows + rpb - 1) / rpb;
    return (int)(b < kNormParts ? (b < 1 ? 1 : b) : kNormParts);
}

template <typename T, bool WHOLE, int TPR, int E>
__global__ void __launch_bounds__(TPR > GS_BLOCK ? TPR : GS_BLOCK) k_rms_norm_bwd(gs_norm_bwd_args a,
                                                                               float* __restrict__ parts) {
    constexpr int N = Piece<T>::N, CH = E / N, RPB = TPR < GS_BLOCK ? GS_BLOCK / TPR : 1;
    __shared__ float part[16];
    __shared__ float comb[RPB > 1 ? GS_BLOCK * N : 1];
    const int t = threadIdx.x % TPR;
    float dw[CH][N], w[CH][N];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        load_weight<N, WHOLE>(a.weight, (c * TPR + t) * N, a.cols, w[c]);
#pragma unroll
        for (int i = 0; i < N; ++i) dw[c][i] = 0.0f;
    }
    for (int64_t first = (int64_t)blockIdx.x * RPB; first < a.rows; first += (int64_t)gridDim.x * RPB) {
        // rows past the end: the last row's address, no columns
        const int64_t mine = first + threadIdx.x / TPR, row = mine < a.rows ? mine : a.rows - 1;
        const int cols = mine < a.rows ? a.cols : 0;
        const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
        const T* tot = static_cast<const T*>(a.total) + row * a.ld_total;
        Raw<T, WHOLE> ts[CH], ys[CH], ds[CH];
        float s[CH][N], g[CH][N];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * TPR + t) * N;
            ts[c].load(tot + col, cols - col);
            ys[c].load(dy + col, cols - col);
            if (WHOLE && a.dtotal)
                ds[c].load(static_cast<const T*>(a.dtotal) + row * a.ld_dtotal + col, cols - col);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            ts[c].floats(s[c]);
            ys[c].floats(g[c]);
        }
        float ss = 0.0f, gs = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ss = fmaf(s[c][i], s[c][i], ss);
                gs = fmaf(g[c][i] * w[c][i], s[c][i], gs);
            }
        ss = row_sum<TPR>(ss, part);
        gs = row_sum<TPR>(gs, part);
        const float r = 1.0f / sqrtf(ss / (float)a.cols + a.eps);
        const float mean = gs * r / (float)a.cols;         // mean of g n
        T* dx = static_cast<T*>(a.dx) + row * a.ld_dx;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * TPR + t) * N;
            if (col >= cols) continue;
            float d[N];
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = 0.0f;
            if (a.dtotal) {
                if (!WHOLE) ds[c].load(static_cast<const T*>(a.dtotal) + row * a.ld_dtotal + col, cols - col);
                ds[c].floats(d);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float n = s[c][i] * r;
                dw[c][i] = fmaf(g[c][i], n, dw[c][i]);
                d[i] += r * (g[c][i] * w[c][i] - n * mean);
            }
            store_piece<T, WHOLE>(dx + col, cols - col, d);
        }
    }
    float* __restrict__ out = parts + (int64_t)blockIdx.x * a.cols;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + t) * N;
        if (RPB > 1) {                                     // the rows side by side, in their order
            float* mine = comb + threadIdx.x * N;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) mine[i] = dw[c][i];
            __syncthreads();
            for (int k = threadIdx.x; k < TPR * N; k += GS_BLOCK) {
                float v = 0.0f;
#pragma unroll
                for (int u = 0; u < RPB; ++u) v += comb[u * TPR * N + k];
                if (c * TPR * N + k < a.cols) out[c * TPR * N + k] = v;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (col + i < a.cols) out[col + i] = dw[c][i];
        }
    }
}

// Sum of the partial rows, a column each: 64 columns by 16 slices of the rows
// in a workgroup, then the slices in ascending order.  Latency: 512 parts of 768
// columns 4.4 us.
__global__ void __launch_bounds__(1024) k_norm_dweight(const float* __restrict__ parts, int n, int cols,
                                                       float* __restrict__ dweight) {
    __shared__ float sum[16][GS_WAVE];
    const int l = threadIdx.x % GS_WAVE, w = threadIdx.x / GS_WAVE;
    const int col = blockIdx.x * GS_WAVE + l;
    const int per = (n + 15) / 16;
    float v = 0.0f;
    if (col < cols)
#pragma unroll 8
        for (int i = w * per; i < min(n, (w + 1) * per); ++i) v += parts[(int64_t)i * cols + col];
    sum[w][l] = v;
    __syncthreads();
    if (w == 0 && col < cols) {
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v += sum[i][l];
        dweight[col] = v;
    }
}

__global__ void k_zero_f32(float* p, int n) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) p[i] = 0.0f;
}

template <typename T>
bool whole(const void* p, int64_t ld, int bytes) {
    return p == nullptr || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && (ld * (int64_t)sizeof(T)) % bytes == 0);
}

template <typename T, bool WHOLE>
hipError_t norm_go(const gs_norm_args& a, hipStream_t st) {
    constexpr int N = Piece<T>::N, NARROW = GS_NORM_BLOCK / N;
    const uint32_t by4 = div_up(a.rows, 4), narrow = div_up(a.rows, GS_BLOCK / NARROW);
    if (a.cols <= GS_NORM_BLOCK) k_rms_norm<T, WHOLE, NARROW, N><<<narrow, GS_BLOCK, 0, st>>>(a);
    else if (a.cols <= 2 * GS_NORM_BLOCK) k_rms_norm<T, WHOLE, NARROW, 2 * N><<<narrow, GS_BLOCK, 0, st>>>(a);
    else if (a.cols <= 1024) k_rms_norm<T, WHOLE, 64, 16><<<by4, GS_BLOCK, 0, st>>>(a);
    else if (a.cols <= 1536) k_rms_norm<T, WHOLE, 64, 24><<<by4, GS_BLOCK, 0, st>>>(a);
    else if (a.cols <= 2048) k_rms_norm<T, WHOLE, 64, 32><<<by4, GS_BLOCK, 0, st>>>(a);
    else if (a.cols <= 8192) k_rms_norm<T, WHOLE, 256, 32><<<a.rows, GS_BLOCK, 0, st>>>(a);
    else k_rms_norm<T, WHOLE, 256, 64><<<a.rows, GS_BLOCK, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t norm_type(const gs_norm_args& a, hipStream_t st) {
    const bool w = a.cols % Piece<T>::N == 0 && whole<T>(a.x, a.ld_x, 16) && whole<T>(a.residual, a.ld_residual, 16) &&
                   whole<T>(a.total, a.ld_total, 16) && whole<T>(a.y, a.ld_y, 16) &&
                   whole<uint8_t>(a.q, a.ld_q, Piece<T>::N) && whole<float>(a.weight, 0, 16);
    return w ? norm_go<T, true>(a, st) : norm_go<T, false>(a, st);
}

template <typename T, bool WHOLE>
hipError_t norm_bwd_go(const gs_norm_bwd_args& a, float* parts, hipStream_t st) {
    constexpr int N = Piece<T>::N, NARROW = GS_NORM_BLOCK / N;
    const int n = norm_parts(a.rows, a.cols <= 2 * GS_NORM_BLOCK ? GS_BLOCK / NARROW : (a.cols <= 2048 ? 4 : 1));
    if (a.cols <= GS_NORM_BLOCK) k_rms_norm_bwd<T, WHOLE, NARROW, N><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else if (a.cols <= 2 * GS_NORM_BLOCK) k_rms_norm_bwd<T, WHOLE, NARROW, 2 * N><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else if (a.cols <= 1024) k_rms_norm_bwd<T, WHOLE, 64, 16><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else if (a.cols <= 1536) k_rms_norm_bwd<T, WHOLE, 64, 24><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else if (a.cols <= 2048) k_rms_norm_bwd<T, WHOLE, 64, 32><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else if (a.cols <= 4096) k_rms_norm_bwd<T, WHOLE, 256, 16><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else k_rms_norm_bwd<T, WHOLE, 1024, 16><<<n, 1024, 0, st>>>(a, parts);
    k_norm_dweight<<<div_up(a.cols, GS_WAVE), 1024, 0, st>>>(parts, n, a.cols, a.dweight);
    return hipGetLastError();
}

template <typename T>
hipError_t norm_bwd_type(const gs_norm_bwd_args& a, float* parts, hipStream_t st) {
    const bool w = a.cols % Piece<T>::N == 0 && whole<T>(a.dy, a.ld_dy, 16) && whole<T>(a.total, a.ld_total, 16) &&
                   whole<T>(a.dtotal, a.ld_dtotal, 16) && whole<T>(a.dx, a.ld_dx, 16) && whole<float>(a.weight, 0, 16);
    return w ? norm_bwd_go<T, true>(a, parts, st) : norm_bwd_go<T, false>(a, parts, st);
}

// ---------------------------------------------------------------------------
// Rotation by position.  Bound by HBM bytes: every element is read and written
// once.  A workgroup takes `per` tokens: their cosines and sines (one fp64
// product, one reduction and one sincos a pair) go to LDS once and serve every
// head of both tensors; then each thread turns V pairs at a time, which are
// two V-element pieces of the head in either layout, and copies what is left
// of the heads.  50,000 fp32 tokens, 8 + 8 heads of 64, three quarters turned by
// three axes: 97 us, 4.2 TB/s; 32,768 bf16 tokens, 32 + 8 heads of 128: 132 us,
// 5.1 TB/s.  Two and four pieces of a thread in flight took as long.  Where the
// pairs are not whole pieces a thread turns four or one at a time: heads of 128 with
// 64, 60 and 63 pairs reach 5.1, 3.9 and 2.2 TB/s.
// ---------------------------------------------------------------------------

constexpr int kRotTrig = 2048;                 // pairs of a workgroup's tokens in LDS (16 KB)

struct RotArgs {
    gs_rotary_args a;
    int per;                                   // tokens of a workgroup
};

template <typename T, int V>
__device__ __forceinline__ void load_some(const T* p, float* f) {
    typedef T vec __attribute__((ext_vector_type(V)));
    if (V == 1) {
        f[0] = (float)p[0];
    } else {
        const vec v = *reinterpret_cast<const vec*>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = (float)v[i];
    }
}

template <typename T, int V>
__device__ __forceinline__ void store_some(T* p, const float* f) {
    typedef T vec __attribute__((ext_vector_type(V)));
    if (V == 1) {
        p[0] = (T)f[0];
    } else {
        vec v;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (T)f[i];
        *reinterpret_cast<vec*>(p) = v;
    }
}

template <typename T, int V, bool INTER>
__global__ void __launch_bounds__(GS_BLOCK) k_rotary(RotArgs ra) {
    const gs_rotary_args& a = ra.a;
    __shared__ __attribute__((aligned(16))) float2 trig[kRotTrig];
    const int t0 = blockIdx.x * ra.per;
    const int n = min(ra.per, a.tokens - t0);
    const int P = a.pairs;
    for (int i = threadIdx.x; i < n * P; i += GS_BLOCK) {
        const int t = i / P, j = i - t * P;
        int axis = 0;
        if (j >= a.axis_pairs[0]) axis = 1;
        if (axis == 1 && j >= a.axis_pairs[0] + a.axis_pairs[1]) axis = 2;
        const double turns = (double)a.pos[(int64_t)(t0 + t) * a.ld_pos + axis] * (double)a.freq[j] *
                             0.15915494309189533577;
        float sn, cs;
        sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
        trig[i] = make_float2(a.amplitude * cs, a.amplitude * (a.inverse ? -sn : sn));
    }
    __syncthreads();
    const int turn = P / V, rest = (a.dim - 2 * P + V - 1) / V, items = turn + rest;
#pragma unroll 1
    for (int k = 0; k < a.n_tensors; ++k) {
        const bool same = a.in[k].ptr == a.out[k].ptr;     // in place: nothing to copy
        const int used = same ? turn : items;
        const int each = a.heads[k] * used;
        const T* in = static_cast<const T*>(a.in[k].ptr);
        T* out = static_cast<T*>(a.out[k].ptr);
        for (int i = threadIdx.x; i < n * each; i += GS_BLOCK) {
            const int t = i / each, h = (i - t * each) / used, m = i - t * each - h * used;
            const T* p = in + (int64_t)(t0 + t) * a.in[k].ld_row + (int64_t)h * a.in[k].ld_head;
            T* o = out + (int64_t)(t0 + t) * a.out[k].ld_row + (int64_t)h * a.out[k].ld_head;
            if (m < turn) {
                const int j = m * V, e0 = INTER ? 2 * j : j, e1 = INTER ? 2 * j + V : P + j;
                float u[2 * V], y[2 * V];
                load_some<T, V>(p + e0, u);
                load_some<T, V>(p + e1, u + V);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float2 cs = trig[t * P + j + v];
                    const int ia = INTER ? 2 * v : v, ib = INTER ? 2 * v + 1 : V + v;
                    y[ia] = u[ia] * cs.x - u[ib] * cs.y;
                    y[ib] = u[ia] * cs.y + u[ib] * cs.x;
                }
                store_some<T, V>(o + e0, y);
                store_some<T, V>(o + e1, y + V);
            } else {
                const int e = 2 * P + (m - turn) * V;
                float u[V];
                load_some<T, V>(p + e, u);
                store_some<T, V>(o + e, u);
            }
        }
    }
}

template <typename T, int V>
hipError_t rotary_go(const RotArgs& r, hipStream_t st) {
    // a launch holds fewer than 2^32 threads: tokens of more than 2^23 workgroups go in several
    const int64_t most = (int64_t)r.per << 23;
    for (int64_t first = 0; first < r.a.tokens; first += most) {
        RotArgs s = r;
        s.a.tokens = (int32_t)std::min<int64_t>(most, r.a.tokens - first);
        s.a.pos = r.a.pos ? r.a.pos + first * r.a.ld_pos : nullptr;
        for (int i = 0; i < r.a.n_tensors; ++i)
            for (gs_rows* t : {&s.a.in[i], &s.a.out[i]})
                if (t->ptr) t->ptr = static_cast<T*>(t->ptr) + first * t->ld_row;
        const uint32_t grid = div_up(s.a.tokens, r.per);
        if (r.a.interleaved) k_rotary<T, V, true><<<grid, GS_BLOCK, 0, st>>>(s);
        else k_rotary<T, V, false><<<grid, GS_BLOCK, 0, st>>>(s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Whether every V-element piece that the kernel touches is aligned to its size.
template <typename T>
bool pieces(const gs_rotary_args& a, int V) {
    if (a.pairs % V != 0 || a.dim % V != 0) return false;
    for (int i = 0; i < a.n_tensors; ++i)
        for (const gs_rows* r : {&a.in[i], &a.out[i]})
            if (!whole<T>(r->ptr, r->ld_row, V * (int)sizeof(T)) || !whole<T>(r->ptr, r->ld_head, V * (int)sizeof(T)))
                return false;
    return true;
}

template <typename T>
hipError_t rotary_type(const gs_rotary_args& a, hipStream_t st) {
    RotArgs r;
    r.a = a;
    // tokens of a workgroup: about eight pieces a thread, as many as the
    // cosines' LDS holds, and enough workgroups to fill the chip
    const int64_t row = (int64_t)(a.heads[0] + (a.n_tensors > 1 ? a.heads[1] : 0)) * a.dim / (2 * Piece<T>::N) + 1;
    int64_t per = std::max<int64_t>(1, 2048 / row);
    if (a.pairs > 0) per = std::min<int64_t>(per, kRotTrig / a.pairs);
    per = std::min<int64_t>(per, std::max<int64_t>(1, a.tokens / 1024));
    r.per = (int)std::max<int64_t>(1, per);
    constexpr int N = Piece<T>::N;
    if (pieces<T>(a, N)) return rotary_go<T, N>(r, st);
    if (N > 4 && pieces<T>(a, 4)) return rotary_go<T, 4>(r, st);
    return rotary_go<T, 1>(r, st);
}

}  // namespace

// A launch holds fewer than 2^32 threads, a row takes up to 256: more rows than
// 2^23 go in several.
hipError_t launch_rms_norm(const gs_norm_args& a, hipStream_t st) {
    constexpr int32_t kMost = 1 << 23;
    const int64_t size = a.dtype == GS_F32 ? 4 : 2;
    auto at = [](const void* p, int64_t bytes) {
        return p ? const_cast<char*>(static_cast<const char*>(p)) + bytes : nullptr;
    };
    for (int64_t first = 0; first < a.rows; first += kMost) {
        gs_norm_args b = a;
        b.rows = (int32_t)std::min<int64_t>(kMost, a.rows - first);
        b.x = at(a.x, first * a.ld_x * size);
        b.residual = at(a.residual, first * a.ld_residual * size);
        b.total = at(a.total, first * a.ld_total * size);
        b.y = at(a.y, first * a.ld_y * size);
        b.q = reinterpret_cast<uint8_t*>(at(a.q, first * a.ld_q));
        b.q_scale = reinterpret_cast<float*>(at(a.q_scale, first * a.ld_scale * 4));
        const hipError_t e = b.dtype == GS_F32    ? norm_type<float>(b, st)
                             : b.dtype == GS_BF16 ? norm_type<bf16_t>(b, st)
                                                  : norm_type<f16_t>(b, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// For the most partial rows that any type's kernel of this width writes.
size_t rms_norm_bwd_ws_bytes(int32_t rows, int32_t cols) {
    return align256((size_t)norm_parts(rows, cols <= 2048 ? 4 : 1) * (size_t)cols * 4);
}

hipError_t launch_rms_norm_bwd(const gs_norm_bwd_args& a, void* ws, hipStream_t st) {
    float* parts = static_cast<float*>(ws);
    if (a.rows == 0) {
        k_zero_f32<<<div_up(a.cols, GS_BLOCK), GS_BLOCK, 0, st>>>(a.dweight, a.cols);
        return hipGetLastError();
    }
    if (a.dtype == GS_F32) return norm_bwd_type<float>(a, parts, st);
    return a.dtype == GS_BF16 ? norm_bwd_type<bf16_t>(a, parts, st) : norm_bwd_type<f16_t>(a, parts, st);
}

hipError_t launch_rotary(const gs_rotary_args& a, hipStream_t st) {
    if (a.dtype == GS_F32) return rotary_type<float>(a, st);
    return a.dtype == GS_BF16 ? rotary_type<bf16_t>(a, st) : rotary_type<f16_t>(a, st);
}

}  // namespace gsmi
