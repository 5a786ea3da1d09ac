// Layer norm with the residual's addition, and its gradient.
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace gsmi {

namespace {

// ---------------------------------------------------------------------------
// Layer norm: s = x + residual, m = mean s, y = (s - m) w / sqrt(mean (s - m)^2
// + eps) + b.  A row is read once and kept in registers as floats, so the
// variance is summed from the differences themselves (mean s^2 - m^2 would lose
// the bits of rows whose mean is large).  TPR threads share a row, thread t of
// them owns the 16-byte pieces t, t + TPR, ...  Bound by HBM bytes: 60,001 bf16
// rows of 1001 columns with a residual 106 us, 4.5 TB/s (pieces are loaded at any
// alignment of an element, so an odd width costs nothing; a copy runs at 4.8).
// ---------------------------------------------------------------------------

// Rows whose squares leave fp32's range (differences of 2^57 and more; or, with
// next to no eps, of 2^-40 and less): their sums are taken over the differences
// times a power of two, and 1/sqrt(mean + eps) is that power times the root of
// what they sum to.  1 for any other row; fp16 reaches neither end.
template <typename T>
__device__ __forceinline__ float fitting(float ss, float eps) {
    if (sizeof(T) == 2 && !__is_same(T, bf16_t)) return 1.0f;
    return ss == INFINITY ? 0x1p-72f : ss < 0x1p-80f && eps < 0x1p-100f ? 0x1p100f : 1.0f;
}

// NaN where even the differences are infinite.
__device__ __forceinline__ float root(float ss, int cols, float eps, float k) {
    return ss == INFINITY ? NAN : 1.0f / sqrtf(ss / (float)cols + eps * k * k);
}

template <typename T, bool TAIL, int TPR, int E>
__global__ void __launch_bounds__(GS_BLOCK) k_layer_norm(gs_layer_args a) {
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
    Span<T, TAIL> xs[CH], rs[CH];
    float s[CH][N], w[CH][N], b[CH][N];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + t) * N;
        xs[c].load(x + col, cols - col);
        if (r) rs[c].load(r + col, cols - col);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + t) * N;
        load_floats<N, TAIL>(a.weight, col, cols, w[c]);
        if (a.bias) {
            load_floats<N, TAIL>(a.bias, col, cols, b[c]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) b[c][i] = 0.0f;
        }
    }
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        xs[c].floats(s[c]);
        if (r) {
            float f[N];
            rs[c].floats(f);
#pragma unroll
            for (int i = 0; i < N; ++i) s[c][i] += f[i];
        }
#pragma unroll
        for (int i = 0; i < N; ++i) sum += s[c][i];
    }
    const float mean = row_sum<TPR>(sum, part) / (float)a.cols;
    if (a.total) {
        T* __restrict__ o = static_cast<T*>(a.total) + row * a.ld_total;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * TPR + t) * N;
            Span<T, TAIL>::store(o + col, cols - col, s[c]);
        }
    }
    float ss = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + t) * N;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[c][i] = (TAIL ? col + i < cols : col < cols) ? s[c][i] - mean : 0.0f;
            ss = fmaf(s[c][i], s[c][i], ss);
        }
    }
    ss = row_sum<TPR>(ss, part);
    const float k = fitting<T>(ss, a.eps);
    if (__any(k != 1.0f)) {                    // the same for all waves of a row
        ss = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < N; ++i) ss = fmaf(s[c][i] * k, s[c][i] * k, ss);
        ss = row_sum<TPR>(ss, part);
    }
    const float rho = k * root(ss, a.cols, a.eps, k);
    T* __restrict__ o = static_cast<T*>(a.y) + row * a.ld_y;
    if (a.y)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * TPR + t) * N;
            float y[N];
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = fmaf(s[c][i] * rho, w[c][i], b[c][i]);
            Span<T, TAIL>::store(o + col, cols - col, y);
        }
}

// Gradient: with n = (s - m) rho and g = dy w,
//   dx = rho (g - mean g - n mean(g n)) + dtotal;  dw = sum dy n;  db = sum dy.
// One read of dy, total and dtotal; two rounds of sums (of s and g, then of
// (s - m)^2 and g (s - m)).  Every workgroup walks rows in steps of the grid,
// keeps dy n and dy of its columns in registers and writes them as one row of
// partial sums; k_layer_join adds those in ascending order.  Bound by HBM bytes:
// 24,000 fp32 rows of 768 columns 60 us, 54 of them this kernel at 5.4 TB/s.
constexpr int kLayerParts = 512;               // two workgroups a compute unit

inline int layer_parts(int32_t rows, int rpb) {
    const int64_t b = ((int64_t)rows + rpb - 1) / rpb;
    return (int)(b < kLayerParts ? (b < 1 ? 1 : b) : kLayerParts);
}

// Adds the RPB rows side by side of a workgroup, in their order, into one row of
// partial sums (columns first .. first + TPR * N).
template <int TPR, int N, int RPB>
__device__ __forceinline__ void put_part(float* comb, const float* v, float* out, int first, int cols) {
    const int t = threadIdx.x % TPR;
    if (RPB > 1) {
        float* mine = comb + threadIdx.x * N;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) mine[i] = v[i];
        __syncthreads();
        for (int k = threadIdx.x; k < TPR * N; k += GS_BLOCK) {
            float sum = 0.0f;
#pragma unroll
            for (int u = 0; u < RPB; ++u) sum += comb[u * TPR * N + k];
            if (first + k < cols) out[first + k] = sum;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (first + t * N + i < cols) out[first + t * N + i] = v[i];
    }
}

template <typename T, bool TAIL, int TPR, int E>
__global__ void __launch_bounds__(TPR > GS_BLOCK ? TPR : GS_BLOCK) k_layer_norm_bwd(gs_layer_bwd_args a,
                                                                                 float* __restrict__ parts) {
    constexpr int N = Piece<T>::N, CH = E / N, RPB = TPR < GS_BLOCK ? GS_BLOCK / TPR : 1;
    constexpr bool LATE = E >= 32;             // dtotal is loaded where it is used: there are no registers to hold it
    __shared__ float part[16];
    __shared__ float comb[RPB > 1 ? GS_BLOCK * N : 1];
    const int t = threadIdx.x % TPR;
    float dw[CH][N], db[CH][N], w[CH][N];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        load_floats<N, TAIL>(a.weight, (c * TPR + t) * N, a.cols, w[c]);
#pragma unroll
        for (int i = 0; i < N; ++i) dw[c][i] = db[c][i] = 0.0f;
    }
    const float inv = 1.0f / (float)a.cols;
    for (int64_t first = (int64_t)blockIdx.x * RPB; first < a.rows; first += (int64_t)gridDim.x * RPB) {
        // rows past the end: the last row's address, no columns
        const int64_t mine = first + threadIdx.x / TPR, row = mine < a.rows ? mine : a.rows - 1;
        const int cols = mine < a.rows ? a.cols : 0;
        const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
        const T* tot = static_cast<const T*>(a.total) + row * a.ld_total;
        Span<T, TAIL> ts[CH], ys[CH], ds[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * TPR + t) * N;
            ts[c].load(tot + col, cols - col);
            ys[c].load(dy + col, cols - col);
            if (!LATE && a.dtotal) ds[c].load(static_cast<const T*>(a.dtotal) + row * a.ld_dtotal + col, cols - col);
        }
        float s[CH][N], g[CH][N];
        float sum = 0.0f, gsum = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            ts[c].floats(s[c]);
            ys[c].floats(g[c]);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                sum += s[c][i];
                gsum = fmaf(g[c][i], w[c][i], gsum);
            }
        }
        const float mean = row_sum<TPR>(sum, part) / (float)a.cols;
        gsum = row_sum<TPR>(gsum, part) * inv;             // mean of g
        float ss = 0.0f, gs = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * TPR + t) * N;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                s[c][i] = (TAIL ? col + i < cols : col < cols) ? s[c][i] - mean : 0.0f;
                ss = fmaf(s[c][i], s[c][i], ss);
                gs = fmaf(g[c][i] * w[c][i], s[c][i], gs);
            }
        }
        ss = row_sum<TPR>(ss, part);
        gs = row_sum<TPR>(gs, part);
        const float k = fitting<T>(ss, a.eps);
        if (__any(k != 1.0f)) {
            ss = gs = 0.0f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    ss = fmaf(s[c][i] * k, s[c][i] * k, ss);
                    gs = fmaf(s[c][i] * k * g[c][i], w[c][i], gs);         // g w of above would be held until here
                }
            ss = row_sum<TPR>(ss, part);
            gs = row_sum<TPR>(gs, part);
        }
        // a row past the end adds 0, with eps 0 too
        float r = cols ? root(ss, a.cols, a.eps, k) : 0.0f;
        const float gn = gs * r * inv;                     // mean of g n
        r *= k;
        T* dx = static_cast<T*>(a.dx) + row * a.ld_dx;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * TPR + t) * N;
            float d[N];
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = 0.0f;
            if (a.dtotal) {
                if (LATE) ds[c].load(static_cast<const T*>(a.dtotal) + row * a.ld_dtotal + col, cols - col);
                ds[c].floats(d);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float n = s[c][i] * r;
                dw[c][i] = fmaf(g[c][i], n, dw[c][i]);
                db[c][i] += g[c][i];
                d[i] += r * (fmaf(g[c][i], w[c][i], -gsum) - n * gn);
            }
            Span<T, TAIL>::store(dx + col, cols - col, d);
        }
    }
    float* __restrict__ out = parts + (int64_t)blockIdx.x * 2 * a.cols;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        put_part<TPR, N, RPB>(comb, dw[c], out, c * TPR * N, a.cols);
        put_part<TPR, N, RPB>(comb, db[c], out + a.cols, c * TPR * N, a.cols);
    }
}

// Sum of the n partial rows [dw, db], a column each: 64 columns by 16 slices of
// the rows in a workgroup, then the slices in ascending order.
__global__ void __launch_bounds__(1024) k_layer_join(const float* __restrict__ parts, int n, int cols,
                                                     float* __restrict__ dweight, float* __restrict__ dbias) {
    __shared__ float sum[16][GS_WAVE];
    const int l = threadIdx.x % GS_WAVE, w = threadIdx.x / GS_WAVE;
    const int col = blockIdx.x * GS_WAVE + l;
    const int per = (n + 15) / 16;
    float v = 0.0f;
    if (col < 2 * cols)
#pragma unroll 8
        for (int i = w * per; i < min(n, (w + 1) * per); ++i) v += parts[(int64_t)i * 2 * cols + col];
    sum[w][l] = v;
    __syncthreads();
    if (w == 0 && col < 2 * cols) {
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v += sum[i][l];
        if (col < cols) dweight[col] = v;
        else if (dbias) dbias[col - cols] = v;
    }
}

// Lanes of a row and their registers by the width: as few as hold it.  46,332 fp16
// rows of 390 columns take 25 us with 32 lanes of 16, 40 with 64 of 16.  (2049 to
// 4096 columns leave half of the wide kernel's pieces empty: 20,000 bf16 rows of
// 3000 with a residual take 124 us, 3.9 TB/s.)
template <typename T, bool TAIL>
hipError_t layer_go(const gs_layer_args& a, hipStream_t st) {
    constexpr int N = Piece<T>::N, NARROW = 128 / N;       // lanes that hold 128 columns
    const uint32_t by4 = div_up(a.rows, 4), narrow = div_up(a.rows, GS_BLOCK / NARROW);
    if (a.cols <= 128) k_layer_norm<T, TAIL, NARROW, N><<<narrow, GS_BLOCK, 0, st>>>(a);
    else if (a.cols <= 256) k_layer_norm<T, TAIL, NARROW, 2 * N><<<narrow, GS_BLOCK, 0, st>>>(a);
    else if (a.cols <= 512) k_layer_norm<T, TAIL, 32, 16><<<div_up(a.rows, 8), GS_BLOCK, 0, st>>>(a);
    else if (a.cols <= 1024) k_layer_norm<T, TAIL, 64, 16><<<by4, GS_BLOCK, 0, st>>>(a);
    else if (a.cols <= 1536) k_layer_norm<T, TAIL, 64, 24><<<by4, GS_BLOCK, 0, st>>>(a);
    else if (a.cols <= 2048) k_layer_norm<T, TAIL, 64, 32><<<by4, GS_BLOCK, 0, st>>>(a);
    else if (a.cols <= 8192) k_layer_norm<T, TAIL, 256, 32><<<a.rows, GS_BLOCK, 0, st>>>(a);
    else k_layer_norm<T, TAIL, 256, 64><<<a.rows, GS_BLOCK, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t layer_type(const gs_layer_args& a, hipStream_t st) {
    return a.cols % Piece<T>::N ? layer_go<T, true>(a, st) : layer_go<T, false>(a, st);
}

template <typename T, bool TAIL>
hipError_t layer_bwd_go(const gs_layer_bwd_args& a, float* parts, hipStream_t st) {
    constexpr int N = Piece<T>::N, NARROW = 128 / N;
    const int n = layer_parts(a.rows, a.cols <= 256 ? GS_BLOCK / NARROW : a.cols <= 512 ? 8 : a.cols <= 2048 ? 4 : 1);
    if (a.cols <= 128) k_layer_norm_bwd<T, TAIL, NARROW, N><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else if (a.cols <= 256) k_layer_norm_bwd<T, TAIL, NARROW, 2 * N><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else if (a.cols <= 512) k_layer_norm_bwd<T, TAIL, 32, 16><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else if (a.cols <= 1024) k_layer_norm_bwd<T, TAIL, 64, 16><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else if (a.cols <= 1536) k_layer_norm_bwd<T, TAIL, 64, 24><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else if (a.cols <= 2048) k_layer_norm_bwd<T, TAIL, 64, 32><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else if (a.cols <= 4096) k_layer_norm_bwd<T, TAIL, 256, 16><<<n, GS_BLOCK, 0, st>>>(a, parts);
    else k_layer_norm_bwd<T, TAIL, 512, 32><<<n, 512, 0, st>>>(a, parts);
    k_layer_join<<<div_up(2 * (int64_t)a.cols, GS_WAVE), 1024, 0, st>>>(parts, n, a.cols, a.dweight, a.dbias);
    return hipGetLastError();
}

template <typename T>
hipError_t layer_bwd_type(const gs_layer_bwd_args& a, float* parts, hipStream_t st) {
    return a.cols % Piece<T>::N ? layer_bwd_go<T, true>(a, parts, st) : layer_bwd_go<T, false>(a, parts, st);
}

}  // namespace

// A launch holds fewer than 2^32 threads, a row takes up to 256: more rows than
// 2^23 go in several.
hipError_t launch_layer_norm(const gs_layer_args& a, hipStream_t st) {
    constexpr int32_t kMost = 1 << 23;
    const int64_t size = a.dtype == GS_F32 ? 4 : 2;
    auto at = [](const void* p, int64_t bytes) {
        return p ? const_cast<char*>(static_cast<const char*>(p)) + bytes : nullptr;
    };
    for (int64_t first = 0; first < a.rows; first += kMost) {
        gs_layer_args b = a;
        b.rows = (int32_t)std::min<int64_t>(kMost, a.rows - first);
        b.x = at(a.x, first * a.ld_x * size);
        b.residual = at(a.residual, first * a.ld_residual * size);
        b.total = at(a.total, first * a.ld_total * size);
        b.y = at(a.y, first * a.ld_y * size);
        const hipError_t e = b.dtype == GS_F32    ? layer_type<float>(b, st)
                             : b.dtype == GS_BF16 ? layer_type<bf16_t>(b, st)
                                                  : layer_type<f16_t>(b, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// For the most partial rows that any type's kernel of this width writes.
size_t layer_norm_bwd_ws_bytes(int32_t rows, int32_t cols) {
    return align256((size_t)layer_parts(rows, cols <= 2048 ? 4 : 1) * 2 * (size_t)cols * 4);
}

hipError_t launch_layer_norm_bwd(const gs_layer_bwd_args& a, void* ws, hipStream_t st) {
    float* parts = static_cast<float*>(ws);
    if (a.rows == 0) {
        k_layer_join<<<div_up(2 * (int64_t)a.cols, GS_WAVE), 1024, 0, st>>>(parts, 0, a.cols, a.dweight, a.dbias);
        return hipGetLastError();
    }
    if (a.dtype == GS_F32) return layer_bwd_type<float>(a, parts, st);
    return a.dtype == GS_BF16 ? layer_bwd_type<bf16_t>(a, parts, st) : layer_bwd_type<f16_t>(a, parts, st);
}

}  // namespace gsmi
