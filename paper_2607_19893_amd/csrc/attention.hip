// Attention forward over ragged segments, shared key heads, windows and key
// masks: one pass over the keys with the running maximum and sum of a softmax.
//
// The rows that read one key head (every token of a segment times the heads of
// its group) are one list, row r = token r / group, head r % group, so a tile
// of keys serves all of them.  k_attention gives a workgroup 128 rows, 32 a
// wave.  Scores are formed transposed, S^T = K Q^T: a lane then holds 16 keys
// of one row, the softmax's maximum and sum stay in the lane but for its
// partner 32 lanes on, and the rounded probabilities are the operand of O^T =
// V^T P^T where they are.  Keys and values pass through LDS, values are read
// from it transposed.
#include <algorithm>

#include "attn.h"

namespace gsmi {

namespace {

constexpr int kRows = 128;                 // rows of a workgroup
constexpr int kKeys = 64;                  // keys of a step
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct FwdArgs {
    AttnArgs a;
    void* out;
    int64_t o_row, o_head;
    float* lse;
    int32_t splits;                        // parts that a segment's keys are cut into
    float* part_o;                         // [splits][n_q * heads][dim], unnormalised
    float2* part_ml;                       // [splits][n_q * heads] maximum (of the raw products) and sum
};

__device__ __forceinline__ float half_max(float v) { return fmaxf(v, __shfl_xor(v, 32, GS_WAVE)); }
__device__ __forceinline__ float half_sum(float v) { return v + __shfl_xor(v, 32, GS_WAVE); }

// Where a row's results go: its part (splits > 1) or the output.
template <typename T, int D>
__device__ __forceinline__ void store_row(const FwdArgs& f, int token, int head, int split, const acc16 (&o)[D / 32],
                                          float m, float l) {
    const int h = lane_id() >> 5;
    const int64_t row = (int64_t)token * f.a.heads + head;
    if (f.splits > 1) {
        const int64_t at = (int64_t)split * f.a.n_q * f.a.heads + row;
        if (h == 0) f.part_ml[at] = make_float2(m, l);
        float* p = f.part_o + at * f.a.dim;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int c = 32 * d + 8 * g + 4 * h;
                if (c < f.a.dim)
                    *reinterpret_cast<float4*>(p + c) =
                        make_float4(o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]);
            }
        return;
    }
    const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);    // a NaN sum stays one
    if (h == 0) f.lse[row] = l == 0.0f ? -INFINITY : m * f.a.scale + kLn2 * log2f(l);
    T* p = static_cast<T*>(f.out) + (int64_t)token * f.o_row + (int64_t)head * f.o_head;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int c = 32 * d + 8 * g + 4 * h;
            op4<T> v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = (T)(o[d][4 * g + i] * inv);
            if (c < f.a.dim) *reinterpret_cast<op4<T>*>(p + c) = v;
        }
}

// One step of the online softmax over a tile of 32 N keys: s (raw products,
// -inf where not admitted) becomes the probabilities against the new maximum.
// c = scale * log2(e).  Returns the factor of what was summed before.
template <int N>
__device__ __forceinline__ float softmax_step(acc16 (&s)[N], float c, float& m, float& l) {
    float t = s[0][0];
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) t = fmaxf(t, s[k][i]);
    t = fmaxf(m, half_max(t));
    const float base = t == -INFINITY ? 0.0f : t * c;      // nothing admitted yet: exp2(-inf) = 0 below
    const float alpha = exp2f(m * c - base);
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[k][i] = exp2f(fmaf(s[k][i], c, -base));
            sum += s[k][i];
        }
    l = l * alpha + sum;                                   // this half's keys; the halves meet at the end
    m = t;
    return alpha;
}

template <typename T, int D>
__global__ void __launch_bounds__(GS_BLOCK, 2) k_attention(FwdArgs f) {
    constexpr int P = D <= 32 ? 32 : (D <= 64 ? 64 : 128), KT = D / 16, DT = D / 32;
    constexpr int PIECES = D / 8, LOADS = kKeys * PIECES / GS_BLOCK;       // 16-byte pieces of a tile a thread
    __shared__ __attribute__((aligned(16))) T ks[kKeys * P];
    __shared__ __attribute__((aligned(16))) T vs[kKeys * P];
    __shared__ __attribute__((aligned(4))) uint8_t on[kKeys];
    const AttnArgs& a = f.a;
    const int total = a.tiles * a.kv_heads * f.splits;
    int id = chiplet_order(blockIdx.x, total);
    if (id >= total) return;
    const int split = id % f.splits;
    id /= f.splits;
    const int kvh = id / a.tiles;
    const Segment sg = find_segment(a, a.cu_q, a.n_q, a.group, kRows, id - kvh * a.tiles);
    const int rows = sg.nq * a.group, row0 = sg.tile * kRows;
    if (row0 >= rows) return;
    const int lane = lane_id(), h = lane >> 5, wave = threadIdx.x / GS_WAVE;
    const int r = row0 + 32 * wave + (lane & 31);
    const bool there = r < rows;
    const int i = (there ? r : rows - 1) / a.group;
    const int token = sg.q0 + i, head = kvh * a.group + (there ? r : rows - 1) - i * a.group;
    const int shift = sg.nk - sg.nq;

    op8<T> q[KT];
    {
        const T* p = static_cast<const T*>(a.q) + (int64_t)token * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            const int c = 16 * t + 8 * h;
            if (c < a.dim) q[t] = *reinterpret_cast<const op8<T>*>(p + c);
            else q[t] = op8<T>{};
        }
    }
    // keys that this lane's row admits, and those that any row of the tile does
    int klo, khi, lo, hi;
    admitted(a, sg.nk, i + shift, i + shift, klo, khi);
    const int last = min(row0 + kRows, rows) - 1;
    admitted(a, sg.nk, row0 / a.group + shift, last / a.group + shift, lo, hi);
    // and those that all do: no test of the window between them
    int alo, ahi;
    admitted(a, sg.nk, last / a.group + shift, row0 / a.group + shift, alo, ahi);
    int j0 = lo / kKeys * kKeys, j1 = hi;
    if (f.splits > 1) {
        const int per = ((max(hi - j0, 0) + f.splits - 1) / f.splits + kKeys - 1) / kKeys * kKeys;
        j0 += split * per;
        j1 = min(hi, j0 + per);
    }

    const float c = a.scale * kLog2e;
    float m = -INFINITY, l = 0.0f;
    acc16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = acc16{};

    for (int j = j0; j < j1; j += kKeys) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int x = threadIdx.x + u * GS_BLOCK, row = x / PIECES, piece = x % PIECES;
            const int key = j + row;
            op8<T> kp{}, vp{};
            if (key < sg.nk && 8 * piece < a.dim && (a.key_on == nullptr || a.key_on[sg.k0 + key])) {
                kp = *reinterpret_cast<const op8<T>*>(static_cast<const T*>(a.k) + (int64_t)(sg.k0 + key) * a.k_row +
                                                      (int64_t)kvh * a.k_head + 8 * piece);
                vp = *reinterpret_cast<const op8<T>*>(static_cast<const T*>(a.v) + (int64_t)(sg.k0 + key) * a.v_row +
                                                      (int64_t)kvh * a.v_head + 8 * piece);
            }
            *reinterpret_cast<op8<T>*>(ks + piece_at<P>(row, piece)) = kp;
            *reinterpret_cast<op8<T>*>(vs + piece_at<P>(row, piece)) = vp;
        }
        if (threadIdx.x < kKeys) {
            const int key = j + threadIdx.x;
            on[threadIdx.x] = key < sg.nk && (a.key_on == nullptr || a.key_on[sg.k0 + key]);
        }
        __syncthreads();
        acc16 s[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            s[k] = acc16{};
#pragma unroll
            for (int t = 0; t < KT; ++t) s[k] = mfma(rows_operand<T, P>(ks, 32 * k, t), q[t], s[k]);
        }
        if (a.key_on != nullptr || j < alo || j + kKeys > ahi) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int at = 32 * k + 8 * g + 4 * h;
                    const uint32_t w = *reinterpret_cast<const uint32_t*>(on + at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = j + at + e;
                        if (key < klo || key >= khi || ((w >> (8 * e)) & 255u) == 0) s[k][4 * g + e] = -INFINITY;
                    }
                }
        }
        const float alpha = softmax_step<2>(s, c, m, l);
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= alpha;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const op8<T> p = tile_operand<T>(s[k], u);
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    o[d] = mfma(columns_operand<T, P>(vs, 32 * k + 16 * u, 32 * d), p, o[d]);
            }
    }
    l = half_sum(l);
    if (there) store_row<T, D>(f, token, head, split, o, m, l);
}

// Joins the parts of a row: 8 lanes... one wave a row, lanes over the elements.
template <typename T>
__global__ void __launch_bounds__(GS_BLOCK) k_attention_join(FwdArgs f) {
    const int64_t rows = (int64_t)f.a.n_q * f.a.heads;
    const int64_t row = (int64_t)blockIdx.x * (GS_BLOCK / GS_WAVE) + threadIdx.x / GS_WAVE;
    if (row >= rows) return;
    const int lane = lane_id();
    float m = -INFINITY;
    for (int s = 0; s < f.splits; ++s) m = fmaxf(m, f.part_ml[s * rows + row].x);
    const float c = f.a.scale * kLog2e, base = m == -INFINITY ? 0.0f : m * c;
    float l = 0.0f, o0 = 0.0f, o1 = 0.0f;
    for (int s = 0; s < f.splits; ++s) {
        const float2 ml = f.part_ml[s * rows + row];
        const float w = exp2f(ml.x * c - base);
        const float* p = f.part_o + (s * rows + row) * f.a.dim;
        l += ml.y * w;
        if (2 * lane < f.a.dim) {
            const float2 v = *reinterpret_cast<const float2*>(p + 2 * lane);
            o0 += v.x * w;
            o1 += v.y * w;
        }
    }
    const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);
    const int64_t token = row / f.a.heads;
    const int head = (int)(row - token * f.a.heads);
    if (lane == 0) f.lse[row] = l == 0.0f ? -INFINITY : m * f.a.scale + kLn2 * log2f(l);
    if (2 * lane < f.a.dim) {
        T* p = static_cast<T*>(f.out) + token * f.o_row + (int64_t)head * f.o_head + 2 * lane;
        p[0] = (T)(o0 * inv);
        p[1] = (T)(o1 * inv);
    }
}

// How a call is cut: from its sizes alone.
struct Plan {
    int32_t tiles, splits;
};

Plan plan(const gs_attn& a) {
    Plan p;
    const int group = a.heads / a.kv_heads;
    p.tiles = attn_tiles((int64_t)a.n_q * group, kRows, a.n_seg);
    p.splits = 1;
    return p;
}

template <typename T, int D>
hipError_t go(const FwdArgs& f, hipStream_t st) {
    const uint32_t grid = chiplet_grid((int64_t)f.a.tiles * f.a.kv_heads * f.splits);
    k_attention<T, D><<<grid, GS_BLOCK, 0, st>>>(f);
    if (f.splits > 1) k_attention_join<T><<<div_up((uint64_t)f.a.n_q * f.a.heads, 4), GS_BLOCK, 0, st>>>(f);
    return hipGetLastError();
}

template <typename T>
hipError_t by_dim(const FwdArgs& f, hipStream_t st) {
    if (f.a.dim <= 32) return go<T, 32>(f, st);
    if (f.a.dim <= 64) return go<T, 64>(f, st);
    if (f.a.dim <= 96) return go<T, 96>(f, st);
    return go<T, 128>(f, st);
}

}  // namespace

size_t attention_ws_bytes(const gs_attn& a) {
    const Plan p = plan(a);
    if (p.splits == 1) return 0;
    const size_t rows = (size_t)a.n_q * a.heads * p.splits;
    return align256(rows * sizeof(float2)) + align256(rows * a.dim * sizeof(float));
}

hipError_t launch_attention(const gs_attn& a, const gs_rows& out, float* lse, void* ws, hipStream_t st) {
    const Plan p = plan(a);
    FwdArgs f;
    f.a = attn_args(a);
    f.a.tiles = p.tiles;
    f.out = out.ptr;
    f.o_row = out.ld_row;
    f.o_head = out.ld_head;
    f.lse = lse;
    f.splits = p.splits;
    f.part_ml = static_cast<float2*>(ws);
    f.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + align256((size_t)a.n_q * a.heads * p.splits * sizeof(float2)));
    return a.dtype == GS_BF16 ? by_dim<bf16_t>(f, st) : by_dim<f16_t>(f, st);
}

}  // namespace gsmi
