// Attention's gradient over ragged segments: the probabilities are recomputed
// from the forward's log sums, and nothing is added by atomics, so that the same
// call gives the same bits.  Two kernels, each with its sums in registers:
//   k_attention_dq   a workgroup owns 128 rows and walks the keys: delta = dout .
//                    out, dq = scale * sum ds k.  3 products a pair.
//   k_attention_dkv  a workgroup owns 128 keys and walks the rows of every head
//                    that reads them: dv = sum p dout, dk = scale * sum ds q.
//                    4 products a pair.
// (One kernel with 5 products would have to add dq, or dk and dv, across
// workgroups.)  Scores are formed in the orientation whose C tile is the next
// product's operand: S^T for dq, S for dk and dv.
#include <algorithm>

#include "attn.h"

namespace gsmi {

namespace {

constexpr int kRows = 128;                 // rows (dq) or keys (dk, dv) of a workgroup
constexpr int kStep = 64;                  // keys or rows of a step
constexpr float kLog2e = 1.44269504088896340736f;

struct BwdArgs {
    AttnArgs a;
    const void *out, *dout;
    void *dq, *dk, *dv;
    int64_t o_row, o_head, do_row, do_head, dq_row, dq_head, dk_row, dk_head, dv_row, dv_head;
    const float* lse;
    float* delta;                          // [n_q * heads]
    int32_t key_tiles;
    int32_t splits;                        // parts that a key tile's rows are cut into
    float* part;                           // [splits][2][n_k * kv_heads][dim]: dk, dv
};

// exp2 base of a row: its log sum in powers of two; +inf (every probability 0)
// for a row that admits nothing.
__device__ __forceinline__ float row_base(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

// A C tile whose columns are token rows' elements 32 d .. +31 of one row a lane.
template <typename T, int DT>
__device__ __forceinline__ void store_tiles(T* p, const acc16 (&o)[DT], float scale, int dim) {
    const int h = lane_id() >> 5;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int c = 32 * d + 8 * g + 4 * h;
            op4<T> v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = (T)(o[d][4 * g + i] * scale);
            if (c < dim) *reinterpret_cast<op4<T>*>(p + c) = v;
        }
}

template <typename T, int D>
__global__ void __launch_bounds__(GS_BLOCK, 2) k_attention_dq(BwdArgs f) {
    constexpr int P = D <= 32 ? 32 : (D <= 64 ? 64 : 128), KT = D / 16, DT = D / 32;
    constexpr int PIECES = D / 8, LOADS = kStep * PIECES / GS_BLOCK;
    __shared__ __attribute__((aligned(16))) T ks[kStep * P];
    __shared__ __attribute__((aligned(16))) T vs[kStep * P];
    __shared__ __attribute__((aligned(4))) uint8_t on[kStep];
    const AttnArgs& a = f.a;
    const Place place = chiplet_place(blockIdx.x, a.tiles, a.kv_heads, 1);
    const int kvh = place.head;
    // the last tiles first: with ordered keys they have the most to do
    const Segment sg = find_segment(a, a.cu_q, a.n_q, a.group, kRows, a.tiles - 1 - place.tile);
    const int rows = sg.nq * a.group, row0 = sg.tile * kRows;
    if (row0 >= rows) return;
    const int lane = lane_id(), h = lane >> 5, wave = threadIdx.x / GS_WAVE;
    const int r = row0 + 32 * wave + (lane & 31);
    const bool there = r < rows;
    const int i = (there ? r : rows - 1) / a.group;
    const int token = sg.q0 + i, head = kvh * a.group + (there ? r : rows - 1) - i * a.group;
    const int shift = sg.nk - sg.nq;
    const int64_t row = (int64_t)token * a.heads + head;
    const float lse = f.lse[row];
    const float base = row_base(lse);

    op8<T> q[KT], dy[KT];
    float delta = 0.0f;
    {
        const T* p = static_cast<const T*>(a.q) + (int64_t)token * a.q_row + (int64_t)head * a.q_head;
        const T* po = static_cast<const T*>(f.out) + (int64_t)token * f.o_row + (int64_t)head * f.o_head;
        const T* pd = static_cast<const T*>(f.dout) + (int64_t)token * f.do_row + (int64_t)head * f.do_head;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            const int c = 16 * t + 8 * h;
            q[t] = dy[t] = op8<T>{};
            if (c < a.dim && lse != -INFINITY) {
                q[t] = *reinterpret_cast<const op8<T>*>(p + c);
                dy[t] = *reinterpret_cast<const op8<T>*>(pd + c);
                const op8<T> y = *reinterpret_cast<const op8<T>*>(po + c);
#pragma unroll
                for (int e = 0; e < 8; ++e) delta = fmaf((float)dy[t][e], (float)y[e], delta);
            }
        }
    }
    delta += __shfl_xor(delta, 32, GS_WAVE);
    if (there && h == 0) f.delta[row] = delta;

    int klo, khi, lo, hi, alo, ahi;
    admitted(a, sg.nk, i + shift, i + shift, klo, khi);
    const int last = min(row0 + kRows, rows) - 1;
    admitted(a, sg.nk, row0 / a.group + shift, last / a.group + shift, lo, hi);
    admitted(a, sg.nk, last / a.group + shift, row0 / a.group + shift, alo, ahi);

    const float c = a.scale * kLog2e;
    Lanes at;
    at.init<P>();
    acc16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = acc16{};
    for (int j = lo / kStep * kStep; j < hi; j += kStep) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int x = threadIdx.x + u * GS_BLOCK, kr = x / PIECES, piece = x % PIECES;
            const int key = j + kr;
            op8<T> kp{}, vp{};
            if (key < sg.nk && 8 * piece < a.dim && (a.key_on == nullptr || a.key_on[sg.k0 + key])) {
                kp = *reinterpret_cast<const op8<T>*>(static_cast<const T*>(a.k) + (int64_t)(sg.k0 + key) * a.k_row +
                                                      (int64_t)kvh * a.k_head + 8 * piece);
                vp = *reinterpret_cast<const op8<T>*>(static_cast<const T*>(a.v) + (int64_t)(sg.k0 + key) * a.v_row +
                                                      (int64_t)kvh * a.v_head + 8 * piece);
            }
            *reinterpret_cast<op8<T>*>(ks + piece_at<P>(kr, piece)) = kp;
            *reinterpret_cast<op8<T>*>(vs + piece_at<P>(kr, piece)) = vp;
        }
        if (threadIdx.x < kStep) {
            const int key = j + threadIdx.x;
            on[threadIdx.x] = key < sg.nk && (a.key_on == nullptr || a.key_on[sg.k0 + key]);
        }
        __syncthreads();
        const bool test = a.key_on != nullptr || j < alo || j + kStep > ahi;
#pragma unroll
        for (int k = 0; k < kStep / 32; ++k) {
            acc16 s{}, dp{};
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                s = mfma(rows_operand<T, P>(ks, at, 32 * k, t), q[t], s);
                dp = mfma(rows_operand<T, P>(vs, at, 32 * k, t), dy[t], dp);
            }
            if (test) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int first = 32 * k + 8 * g + 4 * h;
                    const uint32_t w = *reinterpret_cast<const uint32_t*>(on + first);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = j + first + e;
                        if (key < klo || key >= khi || ((w >> (8 * e)) & 255u) == 0) s[4 * g + e] = -INFINITY;
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c, -base)) * (dp[e] - delta);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const op8<T> ds = tile_operand<T>(s, u);
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] = mfma(columns_operand<T, P>(ks, at, 32 * k + 16 * u, d), ds, o[d]);
            }
        }
    }
    if (there)
        store_tiles<T, DT>(static_cast<T*>(f.dq) + (int64_t)token * f.dq_row + (int64_t)head * f.dq_head, o, a.scale,
                           a.dim);
}

template <typename T, int D>
__global__ void __launch_bounds__(GS_BLOCK, D > 64 ? 1 : 2) k_attention_dkv(BwdArgs f) {
    constexpr int P = D <= 32 ? 32 : (D <= 64 ? 64 : 128), KT = D / 16, DT = D / 32;
    constexpr int PIECES = D / 8, LOADS = kStep * PIECES / GS_BLOCK;
    __shared__ __attribute__((aligned(16))) T qs[kStep * P];
    __shared__ __attribute__((aligned(16))) T ds[kStep * P];
    __shared__ __attribute__((aligned(16))) float bases[kStep], deltas[kStep];
    __shared__ __attribute__((aligned(16))) int klos[kStep], khis[kStep];
    const AttnArgs& a = f.a;
    const Place place = chiplet_place(blockIdx.x, f.key_tiles, a.kv_heads, f.splits);
    const int split = place.split, kvh = place.head;
    const Segment sg = find_segment(a, a.cu_k, a.n_k, 1, kRows, place.tile);
    const int key0 = sg.tile * kRows;
    if (key0 >= sg.nk) return;
    const int lane = lane_id(), h = lane >> 5, wave = threadIdx.x / GS_WAVE;
    const int mine = key0 + 32 * wave + (lane & 31);
    const bool there = mine < sg.nk;
    const bool on = there && (a.key_on == nullptr || a.key_on[sg.k0 + mine]);
    const int key = on ? mine : -1;                        // below every row's first key
    const int shift = sg.nk - sg.nq, rows = sg.nq * a.group;

    op8<T> kf[KT], vf[KT];
    {
        const int64_t at = sg.k0 + (there ? mine : key0);
        const T* pk = static_cast<const T*>(a.k) + at * a.k_row + (int64_t)kvh * a.k_head;
        const T* pv = static_cast<const T*>(a.v) + at * a.v_row + (int64_t)kvh * a.v_head;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            const int c = 16 * t + 8 * h;
            kf[t] = vf[t] = op8<T>{};
            if (c < a.dim && on) {
                kf[t] = *reinterpret_cast<const op8<T>*>(pk + c);
                vf[t] = *reinterpret_cast<const op8<T>*>(pv + c);
            }
        }
    }
    // rows that admit any of the workgroup's keys: place in [first key - right, last key + left]
    const int last = min(key0 + kRows, sg.nk) - 1;
    const int64_t i0 = a.right >= 0 ? max((int64_t)0, (int64_t)key0 - a.right - shift) : 0;
    const int64_t i1 = a.left >= 0 ? min((int64_t)sg.nq, (int64_t)last + a.left - shift + 1) : sg.nq;
    int r0 = (int)min((int64_t)rows, i0 * a.group) / kStep * kStep;
    int r1 = (int)max((int64_t)0, i1 * a.group);
    if (f.splits > 1) {
        const int per = ((max(r1 - r0, 0) + f.splits - 1) / f.splits + kStep - 1) / kStep * kStep;
        const int end = r1;
        r0 += split * per;
        r1 = min(end, r0 + per);
    }
    const float c = a.scale * kLog2e;
    Lanes at;
    at.init<P>();
    acc16 dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) dk[d] = dv[d] = acc16{};
    for (int r = r0; r < r1; r += kStep) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int x = threadIdx.x + u * GS_BLOCK, rr = x / PIECES, piece = x % PIECES;
            op8<T> qp{}, dp{};
            if (r + rr < rows && 8 * piece < a.dim) {
                const int i = (r + rr) / a.group, head = kvh * a.group + (r + rr) - i * a.group;
                const int64_t token = sg.q0 + i;
                if (f.lse[token * a.heads + head] != -INFINITY) {
                    qp = *reinterpret_cast<const op8<T>*>(static_cast<const T*>(a.q) + token * a.q_row +
                                                          (int64_t)head * a.q_head + 8 * piece);
                    dp = *reinterpret_cast<const op8<T>*>(static_cast<const T*>(f.dout) + token * f.do_row +
                                                          (int64_t)head * f.do_head + 8 * piece);
                }
            }
            *reinterpret_cast<op8<T>*>(qs + piece_at<P>(rr, piece)) = qp;
            *reinterpret_cast<op8<T>*>(ds + piece_at<P>(rr, piece)) = dp;
        }
        if (threadIdx.x < kStep) {
            const int rr = r + threadIdx.x;
            float base = INFINITY, delta = 0.0f;
            int lo = 0, hi = 0;
            if (rr < rows) {
                const int i = rr / a.group, head = kvh * a.group + rr - i * a.group;
                const int64_t at = (int64_t)(sg.q0 + i) * a.heads + head;
                base = row_base(f.lse[at]);
                delta = f.delta[at];
                admitted(a, sg.nk, i + shift, i + shift, lo, hi);
            }
            bases[threadIdx.x] = base;
            deltas[threadIdx.x] = delta;
            klos[threadIdx.x] = lo;
            khis[threadIdx.x] = hi;
        }
        __syncthreads();
        // the step's rows all admit all of the workgroup's keys: no test
        int alo, ahi;
        admitted(a, sg.nk, (min(r + kStep, rows) - 1) / a.group + shift, r / a.group + shift, alo, ahi);
        const bool test = a.key_on != nullptr || key0 + kRows > sg.nk || key0 < alo || last >= ahi || r + kStep > rows;
#pragma unroll
        for (int k = 0; k < kStep / 32; ++k) {
            acc16 s{}, dp{};
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                s = mfma(rows_operand<T, P>(qs, at, 32 * k, t), kf[t], s);
                dp = mfma(rows_operand<T, P>(ds, at, 32 * k, t), vf[t], dp);
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int first = 32 * k + 8 * g + 4 * h;
                const float4 b = *reinterpret_cast<const float4*>(bases + first);
                const float4 dl = *reinterpret_cast<const float4*>(deltas + first);
                s[4 * g] = __builtin_amdgcn_exp2f(fmaf(s[4 * g], c, -b.x));
                s[4 * g + 1] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + 1], c, -b.y));
                s[4 * g + 2] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + 2], c, -b.z));
                s[4 * g + 3] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + 3], c, -b.w));
                if (test) {
                    const int4 lo = *reinterpret_cast<const int4*>(klos + first);
                    const int4 hi = *reinterpret_cast<const int4*>(khis + first);
                    if (key < lo.x || key >= hi.x) s[4 * g] = 0.0f;
                    if (key < lo.y || key >= hi.y) s[4 * g + 1] = 0.0f;
                    if (key < lo.z || key >= hi.z) s[4 * g + 2] = 0.0f;
                    if (key < lo.w || key >= hi.w) s[4 * g + 3] = 0.0f;
                }
                dp[4 * g] = s[4 * g] * (dp[4 * g] - dl.x);
                dp[4 * g + 1] = s[4 * g + 1] * (dp[4 * g + 1] - dl.y);
                dp[4 * g + 2] = s[4 * g + 2] * (dp[4 * g + 2] - dl.z);
                dp[4 * g + 3] = s[4 * g + 3] * (dp[4 * g + 3] - dl.w);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const op8<T> p = tile_operand<T>(s, u), z = tile_operand<T>(dp, u);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    dv[d] = mfma(columns_operand<T, P>(ds, at, 32 * k + 16 * u, d), p, dv[d]);
                    dk[d] = mfma(columns_operand<T, P>(qs, at, 32 * k + 16 * u, d), z, dk[d]);
                }
            }
        }
    }
    if (!there) return;
    const int64_t token = sg.k0 + mine;
    if (f.splits > 1) {
        const int64_t n = (int64_t)a.n_k * a.kv_heads;
        float* pk = f.part + ((int64_t)split * 2 * n + token * a.kv_heads + kvh) * a.dim;
        store_tiles<float, DT>(pk, dk, a.scale, a.dim);
        store_tiles<float, DT>(pk + n * a.dim, dv, 1.0f, a.dim);
        return;
    }
    store_tiles<T, DT>(static_cast<T*>(f.dk) + token * f.dk_row + (int64_t)kvh * f.dk_head, dk, a.scale, a.dim);
    store_tiles<T, DT>(static_cast<T*>(f.dv) + token * f.dv_row + (int64_t)kvh * f.dv_head, dv, 1.0f, a.dim);
}

// Sums the parts of dk and dv in ascending order, four elements a thread.
template <typename T>
__global__ void __launch_bounds__(GS_BLOCK) k_attention_dkv_join(BwdArgs f) {
    const AttnArgs& a = f.a;
    const int per = a.dim / 4;
    const int64_t n = (int64_t)a.n_k * a.kv_heads;
    const int64_t x = (int64_t)blockIdx.x * GS_BLOCK + threadIdx.x;
    if (x >= 2 * n * per) return;
    const int which = x >= n * per;
    const int64_t row = (x - which * n * per) / per;
    const int c = (int)(x - which * n * per - row * per) * 4;
    const int64_t token = row / a.kv_heads;
    const int head = (int)(row - token * a.kv_heads);
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s = 0; s < f.splits; ++s) {
        const float4 w = *reinterpret_cast<const float4*>(f.part + ((int64_t)(2 * s + which) * n + row) * a.dim + c);
        v.x += w.x;
        v.y += w.y;
        v.z += w.z;
        v.w += w.w;
    }
    T* p = which ? static_cast<T*>(f.dv) + token * f.dv_row + (int64_t)head * f.dv_head
                 : static_cast<T*>(f.dk) + token * f.dk_row + (int64_t)head * f.dk_head;
    op4<T> o;
    o[0] = (T)v.x;
    o[1] = (T)v.y;
    o[2] = (T)v.z;
    o[3] = (T)v.w;
    *reinterpret_cast<op4<T>*>(p + c) = o;
}

int dkv_splits(const gs_attn& a) { return 1; }

template <typename T, int D>
hipError_t go(const BwdArgs& f, hipStream_t st) {
    if (f.a.n_q > 0)
        k_attention_dq<T, D><<<(uint32_t)(f.a.tiles * f.a.kv_heads), GS_BLOCK, 0, st>>>(f);
    if (f.a.n_k > 0) {
        k_attention_dkv<T, D><<<(uint32_t)(f.key_tiles * f.a.kv_heads * f.splits), GS_BLOCK, 0, st>>>(f);
        if (f.splits > 1)
            k_attention_dkv_join<T>
                <<<div_up((uint64_t)f.a.n_k * f.a.kv_heads * f.a.dim / 2, GS_BLOCK), GS_BLOCK, 0, st>>>(f);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t by_dim(const BwdArgs& f, hipStream_t st) {
    if (f.a.dim <= 32) return go<T, 32>(f, st);
    if (f.a.dim <= 64) return go<T, 64>(f, st);
    if (f.a.dim <= 96) return go<T, 96>(f, st);
    return go<T, 128>(f, st);
}

}  // namespace

size_t attention_bwd_ws_bytes(const gs_attn& a) {
    const int splits = dkv_splits(a);
    const size_t parts = splits > 1 ? (size_t)splits * 2 * a.n_k * a.kv_heads * a.dim * sizeof(float) : 0;
    return align256((size_t)a.n_q * a.heads * sizeof(float)) + align256(parts);
}

hipError_t launch_attention_bwd(const gs_attn& a, const gs_attn_grads& g, void* ws, hipStream_t st) {
    BwdArgs f;
    f.a = attn_args(a);
    f.a.tiles = whole_shares(attn_tiles((int64_t)a.n_q * f.a.group, kRows, a.n_seg), a.kv_heads);
    f.key_tiles = whole_shares(attn_tiles(a.n_k, kRows, a.n_seg), a.kv_heads);
    f.out = g.out.ptr;
    f.o_row = g.out.ld_row;
    f.o_head = g.out.ld_head;
    f.dout = g.dout.ptr;
    f.do_row = g.dout.ld_row;
    f.do_head = g.dout.ld_head;
    f.dq = g.dq.ptr;
    f.dq_row = g.dq.ld_row;
    f.dq_head = g.dq.ld_head;
    f.dk = g.dk.ptr;
    f.dk_row = g.dk.ld_row;
    f.dk_head = g.dk.ld_head;
    f.dv = g.dv.ptr;
    f.dv_row = g.dv.ld_row;
    f.dv_head = g.dv.ld_head;
    f.lse = g.lse;
    f.delta = static_cast<float*>(ws);
    f.splits = dkv_splits(a);
    f.part = reinterpret_cast<float*>(static_cast<char*>(ws) + align256((size_t)a.n_q * a.heads * sizeof(float)));
    return a.dtype == GS_BF16 ? by_dim<bf16_t>(f, st) : by_dim<f16_t>(f, st);
}

}  // namespace gsmi
