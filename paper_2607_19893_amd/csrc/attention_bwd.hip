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
    float* base;                           // [heads][n_q]: the rows' log sums in powers of two
    float* delta;                          // [heads][n_q], behind base: -delta, where dout . v starts from
    int32_t key_tiles;
    int32_t splits;                        // most parts that a key tile's rows are cut into
    int32_t chunk;                         // steps of a part (about)
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

// 64 keys a step.  8192 ordered tokens, 16/4 heads of 128: 413 us, 1.0 PFLOP/s of
// its products under the power limit.  24 regions of 3..1500 tokens, 8 heads of
// 64, a tenth of the keys off: 49 us in a kernel trace, whose two kernels together
// take 112 where the untraced call takes 101; vector units busy 47% of the cycles,
// matrix units 34%, waves waiting for data 42% of their time.
// KEYS: keys may be off.  A step's keys then start their scores at 0 or -inf,
// read from LDS into the tile that the products are added to.
template <typename T, int D, bool KEYS>
__global__ void __launch_bounds__(GS_BLOCK, 2) k_attention_dq(BwdArgs f) {
    constexpr int P = D <= 32 ? 32 : (D <= 64 ? 64 : 128), KT = D / 16, DT = D / 32;
    // two buffers: a step's tiles arrive while the step before computes
    __shared__ __attribute__((aligned(16))) T ks0[kStep * P], vs0[kStep * P];
    __shared__ __attribute__((aligned(16))) T ks1[kStep * P], vs1[kStep * P];
    __shared__ __attribute__((aligned(16))) float on0[KEYS ? kStep : 4], on1[KEYS ? kStep : 4];
    const AttnArgs& a = f.a;
    const Place place = chiplet_place<true>(blockIdx.x, a.tiles, a.kv_heads, 1);
    const int kvh = place.head;
    const Segment sg = find_segment<false, true>(a, kRows, a.tiles, place.tile);
    if (a.fill) fill_rest(a, a.cu_q, a.n_q, a.heads, static_cast<T*>(f.dq), f.dq_row, f.dq_head, nullptr);
    const int rows = sg.nq * a.group, row0 = sg.tile * kRows;
    if (row0 >= rows) return;
    const int lane = lane_id(), h = lane >> 5, wave = threadIdx.x / GS_WAVE;
    const int r = row0 + 32 * wave + (lane & 31);
    const bool there = r < rows;
    const int i = (there ? r : rows - 1) / a.group;
    const int token = sg.q0 + i, head = kvh * a.group + (there ? r : rows - 1) - i * a.group;
    const int shift = sg.nk - sg.nq;
    const float lse = f.lse[(int64_t)token * a.heads + head];
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
    const float2 both = halves(delta);
    delta = both.x + both.y;
    if (there && h == 0) {
        f.base[(int64_t)head * a.n_q + token] = base;
        f.delta[(int64_t)head * a.n_q + token] = -delta;
    }

    acc16 minus_delta;
#pragma unroll
    for (int e = 0; e < 16; ++e) minus_delta[e] = -delta;

    int klo, khi, lo, hi, alo, ahi;
    admitted(a, sg.nk, i + shift, i + shift, klo, khi);
    const int last = min(row0 + kRows, rows) - 1;
    admitted(a, sg.nk, row0 / a.group + shift, last / a.group + shift, lo, hi);
    admitted(a, sg.nk, last / a.group + shift, row0 / a.group + shift, alo, ahi);

    TileLoader<T, P, kStep> kl, vl;
    kl.init(static_cast<const T*>(a.k) + sg.k0 * a.k_row + kvh * a.k_head, sg.nk, a.k_row, a.dim);
    vl.init(static_cast<const T*>(a.v) + sg.k0 * a.v_row + kvh * a.v_head, sg.nk, a.v_row, a.dim);
    // the keys' flags, loaded a step before the tiles that they belong to
    const uint8_t* const flags = a.key_on + sg.k0;
    uint8_t flag = 0;
    auto fetch = [&](T* ks, T* vs, float* on, int j) {
        uint32_t skip = 0;
        if (KEYS) {
            skip = rows_off<P, kStep>(__ballot(flag));
            if (threadIdx.x < kStep) on[threadIdx.x] = flag ? 0.0f : -INFINITY;
            flag = key_flag(flags, j + kStep + fresh(lane), sg.nk);
        }
        kl.load(ks, j, skip);
        vl.load(vs, j, skip);
    };

    const float c = a.scale * kLog2e;
    Lanes at;
    at.init<P>();
    acc16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = acc16{};
    auto step = [&](const T* ks, const T* vs, const float* on, int j) {
        at.refresh();
        // the window's edge, where rows differ; the segment's end has its flags
        const bool test = j < alo || (KEYS ? min(j + kStep, sg.nk) : j + kStep) > ahi;
        uint64_t seen = ~0ull;
        if (test) seen = bits_between(klo - j, khi - j);
#pragma unroll
        for (int k = 0; k < kStep / 32; ++k) {
            // operands are read one product ahead of their use; the barriers keep
            // the compiler from reading more of them ahead, which would not fit
            // the registers of two waves a SIMD
            acc16 s{}, dp = minus_delta;
            if (KEYS) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 v = *reinterpret_cast<const float4*>(on + 32 * k + 8 * g + 4 * h);
                    s[4 * g] = v.x;
                    s[4 * g + 1] = v.y;
                    s[4 * g + 2] = v.z;
                    s[4 * g + 3] = v.w;
                }
            }
            op8<T> x[2], y[2];
            x[0] = rows_operand<T, P>(ks, at, 32 * k, 0);
            y[0] = rows_operand<T, P>(vs, at, 32 * k, 0);
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                if (t + 1 < KT) {
                    x[(t + 1) & 1] = rows_operand<T, P>(ks, at, 32 * k, t + 1);
                    y[(t + 1) & 1] = rows_operand<T, P>(vs, at, 32 * k, t + 1);
                }
                s = mfma(x[t & 1], q[t], s);
                dp = mfma(y[t & 1], dy[t], dp);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (test) keep_some(s, (uint32_t)(seen >> (32 * k)));
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c, -base)) * dp[e];
            op8<T> z[2], ds;
            z[0] = columns_operand<T, P>(ks, at, 32 * k, 0);
#pragma unroll
            for (int e = 0; e < 2 * DT; ++e) {
                if (e + 1 < 2 * DT)
                    z[(e + 1) & 1] = columns_operand<T, P>(ks, at, 32 * k + 16 * ((e + 1) / DT), (e + 1) % DT);
                if (e % DT == 0) ds = tile_operand<T>(s, e / DT);
                o[e % DT] = mfma(z[e & 1], ds, o[e % DT]);
                if (e & 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    const int j0 = lo / kStep * kStep;
    if (j0 < hi) {
        if (KEYS) flag = key_flag(flags, j0 + lane, sg.nk);
        fetch(ks0, vs0, on0, j0);
    }
    __syncthreads();                               // the fetched tiles are in LDS
    for (int j = j0; j < hi; j += 2 * kStep) {
        if (j + kStep < hi) fetch(ks1, vs1, on1, j + kStep);
        step(ks0, vs0, on0, j);
        __syncthreads();
        if (j + kStep < hi) {
            if (j + 2 * kStep < hi) fetch(ks0, vs0, on0, j + 2 * kStep);
            step(ks1, vs1, on1, j + kStep);
        }
        __syncthreads();
    }
    if (there)
        store_tiles<T, DT>(static_cast<T*>(f.dq) + (int64_t)token * f.dq_row + (int64_t)head * f.dq_head, o, a.scale,
                           a.dim);
}

// The steps of a key tile, ST tokens each, all heads of the group one after the
// other: t0 and `per` steps a head, `parts` equal runs of them.
template <int ST>
struct TileRows {
    int lo, hi;                            // tokens that admit any of the tile's keys
    int t0, per, steps, parts;

    __device__ __forceinline__ TileRows(const BwdArgs& f, const Segment& sg, int key0) {
        const int last = min(key0 + kRows, sg.nk) - 1;
        admitting(f.a, sg.nq, sg.nk - sg.nq, key0, last, lo, hi);
        t0 = lo / ST * ST;
        per = max(hi - t0 + ST - 1, 0) / ST;
        steps = per * f.a.group;
        parts = max(1, min(f.splits, (steps + f.chunk - 1) / f.chunk));
    }
};

// Steps of dk's and dv's kernel: 64 tokens, 32 for heads of more than 64 elements.
constexpr int dkv_step(int dim) { return dim > 64 ? 32 : 64; }

// The sums of dk and dv take a lane's registers twice the head's size; keys and
// values beside them leave no room for two waves a SIMD from 96 elements on, so
// there the values are read from LDS (a quarter more of its traffic) and a step
// is 32 rows; at 64 elements that form took 3 us more of 107.  8192 ordered
// tokens, 16/4 heads of 128: 0.85 PFLOP/s of its products (644 us), matrix units
// busy 56% of the cycles: two reads of LDS a matrix instruction where dq has
// 1.3.  24 regions of 3..1500 tokens, 8 heads of 64: 63 us of the same trace.
template <typename T, int D>
__global__ void __launch_bounds__(GS_BLOCK, 2) k_attention_dkv(BwdArgs f) {
    constexpr int P = D <= 32 ? 32 : (D <= 64 ? 64 : 128), KT = D / 16, DT = D / 32;
    constexpr bool BIG = D > 64;
    constexpr int ST = dkv_step(D), NK = ST / 32;
    __shared__ __attribute__((aligned(16))) T qs0[ST * P], ds0[ST * P];
    __shared__ __attribute__((aligned(16))) T qs1[ST * P], ds1[ST * P];
    __shared__ __attribute__((aligned(16))) float st0[2 * 64], st1[2 * 64];            // bases, then -deltas
    __shared__ __attribute__((aligned(16))) T vs[BIG ? kRows * P : 8];
    const AttnArgs& a = f.a;
    const Place place = chiplet_place<true>(blockIdx.x, f.key_tiles, a.kv_heads, f.splits);
    const int split = place.split, kvh = place.head;
    const Segment sg = find_segment<true, false>(a, kRows, f.key_tiles, place.tile);
    if (a.fill) {
        fill_rest(a, a.cu_k, a.n_k, a.kv_heads, static_cast<T*>(f.dk), f.dk_row, f.dk_head, nullptr);
        fill_rest(a, a.cu_k, a.n_k, a.kv_heads, static_cast<T*>(f.dv), f.dv_row, f.dv_head, nullptr);
    }
    const int key0 = sg.tile * kRows;
    if (key0 >= sg.nk) return;
    const TileRows<ST> tr(f, sg, key0);
    if (split >= tr.parts) return;
    const int lane = lane_id(), h = lane >> 5, wave = threadIdx.x / GS_WAVE;
    const int key = key0 + 32 * wave + (lane & 31);
    const bool there = key < sg.nk;
    const bool on = there && (a.key_on == nullptr || a.key_on[sg.k0 + key]);
    const int shift = sg.nk - sg.nq;

    op8<T> kf[KT], vf[BIG ? 1 : KT];
    {
        const int64_t row = sg.k0 + (there ? key : key0);
        const T* pk = static_cast<const T*>(a.k) + row * a.k_row + (int64_t)kvh * a.k_head;
        const T* pv = static_cast<const T*>(a.v) + row * a.v_row + (int64_t)kvh * a.v_head;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            const int c = 16 * t + 8 * h;
            kf[t] = op8<T>{};
            if (c < a.dim && on) kf[t] = *reinterpret_cast<const op8<T>*>(pk + c);
            if (!BIG) {
                vf[t] = op8<T>{};
                if (c < a.dim && on) vf[t] = *reinterpret_cast<const op8<T>*>(pv + c);
            }
        }
    }
    if (BIG) {
        TileLoader<T, P, kRows> vl;
        vl.init(static_cast<const T*>(a.v) + (sg.k0 + key0) * a.v_row + kvh * a.v_head, sg.nk - key0, a.v_row, a.dim);
        uint32_t skip = 0;
        if (a.key_on != nullptr) {
            const int first = key0 + threadIdx.x / vl.PIECES;
#pragma unroll
            for (int u = 0; u < vl.LOADS; ++u)
                if (key_flag(a.key_on + sg.k0, first + u * vl.STEP, sg.nk) == 0) skip |= 1u << u;
        }
        vl.load(vs, 0, skip);
    }
    // tokens that admit all of the workgroup's keys, and those that admit the lane's
    const int last = min(key0 + kRows, sg.nk) - 1;
    int alo, ahi, ilo, ihi;
    admitting(a, sg.nq, shift, last, key0, alo, ahi);
    admitting(a, sg.nq, shift, key, key, ilo, ihi);
    const int t0 = tr.t0, per = tr.per;
    const int each = (tr.steps + tr.parts - 1) / tr.parts, n0 = split * each, n1 = min(tr.steps, n0 + each);
    // a token that admits no key at all may hold anything: its row is left out
    const bool empties = a.key_on != nullptr || (a.right >= 0 && shift + a.right < 0);

    const int end = t0 + per * ST;
    int fg = n0 / max(per, 1), ft = t0 + (n0 - fg * per) * ST;     // head of the group and token of the next fetch
    int ct = ft;                                                    // and of the next step
    auto q_rows = [&] { return static_cast<const T*>(a.q) + sg.q0 * a.q_row + (kvh * a.group + fg) * a.q_head; };
    auto d_rows = [&] {
        return static_cast<const T*>(f.dout) + sg.q0 * f.do_row + (kvh * a.group + fg) * f.do_head;
    };
    TileLoader<T, P, ST> ql, dl;
    ql.init(q_rows(), sg.nq, a.q_row, a.dim);
    dl.init(d_rows(), sg.nq, f.do_row, a.dim);
    // the rows' bases: +inf for a token that admits nothing, loaded a step before the tiles
    auto bases = [&] { return f.base + (int64_t)(kvh * a.group + fg) * a.n_q + sg.q0; };
    float flag = 0.0f;
    auto load_flag = [&] {
        const int t = ft + (fresh(lane) & (ST - 1));
        flag = t < sg.nq ? bases()[t] : INFINITY;
    };
    auto fetch = [&](T* qs, T* ds, float* st, bool more) {
        const uint32_t skip = empties ? rows_off<P, ST>(__ballot(flag != INFINITY)) : 0;
        ql.load(qs, ft, skip);
        dl.load(ds, ft, skip);
        // bases by the first wave, deltas by the second
        if (wave < 2) load_words(st + wave * 64, bases() + (wave ? f.delta - f.base : 0) + ft, sg.nq - ft);
        ft += ST;
        if (ft >= end) {
            ft = t0;
            ++fg;
            ql.move(q_rows());
            dl.move(d_rows());
        }
        if (empties && more) load_flag();
    };

    const float c = a.scale * kLog2e;
    Lanes at;
    at.init<P>();
    acc16 dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) dk[d] = dv[d] = acc16{};
    auto step = [&](const T* qs, const T* ds, const float* st) {
        at.refresh();
        const int t = ct;
        ct = ct + ST < end ? ct + ST : t0;
        const bool test = t < alo || t + ST > ahi;
        uint64_t seen = ~0ull;
        if (test) seen = bits_between(ilo - t, ihi - t);
        acc16 s[NK]{}, dp[NK];
        // operands are read one product ahead of their use; the barriers keep
        // the compiler from reading more of them ahead, which would not fit the
        // registers of two waves a SIMD
        auto products = [&](int k) {
            op8<T> x[2], y[2], z[2];
            auto read = [&](int e) {
                x[e & 1] = rows_operand<T, P>(qs, at, 32 * k, e);
                y[e & 1] = rows_operand<T, P>(ds, at, 32 * k, e);
                z[e & 1] = BIG ? rows_operand<T, P>(vs, at, 32 * wave, e) : vf[BIG ? 0 : e];
            };
#pragma unroll
            for (int g = 0; g < 4; ++g) {          // dout . v starts from -delta
                const float4 d = *reinterpret_cast<const float4*>(st + 64 + 32 * k + 8 * g + 4 * h);
                dp[k][4 * g] = d.x;
                dp[k][4 * g + 1] = d.y;
                dp[k][4 * g + 2] = d.z;
                dp[k][4 * g + 3] = d.w;
            }
            read(0);
#pragma unroll
            for (int e = 0; e < KT; ++e) {
                if (e + 1 < KT) read(e + 1);
                s[k] = mfma(x[e & 1], kf[e], s[k]);
                dp[k] = mfma(y[e & 1], z[e & 1], dp[k]);
                if (BIG) __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto gradients = [&](int k) {
            if (test) keep_some(s[k], (uint32_t)(seen >> (32 * k)));
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 b = *reinterpret_cast<const float4*>(st + 32 * k + 8 * g + 4 * h);
                const float bs[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[k][4 * g + e] = __builtin_amdgcn_exp2f(fmaf(s[k][4 * g + e], c, -bs[e]));
                    dp[k][4 * g + e] *= s[k][4 * g + e];
                }
            }
        };
        auto sums = [&](int k) {
            op8<T> x[2], y[2], p, z;
            auto read = [&](int e) {               // e: u * DT + d
                x[e & 1] = columns_operand<T, P>(ds, at, 32 * k + 16 * (e / DT), e % DT);
                y[e & 1] = columns_operand<T, P>(qs, at, 32 * k + 16 * (e / DT), e % DT);
            };
            read(0);
#pragma unroll
            for (int e = 0; e < 2 * DT; ++e) {
                if (e + 1 < 2 * DT) read(e + 1);
                if (e % DT == 0) {
                    p = tile_operand<T>(s[k], e / DT);
                    z = tile_operand<T>(dp[k], e / DT);
                }
                dv[e % DT] = mfma(x[e & 1], p, dv[e % DT]);
                dk[e % DT] = mfma(y[e & 1], z, dk[e % DT]);
                if (BIG) __builtin_amdgcn_sched_barrier(0);
            }
        };
        products(0);
        __builtin_amdgcn_sched_barrier(0);
        if (NK > 1) products(NK - 1);              // beside the first half's exponentials
        gradients(0);
        __builtin_amdgcn_sched_barrier(0);
        sums(0);                                   // beside the second half's
        if (NK > 1) {
            gradients(NK - 1);
            __builtin_amdgcn_sched_barrier(0);
            sums(NK - 1);
        }
    };
    if (n0 < n1) {
        if (empties) load_flag();
        fetch(qs0, ds0, st0, n0 + 1 < n1);
    }
    __syncthreads();                               // the fetched tiles are in LDS
    for (int n = n0; n < n1; n += 2) {
        if (n + 1 < n1) fetch(qs1, ds1, st1, n + 2 < n1);
        step(qs0, ds0, st0);
        __syncthreads();
        if (n + 1 < n1) {
            if (n + 2 < n1) fetch(qs0, ds0, st0, n + 3 < n1);
            step(qs1, ds1, st1);
        }
        __syncthreads();
    }
    if (!there) return;
    if (!on) {                                     // what a key that is off has summed is in its column alone
#pragma unroll
        for (int d = 0; d < DT; ++d) dk[d] = dv[d] = acc16{};
    }
    const int64_t token = sg.k0 + key;
    if (tr.parts > 1) {
        const int64_t n = (int64_t)a.n_k * a.kv_heads;
        float* pk = f.part + ((int64_t)split * 2 * n + token * a.kv_heads + kvh) * a.dim;
        store_tiles<float, DT>(pk, dk, a.scale, a.dim);
        store_tiles<float, DT>(pk + n * a.dim, dv, 1.0f, a.dim);
        return;
    }
    store_tiles<T, DT>(static_cast<T*>(f.dk) + token * f.dk_row + (int64_t)kvh * f.dk_head, dk, a.scale, a.dim);
    store_tiles<T, DT>(static_cast<T*>(f.dv) + token * f.dv_row + (int64_t)kvh * f.dv_head, dv, 1.0f, a.dim);
}

// Sums the parts of dk or dv of 32 of a key tile's keys in ascending order, four
// elements a thread at a time.  Bound by the parts' bytes: 3.5 parts on average of
// 8192 keys, 4 heads of 128: 22 us.
template <typename T, int ST>
__global__ void __launch_bounds__(GS_BLOCK) k_attention_dkv_join(BwdArgs f) {
    const AttnArgs& a = f.a;
    const int which = blockIdx.x & 1, key1 = blockIdx.x / 2 % 4 * 32;
    const Place place = chiplet_place<false>(blockIdx.x / 8, f.key_tiles, a.kv_heads, 1);
    const int kvh = place.head;
    const Segment sg = find_segment<true, false>(a, kRows, f.key_tiles, place.tile);
    const int key0 = sg.tile * kRows;
    if (key0 + key1 >= sg.nk) return;
    const TileRows<ST> tr(f, sg, key0);
    if (tr.parts == 1) return;                             // written where it belongs
    const int per = a.dim / 4, n = min(32, sg.nk - key0 - key1) * per;
    const int64_t rows = (int64_t)a.n_k * a.kv_heads, token0 = sg.k0 + key0 + key1;
    T* const out = static_cast<T*>(which ? f.dv : f.dk) + kvh * (which ? f.dv_head : f.dk_head);
    const int64_t ld = which ? f.dv_row : f.dk_row;
    for (int x = threadIdx.x; x < n; x += GS_BLOCK) {
        const int key = x / per, c = 4 * (x - key * per);
        const float* p = f.part + (which * rows + (token0 + key) * a.kv_heads + kvh) * a.dim + c;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (int s = 0; s < tr.parts; ++s) {
            const float4 w = *reinterpret_cast<const float4*>(p + 2 * s * rows * a.dim);
            v.x += w.x;
            v.y += w.y;
            v.z += w.z;
            v.w += w.w;
        }
        op4<T> o;
        o[0] = (T)v.x;
        o[1] = (T)v.y;
        o[2] = (T)v.z;
        o[3] = (T)v.w;
        *reinterpret_cast<op4<T>*>(out + (token0 + key) * ld + c) = o;
    }
}

struct DkvPlan {
    int splits, chunk;
};

// How the key tiles' rows are cut, from the sizes alone: into runs of about one
// length, three to a compute unit (two fit it), as long as a run keeps 512
// tokens.  A window makes some tiles' rows fewer, so their mean is taken over 32
// tiles of a segment of mean length.  8192 ordered tokens, 16/4 heads of 128, the
// whole gradient: 1050 us with every tile in two parts, 967 so; 1079 and 1032
// with two and four runs to a unit.
DkvPlan dkv_plan(const gs_attn& a) {
    constexpr int kUnits = 256, kMost = 16, kTiles = 32;
    const int group = a.heads / a.kv_heads, st = dkv_step(a.dim);
    const int64_t nq = a.n_q / a.n_seg, nk = a.n_k / a.n_seg, shift = nk - nq;
    int64_t rows = 0, most = 0;
    for (int i = 0; i < kTiles; ++i) {
        const int64_t key = nk * (2 * i + 1) / (2 * kTiles);
        const int64_t lo = a.right >= 0 ? std::max<int64_t>(0, key - a.right - shift) : 0;
        const int64_t hi = a.left >= 0 ? std::min<int64_t>(nq, key + a.left - shift + 1) : nq;
        rows += std::max<int64_t>(0, hi - lo);
        most = std::max(most, hi - lo);
    }
    const int64_t groups = (int64_t)attn_tiles(a.n_k, kRows, a.n_seg) * a.kv_heads;
    const int64_t mean = (rows + kTiles - 1) / kTiles;     // rounded up: below one, a part would be as short as can be
    const int64_t steps = (mean + st - 1) / st * group, longest = (most + st - 1) / st * group;
    const int64_t chunk = std::max<int64_t>(512 / st, groups * steps / (3 * kUnits));
    DkvPlan p;
    p.chunk = (int)std::min<int64_t>(chunk, 1 << 30);
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>((longest + p.chunk - 1) / p.chunk, kMost));
    return p;
}

template <typename T, int D>
hipError_t go(const BwdArgs& f, hipStream_t st) {
    if (f.a.n_q > 0)
        (f.a.key_on ? k_attention_dq<T, D, true> : k_attention_dq<T, D, false>)
            <<<(uint32_t)(f.a.tiles * f.a.kv_heads), GS_BLOCK, 0, st>>>(f);
    if (f.a.n_k > 0) {
        const uint32_t tiles = (uint32_t)(f.key_tiles * f.a.kv_heads);
        k_attention_dkv<T, D><<<tiles * f.splits, GS_BLOCK, 0, st>>>(f);
        if (f.splits > 1) k_attention_dkv_join<T, dkv_step(D)><<<8 * tiles, GS_BLOCK, 0, st>>>(f);
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
    const int splits = dkv_plan(a).splits;
    const size_t parts = splits > 1 ? (size_t)splits * 2 * a.n_k * a.kv_heads * a.dim * sizeof(float) : 0;
    return align256((size_t)a.n_q * a.heads * 2 * sizeof(float)) + align256(parts);
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
    f.do_row = row_stride(g.dout, a.n_q, a.dim);
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
    f.base = static_cast<float*>(ws);
    f.delta = f.base + (size_t)a.n_q * a.heads;
    const DkvPlan plan = dkv_plan(a);
    f.splits = plan.splits;
    f.chunk = plan.chunk;
    f.part = reinterpret_cast<float*>(static_cast<char*>(ws) + align256((size_t)a.n_q * a.heads * 2 * sizeof(float)));
    return (a.dtype & ~GS_ATTN_FILL) == GS_BF16 ? by_dim<bf16_t>(f, st) : by_dim<f16_t>(f, st);
}

}  // namespace gsmi
