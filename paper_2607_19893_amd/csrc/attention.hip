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
constexpr int kPart = 1024, kPartFew = 256;    // least keys of a part
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct FwdArgs {
    AttnArgs a;
    void* out;
    int64_t o_row, o_head;
    float* lse;
    int32_t splits;                        // most parts that a segment's keys are cut into
    int32_t chunk;                         // few rows: keys of a part; 0: every segment has `splits` parts
    float* part_o;                         // [splits][n_q * heads][dim], unnormalised
    float2* part_ml;                       // [splits][n_q * heads] maximum (of the raw products) and sum
};

__device__ __forceinline__ float half_max(float v) {
    const float2 h = halves(v);
    return fmaxf(h.x, h.y);
}
__device__ __forceinline__ float half_sum(float v) {
    const float2 h = halves(v);
    return h.x + h.y;
}

__device__ __forceinline__ float row_scale(float l) { return l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l); }
__device__ __forceinline__ float row_lse(float m, float l, float scale) {
    return l == 0.0f ? -INFINITY : m * scale + kLn2 * log2f(l);
}

// Where a row's results go: its part of the keys, or the output.
// The maximum is that of the raw products, the tile holds 32 elements of a row.
__device__ __forceinline__ void store_sums(const FwdArgs& f, bool parts, int token, int head, int split, float m,
                                           float l) {
    const int64_t row = (int64_t)token * f.a.heads + head;
    if (lane_id() >= 32) return;
    if (parts) f.part_ml[(int64_t)split * f.a.n_q * f.a.heads + row] = make_float2(m, l);
    else f.lse[row] = row_lse(m, l, f.a.scale);
}

template <typename T>
__device__ __forceinline__ void store_tile(const FwdArgs& f, bool parts, int token, int head, int split, int d,
                                           const acc16& o, float l) {
    const int h = fresh(lane_id()) >> 5;
    if (parts) {
        const int64_t row = (int64_t)token * f.a.heads + head;
        float* p = f.part_o + ((int64_t)split * f.a.n_q * f.a.heads + row) * f.a.dim;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int c = 32 * d + 8 * g + 4 * h;
            if (c < f.a.dim)
                *reinterpret_cast<float4*>(p + c) = make_float4(o[4 * g], o[4 * g + 1], o[4 * g + 2], o[4 * g + 3]);
        }
        return;
    }
    const float inv = row_scale(l);                        // a NaN sum stays one
    T* p = static_cast<T*>(f.out) + (int64_t)token * f.o_row + (int64_t)head * f.o_head;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int c = 32 * d + 8 * g + 4 * h;
        op4<T> v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (T)(o[4 * g + i] * inv);
        if (c < f.a.dim) *reinterpret_cast<op4<T>*>(p + c) = v;
    }
}

// What a sum against maximum m counts against another, base = its rounded product
// with c.  The probabilities stand against the rounded m c, so that is what is
// taken here.  With the exact product every rise in a wave changed the sums of its
// other rows by a factor 2^(m c's rounding): scores of 4000 that met 128 rises had
// outputs off by 0.005 of their values.
__device__ __forceinline__ float against(float m, float c, float base) {
#pragma clang fp contract(off)
    const float mc = m * c;
    return __builtin_amdgcn_exp2f(mc - base);
}

// One step of the online softmax over a tile of 32 N keys: s (raw products,
// -inf where not admitted) becomes the probabilities against the running
// maximum m.  c = scale * log2(e).  The maximum is held until a score passes it
// by more than kHeld powers of two: probabilities up to 2^kHeld lose nothing in
// either type, and in most steps neither the sum nor the output is rescaled.
// Returns whether the output is to be, by alpha.
constexpr float kHeld = 8.0f;

__device__ __forceinline__ float held(float c) { return fminf(kHeld / c, 3.0e38f); }

template <int N>
__device__ __forceinline__ bool softmax_step(acc16 (&s)[N], float c, float slack, float& m, float& l, float& alpha) {
    // four chains each for the maximum and the sum: one would wait for itself
    float t4[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) t4[i & 3] = fmaxf(t4[i & 3], s[k][i]);
    const float t = half_max(fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])));
    const bool rise = __any(t > m + slack);
    if (rise) {
        const float top = fmaxf(m, t);
        alpha = against(m, c, top == -INFINITY ? 0.0f : top * c);
        l *= alpha;
        m = top;
    }
    const float base = m == -INFINITY ? 0.0f : m * c;      // nothing admitted yet: exp2(-inf) = 0 below
    float sum4[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[k][i] = __builtin_amdgcn_exp2f(fmaf(s[k][i], c, -base));
            sum4[i & 3] += s[k][i];
        }
    l += (sum4[0] + sum4[1]) + (sum4[2] + sum4[3]);        // this half's keys; the halves meet at the end
    return rise;
}

// 128 rows a workgroup, 64 keys a step.  Up to 64 elements a head three waves fit
// a SIMD, from 96 on two.  8192 ordered tokens, 16/4 heads of 128: 281 us, 980
// TFLOP/s of the products that the mask leaves; matrix units busy 53% of the
// cycles and vector units 54%, at clocks that the power limit sets (operands of
// zeros run 1.35 times faster).  40 regions of 40..1600 fp16 tokens, 8 heads of
// 64: 48 us, vector units busy 66% and matrix units 28%, waves waiting for data 30%
// of their time: a score's exponential, maximum, sum and rounding cost more issue
// cycles there than its 256 multiply-adds.
template <typename T, int D>
__global__ void __launch_bounds__(GS_BLOCK, D <= 64 ? 3 : 2) k_attention(FwdArgs f) {
    constexpr int P = D <= 32 ? 32 : (D <= 64 ? 64 : 128), KT = D / 16, DT = D / 32;
    constexpr int G = KT < 4 ? 2 : 4;                           // products whose operands are read together
    // two buffers: a step's tiles arrive while the step before computes
    __shared__ __attribute__((aligned(16))) T ks0[kKeys * P], vs0[kKeys * P];
    __shared__ __attribute__((aligned(16))) T ks1[kKeys * P], vs1[kKeys * P];
    const AttnArgs& a = f.a;
    const Place place = chiplet_place<(D > 64)>(blockIdx.x, a.tiles, a.kv_heads, f.splits);
    const int split = place.split, kvh = place.head;
    const Segment sg = find_segment<false, true>(a, kRows, a.tiles, place.tile);
    if (a.fill) fill_rest(a, a.cu_q, a.n_q, a.heads, static_cast<T*>(f.out), f.o_row, f.o_head, f.lse);
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
        const int per = max(((max(hi - j0, 0) + f.splits - 1) / f.splits + kKeys - 1) / kKeys * kKeys, kPart);
        j0 += split * per;
        j1 = min(hi, j0 + per);
        if (j0 >= j1 && split > 0) {                       // nothing left for this part
            if (there) store_sums(f, f.splits > 1, token, head, split, -INFINITY, 0.0f);
            return;
        }
    }

    TileLoader<T, P, kKeys> kl, vl;
    kl.init(static_cast<const T*>(a.k) + sg.k0 * a.k_row + kvh * a.k_head, sg.nk, a.k_row, a.dim);
    vl.init(static_cast<const T*>(a.v) + sg.k0 * a.v_row + kvh * a.v_head, sg.nk, a.v_row, a.dim);
    // Which keys of a step are on is loaded a step before its tiles, so that
    // nothing waits for it: `on` for the step that computes, `on_next` for the
    // one whose tiles arrive, `flag` (a key a lane) for the one after.
    const uint8_t* const flags = a.key_on + sg.k0;
    uint64_t on = ~0ull, on_next = ~0ull;
    uint8_t flag = 1;
    auto fetch = [&](T* ks, T* vs, int j) {
        uint32_t skip = 0;
        if (a.key_on != nullptr) {
            on_next = __ballot(flag);
            flag = key_flag(flags, j + kKeys + fresh(lane), sg.nk);
            skip = rows_off<P, kKeys>(on_next);
        }
        kl.load(ks, j, 0);
        vl.load(vs, j, skip);     // a probability of 0 does not stop a NaN
    };

    const float c = a.scale * kLog2e, slack = held(c);
    float m = -INFINITY, l = 0.0f;
    acc16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = acc16{};

    Lanes at;
    at.init<P>();
    auto step = [&](const T* ks, const T* vs, int j) {
        // operands are read a group of products ahead of their use; the
        // barriers keep the compiler from reading more of them ahead, which
        // would not fit the registers of two waves a SIMD
        at.refresh();
        acc16 s[2];
        op8<T> x[2][G];
#pragma unroll
        for (int e = 0; e < G; ++e) x[0][e] = rows_operand<T, P>(ks, at, 0, e);
#pragma unroll
        for (int g = 0; g < 2 * KT / G; ++g) {
            if (g + 1 < 2 * KT / G) {
#pragma unroll
                for (int e = 0; e < G; ++e)
                    x[(g + 1) & 1][e] = rows_operand<T, P>(ks, at, ((g + 1) * G + e) / KT * 32, ((g + 1) * G + e) % KT);
            }
#pragma unroll
            for (int e = 0; e < G; ++e) {
                const int n = g * G + e;
                s[n / KT] = mfma(x[g & 1][e], q[n % KT], n % KT == 0 ? acc16{} : s[n / KT]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (a.key_on != nullptr || j < alo || j + kKeys > ahi) {
            const uint64_t seen = bits_between(klo - j, khi - j) & on;
            keep_some(s[0], (uint32_t)seen);
            keep_some(s[1], (uint32_t)(seen >> 32));
        }
        op8<T> y[2][DT];                           // on their way while the exponentials run
#pragma unroll
        for (int d = 0; d < DT; ++d) y[0][d] = columns_operand<T, P>(vs, at, 0, d);
#pragma unroll
        for (int d = 0; d < DT; ++d) y[1][d] = columns_operand<T, P>(vs, at, 16, d);
        __builtin_amdgcn_sched_barrier(0);
        float alpha;
        if (softmax_step<2>(s, c, slack, m, l, alpha)) {
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= alpha;
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const op8<T> p = tile_operand<T>(s[g / 2], g % 2);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                o[d] = mfma(y[g & 1][d], p, o[d]);
                if (g < 2) y[g & 1][d] = columns_operand<T, P>(vs, at, 16 * (g + 2), d);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    if (j0 < j1) {
        if (a.key_on != nullptr) flag = key_flag(flags, j0 + lane, sg.nk);
        fetch(ks0, vs0, j0);
    }
    __syncthreads();                               // the fetched tiles are in LDS
    for (int j = j0; j < j1; j += 2 * kKeys) {
        on = on_next;
        if (j + kKeys < j1) fetch(ks1, vs1, j + kKeys);
        step(ks0, vs0, j);
        __syncthreads();
        if (j + kKeys < j1) {
            on = on_next;
            if (j + 2 * kKeys < j1) fetch(ks0, vs0, j + 2 * kKeys);
            step(ks1, vs1, j + kKeys);
        }
        __syncthreads();
    }
    l = half_sum(l);
    if (!there) return;
    store_sums(f, f.splits > 1, token, head, split, m, l);
#pragma unroll
    for (int d = 0; d < DT; ++d) store_tile<T>(f, f.splits > 1, token, head, split, d, o[d], l);
}

// Few rows over many keys: a workgroup takes a part of a segment's keys, for all
// of the segment's rows (32 at a time, seldom more), and every wave of it its own
// keys (32 a step, its waves' steps interleaved), with a running maximum and sum
// of its own; the waves meet in LDS at the end.  Segments are cut into parts of
// about the same length, so long and short ones load the chip alike.  The keys'
// bytes bound it, so a step's keys go from memory straight into the operand's
// registers, its values through a piece of LDS that only this wave touches (no
// barrier in the loop), and both are fetched a step ahead.  One token over 32,768
// keys, 32/8 heads of 128: 29 us, 4.6 TB/s.  24 segments of 1..16 rows over
// 900..9000 keys, 16 heads of 64: 75 us, 4.2 TB/s (two waves a SIMD; held to the
// registers of three it took 3 us more).
constexpr int kFewRows = 32;

template <typename T, int D>
__global__ void __launch_bounds__(GS_BLOCK, 2) k_attention_few(FwdArgs f) {
    constexpr int P = D <= 32 ? 32 : (D <= 64 ? 64 : 128), KT = D / 16, DT = D / 32;
    constexpr int PIECES = P / 8, LOADS = 32 * PIECES / GS_WAVE, WAVES = GS_BLOCK / GS_WAVE;
    __shared__ __attribute__((aligned(16))) T vs[WAVES][32 * P];
    __shared__ float ml[2][WAVES][32];
    __shared__ float tile[WAVES][16 * GS_WAVE];              // a C tile of each wave, register by register
    const AttnArgs& a = f.a;
    const Place place = chiplet_place<false>(blockIdx.x, a.tiles, a.kv_heads, 1);
    const int kvh = place.head;
    const Segment sg = find_segment<true, false, true>(a, f.chunk, a.tiles, place.tile);
    if (a.fill) fill_rest(a, a.cu_q, a.n_q, a.heads, static_cast<T*>(f.out), f.o_row, f.o_head, f.lse);
    const int parts = max((sg.nk + f.chunk - 1) / f.chunk, 1), split = sg.tile;
    const int rows = sg.nq * a.group;
    if (split >= parts) return;
    const int per = ((sg.nk + parts - 1) / parts + 127) / 128 * 128;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / GS_WAVE);
#pragma unroll 1
    for (int row0 = 0; row0 < rows; row0 += kFewRows) {
        const int lane = fresh(lane_id()), h = lane >> 5;      // nothing of it is held over the loop
        const int r = row0 + (lane & 31);
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
        int klo, khi, lo, hi, alo, ahi;
        admitted(a, sg.nk, i + shift, i + shift, klo, khi);
        const int last = min(row0 + kFewRows, rows) - 1;
        admitted(a, sg.nk, row0 / a.group + shift, last / a.group + shift, lo, hi);
        admitted(a, sg.nk, last / a.group + shift, row0 / a.group + shift, alo, ahi);
        const int j0 = max(lo / 32 * 32, split * per), j1 = min(hi, (split + 1) * per);
        if (j0 >= j1 && split > 0) {                           // the window leaves nothing of this part
            if (wave == 0 && there) store_sums(f, true, token, head, split, -INFINITY, 0.0f);
            continue;
        }
        constexpr int STEP = GS_WAVE / PIECES;
        RowBuffer<T> kb, vb;
        kb.init(static_cast<const T*>(a.k) + sg.k0 * a.k_row + kvh * a.k_head, sg.nk, a.k_row);
        vb.init(static_cast<const T*>(a.v) + sg.k0 * a.v_row + kvh * a.v_head, sg.nk, a.v_row);
        const int koff = (lane & 31) * kb.ld + 16 * h;
        const int voff = 8 * (lane % PIECES) < a.dim ? lane / PIECES * vb.ld + 16 * (lane % PIECES) : vb.kOutside;
        const uint8_t* const flags = a.key_on + sg.k0;
        op8<T> kp[KT], vp[LOADS];
        uint8_t flag = 1;                                      // of key lane & 31 of the step
        auto fetch = [&](int j) {
            if (a.key_on != nullptr) flag = key_flag(flags, j + (fresh(lane) & 31), sg.nk);
            const int ka = koff + kb.place(j), va = vb.place(j);
#pragma unroll
            for (int t = 0; t < KT; ++t) kp[t] = kb.piece(16 * t + 8 * h < a.dim ? ka + 32 * t : kb.kOutside);
#pragma unroll
            for (int u = 0; u < LOADS; ++u) vp[u] = vb.piece((int)((uint32_t)voff + (uint32_t)(va + u * STEP * vb.ld)));
        };

        const float c = a.scale * kLog2e, slack = held(c);
        float m = -INFINITY, l = 0.0f;
        acc16 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = acc16{};
        Lanes at;
        at.init<P>();
        T* const mine = vs[wave];
        int j = j0 + 32 * wave;
        fetch(j < j1 ? j : sg.nk);
        for (; j < j1; j += 32 * WAVES) {
            at.refresh();
            acc16 s[1];
            s[0] = acc16{};
#pragma unroll
            for (int t = 0; t < KT; ++t) s[0] = mfma(kp[t], q[t], s[0]);
            uint32_t on = ~0u;
            if (a.key_on != nullptr) {
                on = (uint32_t)__ballot(flag);
                // the values of a key that is off may be anything, and a
                // probability of 0 does not stop a NaN
#pragma unroll
                for (int u = 0; u < LOADS; ++u)
                    if (((on >> (u * STEP + fresh(lane) / PIECES)) & 1) == 0) vp[u] = op8<T>{};
            }
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                const int x = lane + u * GS_WAVE;
                *reinterpret_cast<op8<T>*>(mine + piece_at<P>(x / PIECES, x % PIECES)) = vp[u];
            }
            if (a.key_on != nullptr || j < alo || j + 32 > ahi)
                keep_some(s[0], (uint32_t)bits_between(klo - j, khi - j) & on);
            // behind the part's end: from past the segment's, which reads nothing
            // (a condition on the loads would keep both outcomes' registers)
            fetch(j + 32 * WAVES < j1 ? j + 32 * WAVES : sg.nk);
            float alpha;
            if (softmax_step<1>(s, c, slack, m, l, alpha)) {
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] *= alpha;
            }
            // this wave's values are in LDS before any of its lanes reads them
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const op8<T> p = tile_operand<T>(s[0], u);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    o[d] = mfma(columns_operand<T, P>(mine, at, 16 * u, d), p, o[d]);
                    if (d & 1) __builtin_amdgcn_sched_barrier(0);      // no operands further ahead: two waves a SIMD
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        // the waves meet: the largest maximum, every sum and tile against it
        l = half_sum(l);
        const int me = fresh(lane_id()), column = me & 31;
        if (me < 32) {
            ml[0][wave][me] = m;
            ml[1][wave][me] = l;
        }
        __syncthreads();
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ml[0][w][column]);
        const float base = top == -INFINITY ? 0.0f : top * c;
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
            sum = fmaf(ml[1][w][column], against(ml[0][w][column], c, base), sum);
        const float alpha = against(m, c, base);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
#pragma unroll
            for (int e = 0; e < 16; ++e) tile[wave][e * GS_WAVE + me] = o[d][e] * alpha;
            __syncthreads();
            if (wave == d % WAVES && there) {
                acc16 v;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    v[e] = tile[0][e * GS_WAVE + me];
#pragma unroll
                    for (int w = 1; w < WAVES; ++w) v[e] += tile[w][e * GS_WAVE + me];
                }
                store_tile<T>(f, parts > 1, token, head, split, d, v, sum);
            }
            __syncthreads();
        }
        if (wave == 0 && there) store_sums(f, parts > 1, token, head, split, top, sum);
    }
}

// Joins the parts of a row (at most kMaxSplits): lanes take the parts' maxima
// and sums together, then two elements each and the parts in turn, 8 or 16 tiles
// of a wave on their way at once.  Bound by the latency of these two reads, one
// behind the other.  A wave a row where there are up to 8 parts on average (24
// segments, 16 heads of 64: the call 83.2 us, 84.9 with four waves), four up to
// 64 (32 parts of 32 rows of 128: 4.2 us), 16 beyond (one row of 128 in 256 parts:
// the call 18.4 us, 19.9 with four).
constexpr int kMaxSplits = 256;

template <typename T, int WAVES>
__global__ void __launch_bounds__(WAVES == 1 ? GS_BLOCK : WAVES * GS_WAVE) k_attention_join(FwdArgs f) {
    constexpr int N = kMaxSplits / GS_WAVE, GROUPS = WAVES == 1 ? 1 : WAVES / 4;
    constexpr int EACH = WAVES == 1 ? 8 : 16, STEP = WAVES == 1 ? 1 : 4;
    __shared__ float2 got[WAVES][GS_WAVE];
    const int64_t rows = (int64_t)f.a.n_q * f.a.heads;
    const int wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / GS_WAVE);
    const int64_t row = WAVES == 1 ? (int64_t)blockIdx.x * (GS_BLOCK / GS_WAVE) + threadIdx.x / GS_WAVE : blockIdx.x;
    if (row >= rows) return;
    const int lane = lane_id();
    const int64_t token = row / f.a.heads;
    int parts = f.splits;
    if (f.chunk > 0 || f.a.cu_q != nullptr) {
        const int keys = __builtin_amdgcn_readfirstlane(keys_of_token(f.a, (int)token));
        if (keys < 0) return;                              // in no segment
        if (f.chunk > 0) {
            if (keys <= f.chunk) return;                   // one part: written where it belongs
            parts = (keys + f.chunk - 1) / f.chunk;
        }
    }
    float2 part[N];
    float m = -INFINITY;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int s = n * GS_WAVE + lane;
        part[n] = s < parts ? f.part_ml[s * rows + row] : make_float2(-INFINITY, 0.0f);
        m = fmaxf(m, part[n].x);
    }
#pragma unroll
    for (int d = 1; d < GS_WAVE; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, GS_WAVE));
    const float c = f.a.scale * kLog2e, base = m == -INFINITY ? 0.0f : m * c;
    float w[N], l = 0.0f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        w[n] = against(part[n].x, c, base);
        l = fmaf(part[n].y, w[n], l);
    }
    l = wave_sum(l);
    float2 o = make_float2(0.0f, 0.0f);
    const float* p = f.part_o + row * f.a.dim + (2 * lane < f.a.dim ? 2 * lane : 0);
    const int64_t step = rows * f.a.dim;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n * GS_WAVE >= parts || n % GROUPS != wave / 4) continue;
        // a part that found no keys may have written no tile
        const uint64_t wrote = __ballot(part[n].y != 0.0f);
#pragma unroll 1
        for (int first = 0; first < min(parts - n * GS_WAVE, GS_WAVE); first += EACH * STEP) {
            float2 v[EACH];
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                v[i] = make_float2(0.0f, 0.0f);
                const int s = first + wave % 4 + STEP * i;
                if ((wrote >> s) & 1) v[i] = *reinterpret_cast<const float2*>(p + (n * GS_WAVE + s) * step);
            }
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int s = first + wave % 4 + STEP * i;
                const float ws = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w[n]), s));
                o.x = fmaf(v[i].x, ws, o.x);
                o.y = fmaf(v[i].y, ws, o.y);
            }
        }
    }
    if (WAVES > 1) {
        got[wave][lane] = o;
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int k = 1; k < WAVES; ++k) {
            o.x += got[k][lane].x;
            o.y += got[k][lane].y;
        }
    }
    const float inv = row_scale(l);
    const int head = (int)(row - token * f.a.heads);
    if (lane == 0) f.lse[row] = row_lse(m, l, f.a.scale);
    if (2 * lane < f.a.dim) {
        T* p = static_cast<T*>(f.out) + token * f.o_row + (int64_t)head * f.o_head + 2 * lane;
        p[0] = (T)(o.x * inv);
        p[1] = (T)(o.y * inv);
    }
}

// How a call is cut, from its sizes alone.
struct Plan {
    bool few;
    int32_t tiles, splits, chunk;
};

// Few rows: where a segment's rows fit one 32-row tile on average.  The keys of
// all segments and key heads are cut into parts for one workgroup a compute unit,
// or for three where the segments' lengths may differ (two are there at a time,
// the third evens out the ends), but at least 256 keys, which pay for a start and
// a join; a longer segment has more of them.  Heads of 32, 64, 96 and 128, one a
// unit against three: 24 regions of 900..9000 keys, 16 heads, 62 100 157 169
// against 66 87 143 151 us; one row over 32,768 keys, 32/8 heads, 21 24 32 38
// against 21 29 36 42.  Equal segments of 64, 16/8 heads: 8 of 16,384 65 against
// 77, 64 of 1500 56 against 67, 24 of 4000 63 against 59.  The parts' sums may
// take 64 MB.
// More rows: 128-row tiles, and the keys into parts where those tiles leave
// compute units idle.
Plan plan(const gs_attn& a) {
    constexpr int kUnits = 256;                            // compute units
    Plan p;
    const int group = a.heads / a.kv_heads;
    const int64_t rows = (int64_t)a.n_q * group, keys = a.n_k / a.n_seg;
    p.few = rows <= (int64_t)kFewRows * a.n_seg;
    if (p.few) {
        const bool equal = a.cu_q == nullptr || a.n_seg == 1;
        const int64_t longest = equal ? keys : a.n_k;      // as far as it is known here
        const int64_t want = kUnits * (equal ? 1 : 3);
        const int64_t part = std::max<int64_t>(1, (int64_t)a.n_q * a.heads) * a.dim * 4;
        const int64_t room = std::max<int64_t>(1, (64 << 20) / part);
        const int64_t most = std::min<int64_t>(kMaxSplits, room);
        int64_t chunk = std::max<int64_t>({kPartFew, (int64_t)a.n_k * a.kv_heads / want, (longest + most - 1) / most});
        chunk = (chunk + 127) / 128 * 128;
        p.chunk = (int32_t)std::min<int64_t>(chunk, 0x7FFFFF00);
        p.splits = (int32_t)std::max<int64_t>(1, (longest + p.chunk - 1) / p.chunk);
        p.tiles = whole_shares(attn_tiles(a.n_k, p.chunk, a.n_seg), a.kv_heads);
        return p;
    }
    p.chunk = 0;
    p.tiles = whole_shares(attn_tiles(rows, kRows, a.n_seg), a.kv_heads);
    const int64_t groups = (int64_t)p.tiles * a.kv_heads;
    p.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>((2 * kUnits + groups - 1) / groups, keys / kPart));
    return p;
}

template <typename T, int D>
hipError_t go(const FwdArgs& f, bool few, hipStream_t st) {
    const uint32_t grid = (uint32_t)(f.a.tiles * f.a.kv_heads * (few ? 1 : f.splits));
    if (few) k_attention_few<T, D><<<grid, GS_BLOCK, 0, st>>>(f);
    else k_attention<T, D><<<grid, GS_BLOCK, 0, st>>>(f);
    const uint64_t rows = (uint64_t)f.a.n_q * f.a.heads;
    if (f.splits > 1) {
        // parts of a row: all have `splits`, or the mean of the segments
        const bool equal = f.chunk == 0 || f.a.n_seg == 1;
        const int parts = equal ? f.splits : (f.a.n_k / f.a.n_seg + f.chunk - 1) / f.chunk;
        if (parts <= 8) k_attention_join<T, 1><<<div_up(rows, 4), GS_BLOCK, 0, st>>>(f);
        else if (parts <= 64) k_attention_join<T, 4><<<(uint32_t)rows, GS_BLOCK, 0, st>>>(f);
        else k_attention_join<T, 16><<<(uint32_t)rows, 16 * GS_WAVE, 0, st>>>(f);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t by_dim(const FwdArgs& f, bool few, hipStream_t st) {
    if (f.a.dim <= 32) return go<T, 32>(f, few, st);
    if (f.a.dim <= 64) return go<T, 64>(f, few, st);
    if (f.a.dim <= 96) return go<T, 96>(f, few, st);
    return go<T, 128>(f, few, st);
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
    f.chunk = p.chunk;
    f.part_ml = static_cast<float2*>(ws);
    const size_t sums = align256((size_t)a.n_q * a.heads * p.splits * sizeof(float2));
    f.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + sums);
    return (a.dtype & ~GS_ATTN_FILL) == GS_BF16 ? by_dim<bf16_t>(f, p.few, st) : by_dim<f16_t>(f, p.few, st);
}

}  // namespace gsmi
