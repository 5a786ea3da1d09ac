// Gated linear recurrence over ragged segments, and its gradient.
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace gsmi {

namespace {

// ---------------------------------------------------------------------------
//   a_t = sigma(gate_t);  h_t = a_t h_{t-1} + (1 - a_t) x_t
// A run of tokens maps the state in front of it to the one behind it by
// h -> A h + B, and two runs in a row by (A2 A1, A2 B1 + B2); a segment's first
// token starts anew (B alone, whatever the state was).  So all segments are one
// list of tokens, cut into chunks of kWaves * kSteps: a wave takes kSteps tokens
// of 128 channels, two a lane, and finds its own map with every gate and token
// in registers; the maps of a chunk's waves meet in LDS, those of the chunks in
// global memory.  `reverse` turns the list around (place p is token n - 1 - p).
// Three launches for long lists: the chunks' maps, the states in front of them,
// the tokens once more with those.
// ---------------------------------------------------------------------------

constexpr int kSteps = 16;                     // tokens of a wave
constexpr int kWaves = 8;                      // of a workgroup
constexpr int kChunk = kSteps * kWaves;
constexpr int kCols = 2 * GS_WAVE;             // channels of a workgroup
constexpr int kKeptWaves = GS_RECUR_KEEP / kSteps;
static_assert(GS_RECUR_KEEP % kSteps == 0 && kChunk % GS_RECUR_KEEP == 0, "a kept state is in front of a wave");

constexpr uint32_t kStart = 1, kEnd = 2, kOutside = 0xFFFFFFFFu;

struct Recur {
    gs_recur a;
    const uint32_t* map;                       // of place p: segment << 2 | kEnd | kStart, or kOutside
    float2* maps;                              // [chunks][blocks * kCols]: (A, B)
    float* states;                             // [chunks][blocks * kCols]: in front of (behind, on the way back)
    uint32_t* anew;                            // [chunks]: a segment starts (ends) in it
    int32_t chunks, blocks;
};

struct RecurOut {
    void* y;
    float* final;
    float* kept;
    int64_t ld_y;
};

__device__ __forceinline__ int32_t start_of(const gs_recur& a, int32_t s) {
    if (a.cu == nullptr) return (int32_t)((int64_t)a.n / a.n_seg * s);
    return min(max(a.cu[s], 0), a.n);
}

// What the map holds for place p.
__device__ __forceinline__ uint32_t place_word(const gs_recur& a, int32_t p) {
    const int32_t t = a.reverse ? a.n - 1 - p : p;
    int32_t lo = 0, hi = a.n_seg;              // the last s with start_of(s) <= t
    if (a.cu == nullptr) {
        lo = t / (a.n / a.n_seg);
    } else {
        while (lo < hi) {
            const int32_t mid = (int32_t)(((int64_t)lo + hi + 1) / 2);
            if (start_of(a, mid) <= t) lo = mid;
            else hi = mid - 1;
        }
    }
    if (lo >= a.n_seg) return kOutside;
    const int32_t first = start_of(a, lo), end = start_of(a, lo + 1);
    if (t < first || t >= end) return kOutside;
    const bool at_first = t == first, at_last = t == end - 1;
    return (uint32_t)lo << 2 | ((a.reverse ? at_first : at_last) ? kEnd : 0u) | ((a.reverse ? at_last : at_first) ? kStart : 0u);
}

__global__ void __launch_bounds__(GS_BLOCK) k_recur_map(gs_recur a, uint32_t* __restrict__ map) {
    const int64_t p = (int64_t)blockIdx.x * GS_BLOCK + threadIdx.x;
    if (p < a.n) map[p] = place_word(a, (int32_t)p);
}

// A wave's tokens: bit i of the masks is place p0 + i (scalars).
struct Tokens {
    uint32_t word;                             // lane i: of place p0 + i
    uint32_t starts, ends, inside;
    int32_t p0;

    template <bool MAPPED>
    __device__ __forceinline__ void find(const Recur& r, int32_t first) {
        p0 = first;
        const int l = lane_id();
        word = kOutside;
        if (l < kSteps && (int64_t)first + l < r.a.n) word = MAPPED ? r.map[first + l] : place_word(r.a, first + l);
        const bool in = word != kOutside;
        inside = (uint32_t)__ballot(in);
        starts = (uint32_t)__ballot(in && (word & kStart)) | (~inside & ((1u << kSteps) - 1));
        ends = (uint32_t)__ballot(in && (word & kEnd)) | (~inside & ((1u << kSteps) - 1));
    }
    __device__ __forceinline__ int32_t segment(int i) const { return (int32_t)(__builtin_amdgcn_readlane((int)word, i) >> 2 & 0x3FFFFFFF); }
    // the token of place p0 + i; behind the last place the last one, whose values are not used
    __device__ __forceinline__ int64_t token(const gs_recur& a, int i) const {
        const int64_t p = min((int64_t)p0 + i, (int64_t)a.n - 1);
        return a.reverse ? a.n - 1 - p : p;
    }
};

// Two elements of a lane's channels at any alignment of an element, as floats;
// `there` of them.
template <typename T, bool TAIL>
struct Two {
    typedef T vec __attribute__((ext_vector_type(2)));
    typedef vec __attribute__((aligned(sizeof(T)))) loose;
    vec v;
    // row: the same for the wave, so that an address is a scalar and the lane's column
    __device__ __forceinline__ void load(const T* row, uint32_t col, int there) {
        v = vec{};
        if (there >= 2) v = *reinterpret_cast<const loose*>(row + col);
        else if (TAIL && there == 1) v[0] = row[col];
    }
    __device__ __forceinline__ float operator[](int i) const { return (float)v[i]; }
    static __device__ __forceinline__ void store(T* row, uint32_t col, int there, float a, float b) {
        vec v;
        v[0] = (T)a;
        v[1] = (T)b;
        if (there >= 2) *reinterpret_cast<loose*>(row + col) = v;
        else if (TAIL && there == 1) row[col] = v[0];
    }
};

// A gate in one register: the smaller of a and 1 - a, t / (1 + t) with t =
// exp(-|g|), with g's sign.  The other is 1 less it, so both keep their own last
// bits (1 - a of a rounded a would lose those of a small one).
__device__ __forceinline__ float gate_of(float g) {
    const float t = __expf(-fabsf(g));
    return copysignf(t * __builtin_amdgcn_rcpf(1.0f + t), g);
}
__device__ __forceinline__ void open(float gate, float& a, float& z) {
    const float small = fabsf(gate), big = 1.0f - small;
    const bool low = __float_as_int(gate) < 0;
    a = low ? small : big;
    z = low ? big : small;
}

__device__ __forceinline__ bool bit(uint32_t mask, int i) { return (mask >> i & 1u) != 0; }

// The state that a chunk's earlier waves leave, from the one in front of wave `from`.
__device__ __forceinline__ void through(const float4* maps, const uint32_t* anew, int from, int to, int lane, float* h) {
    for (int w = from; w < to; ++w) {
        const float4 m = maps[w * GS_WAVE + lane];         // A0, A1, B0, B1
        if (anew[w]) {
            h[0] = m.z;
            h[1] = m.w;
        } else {
            h[0] = fmaf(m.x, h[0], m.z);
            h[1] = fmaf(m.y, h[1], m.w);
        }
    }
}

// Segments without a token pass their states on.
__global__ void __launch_bounds__(GS_BLOCK) k_recur_empty(gs_recur a, const float* from, float* to) {
    for (int32_t s = blockIdx.x; s < a.n_seg; s += gridDim.x) {
        if (a.n > 0 && (a.cu == nullptr || start_of(a, s) < start_of(a, s + 1))) continue;
        for (int32_t c = threadIdx.x; c < a.cols; c += GS_BLOCK)
            to[(int64_t)s * a.cols + c] = from ? from[(int64_t)s * a.cols + c] : 0.0f;
    }
}

enum { kMapsOnly = 0, kWithStates = 1, kAlone = 2 };

// Forward.  PHASE kMapsOnly: writes the chunk's map; kWithStates: the outputs,
// from the state in front of the chunk; kAlone: the only chunk, without a map.
template <typename T, bool TAIL, int PHASE>
__global__ void __launch_bounds__(kWaves * GS_WAVE) k_recur(Recur r, RecurOut o) {
    __shared__ float4 maps[kWaves * GS_WAVE];
    __shared__ uint32_t anew[kWaves];
    const gs_recur& a = r.a;
    const int w = threadIdx.x / GS_WAVE, l = lane_id();
    const int chunk = blockIdx.x / r.blocks, block = blockIdx.x % r.blocks;
    const uint32_t col = block * kCols + 2 * l;
    const int there = a.cols - (int)col;
    Tokens tk;
    tk.find<PHASE != kAlone>(r, __builtin_amdgcn_readfirstlane(chunk * kChunk + w * kSteps));
    Two<T, TAIL> gs[kSteps], xs[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int64_t t = tk.token(a, i);
        gs[i].load(static_cast<const T*>(a.gate) + t * a.ld_gate, col, there);
        xs[i].load(static_cast<const T*>(a.x) + t * a.ld_x, col, there);
    }
    float h0[kSteps][2];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        h0[i][0] = h0[i][1] = 0.0f;
        if (a.initial && bit(tk.starts & tk.inside, i)) {
            Two<float, TAIL> v;
            v.load(a.initial + (int64_t)tk.segment(i) * a.cols, col, there);
            h0[i][0] = v[0];
            h0[i][1] = v[1];
        }
    }
    float A[kSteps][2], B[kSteps][2], m[2] = {1.0f, 1.0f}, h[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const bool starts = bit(tk.starts, i), in = bit(tk.inside, i);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float z;
            open(gate_of(gs[i][c]), A[i][c], z);
            const float zx = z * xs[i][c];
            B[i][c] = !in ? 0.0f : starts ? (a.initial ? fmaf(A[i][c], h0[i][c], zx) : zx) : zx;
            m[c] = starts ? 0.0f : m[c] * A[i][c];
            h[c] = starts ? B[i][c] : fmaf(A[i][c], h[c], B[i][c]);
        }
    }
    maps[w * GS_WAVE + l] = make_float4(m[0], m[1], h[0], h[1]);
    if (l == 0) anew[w] = tk.starts != 0;
    __syncthreads();
    const int64_t wide = (int64_t)r.blocks * kCols;
    if (PHASE == kMapsOnly) {
        if (w != 0) return;
        float all[2] = {0.0f, 0.0f}, mm[2] = {1.0f, 1.0f};
        bool any = false;
        through(maps, anew, 0, kWaves, l, all);
        for (int u = 0; u < kWaves; ++u) {
            const float4 v = maps[u * GS_WAVE + l];
            mm[0] *= v.x;
            mm[1] *= v.y;
            any |= anew[u] != 0;
        }
        reinterpret_cast<float4*>(r.maps)[(chunk * wide + block * kCols) / 2 + l] = make_float4(mm[0], all[0], mm[1], all[1]);
        if (block == 0 && l == 0) r.anew[chunk] = any;
        return;
    }
    h[0] = h[1] = 0.0f;
    if (PHASE == kWithStates) {
        const float2 v = reinterpret_cast<const float2*>(r.states)[(chunk * wide + block * kCols) / 2 + l];
        h[0] = v.x;
        h[1] = v.y;
    }
    through(maps, anew, 0, w, l, h);
    if (o.kept && tk.p0 % GS_RECUR_KEEP == 0 && tk.p0 < a.n)
        Two<float, TAIL>::store(o.kept + (int64_t)(tk.p0 / GS_RECUR_KEEP) * a.cols, col, there,
                                bit(tk.starts, 0) ? 0.0f : h[0], bit(tk.starts, 0) ? 0.0f : h[1]);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const bool starts = bit(tk.starts, i);
#pragma unroll
        for (int c = 0; c < 2; ++c) h[c] = starts ? B[i][c] : fmaf(A[i][c], h[c], B[i][c]);
        const bool in = bit(tk.inside, i);
        if (in || (a.fill && (int64_t)tk.p0 + i < a.n))
            Two<T, TAIL>::store(static_cast<T*>(o.y) + tk.token(a, i) * o.ld_y, col, there, h[0], h[1]);
        if (in && o.final && bit(tk.ends, i))
            Two<float, TAIL>::store(o.final + (int64_t)tk.segment(i) * a.cols, col, there, h[0], h[1]);
    }
}

// The states in front of the chunks (behind them, from the last one on, on the way back).
__global__ void __launch_bounds__(GS_WAVE) k_recur_states(Recur r, int back) {
    const int64_t wide = (int64_t)r.blocks * kCols, c = (int64_t)blockIdx.x * GS_WAVE + threadIdx.x;
    float h = 0.0f;
#pragma unroll 8
    for (int i = 0; i < r.chunks; ++i) {
        const int k = back ? r.chunks - 1 - i : i;
        const float2 v = r.maps[k * wide + c];
        r.states[k * wide + c] = h;
        h = r.anew[k] ? v.y : fmaf(v.x, h, v.y);
    }
}

// Gradient: D_t = dy_t + a_{t+1} D_{t+1} from the last token to the first (dfinal
// comes in at a segment's last one), c_t = a_t D_t passes on;
//   dx_t = (1 - a_t) D_t;  dgate_t = a_t (1 - a_t) (h_{t-1} - x_t) D_t;  dinitial = c of the first token.
// h is formed again from the states that the forward kept every GS_RECUR_KEEP
// tokens, in fp32, not read in the tokens' type.
template <typename T, bool TAIL, int PHASE>
__global__ void __launch_bounds__(kWaves * GS_WAVE) k_recur_bwd(Recur r, gs_recur_grads o) {
    __shared__ float4 maps[kWaves * GS_WAVE], back[kWaves * GS_WAVE];
    __shared__ uint32_t anew[kWaves], ended[kWaves];
    const gs_recur& a = r.a;
    const int w = threadIdx.x / GS_WAVE, l = lane_id();
    const int chunk = blockIdx.x / r.blocks, block = blockIdx.x % r.blocks;
    const uint32_t col = block * kCols + 2 * l;
    const int there = a.cols - (int)col;
    Tokens tk;
    tk.find<PHASE != kAlone>(r, __builtin_amdgcn_readfirstlane(chunk * kChunk + w * kSteps));
    Two<T, TAIL> gs[kSteps], xs[kSteps], ds[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int64_t t = tk.token(a, i);
        gs[i].load(static_cast<const T*>(a.gate) + t * a.ld_gate, col, there);
        ds[i].load(static_cast<const T*>(o.dy) + t * o.ld_dy, col, there);
        if (PHASE != kMapsOnly) xs[i].load(static_cast<const T*>(a.x) + t * a.ld_x, col, there);
    }
    // the way back through the wave's tokens: c -> m c + b
    float D[kSteps][2], S[kSteps][2], m[2] = {1.0f, 1.0f}, b[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i) {
        const bool in = bit(tk.inside, i), ends = bit(tk.ends, i);
        D[i][0] = in ? ds[i][0] : 0.0f;
        D[i][1] = in ? ds[i][1] : 0.0f;
        if (in && ends && o.dfinal) {
            Two<float, TAIL> v;
            v.load(o.dfinal + (int64_t)tk.segment(i) * a.cols, col, there);
            D[i][0] += v[0];
            D[i][1] += v[1];
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float A, z;
            S[i][c] = gate_of(gs[i][c]);
            open(S[i][c], A, z);
            if (!in) A = 0.0f;
            m[c] = ends ? 0.0f : m[c] * A;
            b[c] = A * (ends ? D[i][c] : D[i][c] + b[c]);
        }
    }
    back[(kWaves - 1 - w) * GS_WAVE + l] = make_float4(m[0], m[1], b[0], b[1]);
    if (l == 0) ended[kWaves - 1 - w] = tk.ends != 0;
    const int64_t wide = (int64_t)r.blocks * kCols;
    if (PHASE == kMapsOnly) {
        __syncthreads();
        if (w != 0) return;
        float all[2] = {0.0f, 0.0f}, mm[2] = {1.0f, 1.0f};
        bool any = false;
        through(back, ended, 0, kWaves, l, all);
        for (int u = 0; u < kWaves; ++u) {
            const float4 v = back[u * GS_WAVE + l];
            mm[0] *= v.x;
            mm[1] *= v.y;
            any |= ended[u] != 0;
        }
        reinterpret_cast<float4*>(r.maps)[(chunk * wide + block * kCols) / 2 + l] = make_float4(mm[0], all[0], mm[1], all[1]);
        if (block == 0 && l == 0) r.anew[chunk] = any;
        return;
    }
    // the states again: the wave's own map, then those of the waves behind the kept state
    float h[2] = {0.0f, 0.0f}, fm[2] = {1.0f, 1.0f};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const bool starts = bit(tk.starts, i), in = bit(tk.inside, i);
        float h0[2] = {0.0f, 0.0f};
        if (in && starts && a.initial) {
            Two<float, TAIL> v;
            v.load(a.initial + (int64_t)tk.segment(i) * a.cols, col, there);
            h0[0] = v[0];
            h0[1] = v[1];
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float A, z;
            loaded(S[i][c]);                   // opened again in each walk: held open, gates take twice the registers
            open(S[i][c], A, z);
            const float zx = in ? z * xs[i][c] : 0.0f;
            fm[c] = starts ? 0.0f : fm[c] * A;
            h[c] = !starts ? fmaf(A, h[c], zx) : in && a.initial ? fmaf(A, h0[c], zx) : zx;
        }
    }
    maps[w * GS_WAVE + l] = make_float4(fm[0], fm[1], h[0], h[1]);
    if (l == 0) anew[w] = tk.starts != 0;
    __syncthreads();
    h[0] = h[1] = 0.0f;
    if (tk.p0 < a.n) {
        Two<float, TAIL> v;
        v.load(o.kept + (int64_t)(tk.p0 / GS_RECUR_KEEP) * a.cols, col, there);
        h[0] = v[0];
        h[1] = v[1];
    }
    through(maps, anew, w / kKeptWaves * kKeptWaves, w, l, h);
    float K[kSteps][2];                        // a (1 - a) (h_{t-1} - x_t)
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const bool starts = bit(tk.starts, i), in = bit(tk.inside, i);
        if (starts) {
            h[0] = h[1] = 0.0f;
            if (in && a.initial) {
                Two<float, TAIL> v;
                v.load(a.initial + (int64_t)tk.segment(i) * a.cols, col, there);
                h[0] = v[0];
                h[1] = v[1];
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float A, z;
            loaded(S[i][c]);
            open(S[i][c], A, z);
            K[i][c] = A * z * (h[c] - xs[i][c]);
            h[c] = fmaf(A, h[c], z * xs[i][c]);
        }
    }
    float g[2] = {0.0f, 0.0f};
    if (PHASE == kWithStates) {
        const float2 v = reinterpret_cast<const float2*>(r.states)[(chunk * wide + block * kCols) / 2 + l];
        g[0] = v.x;
        g[1] = v.y;
    }
    through(back, ended, 0, kWaves - 1 - w, l, g);
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i) {
        const bool in = bit(tk.inside, i), ends = bit(tk.ends, i);
        float dx[2], dg[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float A, z;
            loaded(S[i][c]);
            open(S[i][c], A, z);
            const float d = ends ? D[i][c] : D[i][c] + g[c];
            dx[c] = in ? z * d : 0.0f;
            dg[c] = in ? K[i][c] * d : 0.0f;
            g[c] = in ? A * d : 0.0f;
        }
        if (in || (a.fill && (int64_t)tk.p0 + i < a.n)) {
            const int64_t t = tk.token(a, i);
            Two<T, TAIL>::store(static_cast<T*>(o.dx) + t * o.ld_dx, col, there, dx[0], dx[1]);
            Two<T, TAIL>::store(static_cast<T*>(o.dgate) + t * o.ld_dgate, col, there, dg[0], dg[1]);
        }
        if (in && o.dinitial && bit(tk.starts, i))
            Two<float, TAIL>::store(o.dinitial + (int64_t)tk.segment(i) * a.cols, col, there, g[0], g[1]);
    }
}

struct RecurPlan {
    int32_t chunks, blocks;
    size_t map, maps, states, anew, bytes;
};

RecurPlan recur_plan(int32_t n, int32_t cols) {
    RecurPlan p;
    p.chunks = (int32_t)div_up(n, kChunk);
    p.blocks = (int32_t)div_up(cols, kCols);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align256(bytes);
        return here;
    };
    const size_t wide = (size_t)p.chunks * p.blocks * kCols;
    const bool alone = p.chunks <= 1;
    p.map = take(alone ? 0 : (size_t)n * 4);
    p.maps = take(alone ? 0 : wide * 8);
    p.states = take(alone ? 0 : wide * 4);
    p.anew = take(alone ? 0 : (size_t)p.chunks * 4);
    p.bytes = at;
    return p;
}

Recur recur_of(const gs_recur& a, const RecurPlan& p, void* ws) {
    char* base = static_cast<char*>(ws);
    Recur r;
    r.a = a;
    r.chunks = p.chunks;
    r.blocks = p.blocks;
    const bool alone = p.chunks <= 1;
    r.map = alone ? nullptr : reinterpret_cast<uint32_t*>(base + p.map);
    r.maps = alone ? nullptr : reinterpret_cast<float2*>(base + p.maps);
    r.states = alone ? nullptr : reinterpret_cast<float*>(base + p.states);
    r.anew = alone ? nullptr : reinterpret_cast<uint32_t*>(base + p.anew);
    return r;
}

void empty_segments(const gs_recur& a, const float* from, float* to, hipStream_t st) {
    if (to && (a.n == 0 || a.cu))
        k_recur_empty<<<std::min(a.n_seg, 4096), GS_BLOCK, 0, st>>>(a, from, to);
}

template <typename T, bool TAIL>
hipError_t recur_go(const Recur& r, const RecurOut& o, hipStream_t st) {
    const uint32_t grid = (uint32_t)r.chunks * r.blocks;
    if (r.chunks == 1) {
        k_recur<T, TAIL, kAlone><<<grid, kWaves * GS_WAVE, 0, st>>>(r, o);
    } else {
        k_recur_map<<<div_up(r.a.n, GS_BLOCK), GS_BLOCK, 0, st>>>(r.a, const_cast<uint32_t*>(r.map));
        k_recur<T, TAIL, kMapsOnly><<<grid, kWaves * GS_WAVE, 0, st>>>(r, o);
        k_recur_states<<<r.blocks * (kCols / GS_WAVE), GS_WAVE, 0, st>>>(r, 0);
        k_recur<T, TAIL, kWithStates><<<grid, kWaves * GS_WAVE, 0, st>>>(r, o);
    }
    return hipGetLastError();
}

template <typename T, bool TAIL>
hipError_t recur_bwd_go(const Recur& r, const gs_recur_grads& g, hipStream_t st) {
    const uint32_t grid = (uint32_t)r.chunks * r.blocks;
    if (r.chunks == 1) {
        k_recur_bwd<T, TAIL, kAlone><<<grid, kWaves * GS_WAVE, 0, st>>>(r, g);
    } else {
        k_recur_map<<<div_up(r.a.n, GS_BLOCK), GS_BLOCK, 0, st>>>(r.a, const_cast<uint32_t*>(r.map));
        k_recur_bwd<T, TAIL, kMapsOnly><<<grid, kWaves * GS_WAVE, 0, st>>>(r, g);
        k_recur_states<<<r.blocks * (kCols / GS_WAVE), GS_WAVE, 0, st>>>(r, 1);
        k_recur_bwd<T, TAIL, kWithStates><<<grid, kWaves * GS_WAVE, 0, st>>>(r, g);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t recur_type(const Recur& r, const RecurOut& o, hipStream_t st) {
    return r.a.cols % 2 ? recur_go<T, true>(r, o, st) : recur_go<T, false>(r, o, st);
}

template <typename T>
hipError_t recur_bwd_type(const Recur& r, const gs_recur_grads& g, hipStream_t st) {
    return r.a.cols % 2 ? recur_bwd_go<T, true>(r, g, st) : recur_bwd_go<T, false>(r, g, st);
}

}  // namespace

size_t recurrence_ws_bytes(const gs_recur& a) { return recur_plan(a.n, a.cols).bytes; }

hipError_t launch_recurrence(const gs_recur& a, void* y, int64_t ld_y, float* final, float* kept, void* ws,
                             hipStream_t st) {
    empty_segments(a, a.initial, final, st);
    if (a.n == 0) return hipGetLastError();
    const RecurPlan p = recur_plan(a.n, a.cols);
    const Recur r = recur_of(a, p, ws);
    const RecurOut o = {y, final, kept, ld_y};
    if (a.dtype == GS_F32) return recur_type<float>(r, o, st);
    return a.dtype == GS_BF16 ? recur_type<bf16_t>(r, o, st) : recur_type<f16_t>(r, o, st);
}

hipError_t launch_recurrence_bwd(const gs_recur& a, const gs_recur_grads& g, void* ws, hipStream_t st) {
    empty_segments(a, g.dfinal, g.dinitial, st);
    if (a.n == 0) return hipGetLastError();
    const RecurPlan p = recur_plan(a.n, a.cols);
    const Recur r = recur_of(a, p, ws);
    if (a.dtype == GS_F32) return recur_bwd_type<float>(r, g, st);
    return a.dtype == GS_BF16 ? recur_bwd_type<bf16_t>(r, g, st) : recur_bwd_type<f16_t>(r, g, st);
}

}  // namespace gsmi
