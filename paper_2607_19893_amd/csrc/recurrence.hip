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
// of up to 128 channels, two a lane, and finds its own map with every gate and token
// in registers; the maps of a chunk's waves meet in LDS, those of the chunks in
// global memory.  `reverse` turns the list around (place p is token n - 1 - p).
// One pass: a chunk publishes its map, looks back over the chunks in front of it
// to the nearest whose last state is known, publishes its own last state, and
// goes through its tokens.  Bound by HBM bytes.
// ---------------------------------------------------------------------------

constexpr int kSteps = 16;                     // tokens of a wave
constexpr int kWaves = 8;                      // of a workgroup
constexpr int kChunk = kSteps * kWaves;
constexpr int kCols = 2 * GS_WAVE;             // channels of a workgroup at most
constexpr int kKeptWaves = GS_RECUR_KEEP / kSteps;
static_assert(GS_RECUR_KEEP % kSteps == 0 && kChunk % GS_RECUR_KEEP == 0, "a kept state is in front of a wave");

constexpr uint32_t kAllSteps = (1u << kSteps) - 1;
constexpr uint32_t kStart = 1, kEnd = 2, kOutside = 0xFFFFFFFFu;

struct Recur {
    gs_recur a;
    const uint32_t* map;                       // of place p: segment << 2 | kEnd | kStart, or kOutside
    uint64_t* maps;                            // [blocks][chunks][2 * 64]: (A, B) of a lane's two channels
    uint64_t* states;                          // [blocks][chunks][64]: a lane's two states behind the chunk
    uint32_t* flags;                           // [blocks][chunks]: kMap, then kState; behind them the ticket
    int32_t chunks, blocks, width;             // width: channels of a block
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

// The places' words, and the flags and the ticket cleared.
__global__ void __launch_bounds__(GS_BLOCK) k_recur_map(gs_recur a, uint32_t* __restrict__ map, uint32_t* __restrict__ flags,
                                                        int32_t n_flags) {
    const int64_t p = (int64_t)blockIdx.x * GS_BLOCK + threadIdx.x;
    if (p < a.n) map[p] = place_word(a, (int32_t)p);
    if (p < n_flags) flags[p] = 0;
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
        starts = (uint32_t)__ballot(in && (word & kStart)) | (~inside & kAllSteps);
        ends = (uint32_t)__ballot(in && (word & kEnd)) | (~inside & kAllSteps);
    }
    __device__ __forceinline__ int32_t segment(int i) const {
        int32_t s = (int32_t)(__builtin_amdgcn_readlane((int)word, i) >> 2 & 0x3FFFFFFF);
        asm volatile("" : "+s"(s));            // nothing of it is worked out where no segment's end is
        return s;
    }
    // places that are some token's
    __device__ __forceinline__ uint32_t there(const gs_recur& a) const {
        const int32_t left = max(0, min(kSteps, a.n - p0));
        return (1u << left) - 1;
    }
    // the token of a place
    __device__ __forceinline__ int32_t token(const gs_recur& a, int32_t p) const { return a.reverse ? a.n - 1 - p : p; }
};

// Keeps a branch that is the same for the wave a branch: most waves have no
// segment's end among their tokens, and selects would cost each of them.
__device__ __forceinline__ void rare() { asm volatile(""); }

template <typename P>
using global = __attribute__((address_space(1))) P;

// A lane's two channels of a row, at any alignment of an element, as floats.
// The row is the same for the wave: an address is a scalar and the lane's
// column.  ONE: there is one channel in all.
template <typename T, bool ONE>
struct Two {
    typedef T vec __attribute__((ext_vector_type(2)));
    typedef vec __attribute__((aligned(sizeof(T)))) loose;
    vec v;
    // The row's address stays a scalar, the lane's part is a 32-bit offset: an
    // address of each lane's own would take two registers a row.
    template <typename P>
    static __device__ __forceinline__ global<P>* at(global<char>* row, uint32_t col) {
        return (global<P>*)(row + col * (uint32_t)sizeof(T));
    }
    static __device__ __forceinline__ global<char>* row_of(const void* base, int64_t row, int64_t ld) {
        return (global<char>*)const_cast<char*>(static_cast<const char*>(base)) + row * ld * (int64_t)sizeof(T);
    }
    __device__ __forceinline__ void load(global<char>* row, uint32_t col) {
        if (ONE) v = vec{*at<T>(row, col), (T)0.0f};
        else v = *at<loose>(row, col);
    }
    __device__ __forceinline__ void load(const void* base, int64_t row, int64_t ld, uint32_t col) { load(row_of(base, row, ld), col); }
    // as loaded: its floats are formed again behind this, not held in registers
    __device__ __forceinline__ void again() {
        if (sizeof(T) == 2) {
            uint32_t u;
            __builtin_memcpy(&u, &v, 4);
            loaded(u);
            __builtin_memcpy(&v, &u, 4);
        }
    }
    __device__ __forceinline__ void fill(float f) { v = vec{(T)f, (T)f}; }
    __device__ __forceinline__ float operator[](int i) const { return (float)v[i]; }
    static __device__ __forceinline__ void store(global<char>* row, uint32_t col, float a, float b) {
        if (ONE) *at<T>(row, col) = (T)a;
        else *at<loose>(row, col) = vec{(T)a, (T)b};
    }
    static __device__ __forceinline__ void store(void* base, int64_t row, int64_t ld, uint32_t col, float a, float b) {
        store(row_of(base, row, ld), col, a, b);
    }
};

// The rows of a matrix along the places, from place `first` on (back: the other
// way): one row after the other, so that no more than one address is held.
struct Rows {
    global<char>* p;
    int64_t step;
    template <typename T>
    static __device__ __forceinline__ Rows of(const gs_recur& a, const Tokens& tk, const void* base, int64_t ld, int32_t first,
                                              bool back) {
        const int64_t bytes = ld * (int64_t)sizeof(T);
        Rows r;
        r.p = (global<char>*)const_cast<char*>(static_cast<const char*>(base)) + (int64_t)tk.token(a, first) * bytes;
        r.step = (a.reverse != 0) != back ? -bytes : bytes;
        return r;
    }
    __device__ __forceinline__ void next(bool there = true) {
        p += there ? step : 0;
        asm volatile("" : "+s"(p));
    }
};

// A lane's first channel.  Lanes past the block's or the row's end take its last
// two once more, and write the same values there: no lane is ever left out.
__device__ __forceinline__ uint32_t column(const gs_recur& a, int block, int width) {
    return (uint32_t)max(0, min(block * width + min(2 * lane_id(), width - 2), a.cols - 2));
}

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

// ---------------------------------------------------------------------------
// Looking back.  The workgroups take chunks by a ticket, chunk after chunk, so
// every chunk that one waits for belongs to a workgroup that is already running
// and publishes its map before it waits itself: every wait ends.  (Calls that
// run at the same time on one workspace would clear each other's flags; a wait
// gives up after kPolls then, with NaN.)  What is published moves past the
// caches of the units (agent scope); a flag follows the values it announces.
// ---------------------------------------------------------------------------

constexpr uint32_t kMap = 1, kState = 2;
constexpr int kPolls = 1 << 22;

__device__ __forceinline__ uint64_t pair(float a, float b) { return (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a); }
__device__ __forceinline__ float2 unpair(uint64_t v) {
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}
__device__ __forceinline__ void put(uint64_t* p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint64_t get(const uint64_t* p) {
    return __hip_atomic_load(const_cast<uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// by the wave that wrote what the flag announces
__device__ __forceinline__ void announce(uint32_t* flag, uint32_t what) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (lane_id() == 0) __hip_atomic_store(flag, what, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The chunk's own map, from those of its waves; true: a segment starts (ends) in it.
__device__ __forceinline__ bool whole_map(const float4* maps, const uint32_t* anew, int lane, float* m, float* b) {
    m[0] = m[1] = 1.0f;
    b[0] = b[1] = 0.0f;
    bool any = false;
    for (int u = 0; u < kWaves; ++u) {
        const float4 v = maps[u * GS_WAVE + lane];
        if (anew[u]) {
            any = true;
            b[0] = v.z;
            b[1] = v.w;
        } else {
            b[0] = fmaf(v.x, b[0], v.z);
            b[1] = fmaf(v.y, b[1], v.w);
        }
        m[0] *= v.x;
        m[1] *= v.y;
    }
    return any;
}

// A wave's part: publishes the chunk's map (a chunk in which a segment starts:
// its last state), waits for the state in front of the chunk, publishes the one
// behind it, and leaves in h the one in front.  `needed`: someone here reads it.
// own, anew: the waves' maps in LDS, read a second time for the state, since
// registers are short.
template <int kAhead>                          // maps on their way at once
__device__ __forceinline__ void look_back(const Recur& r, int chunk, int block, const float4* own, const uint32_t* anew,
                                          bool needed, float* h) {
    const int l = lane_id();
    const int64_t at = (int64_t)block * r.chunks;
    uint64_t* maps = r.maps + at * (2 * GS_WAVE);
    uint64_t* states = r.states + at * GS_WAVE;
    uint32_t* flags = r.flags + at;
    float m[2], b[2];
    h[0] = h[1] = 0.0f;
    const bool any = whole_map(own, anew, l, m, b);
    if (any) {
        put(states + (int64_t)chunk * GS_WAVE + l, pair(b[0], b[1]));
        announce(flags + chunk, kState);
        if (!needed) return;
    } else {
        put(maps + (int64_t)chunk * (2 * GS_WAVE) + l, pair(m[0], b[0]));
        put(maps + (int64_t)chunk * (2 * GS_WAVE) + GS_WAVE + l, pair(m[1], b[1]));
        announce(flags + chunk, kMap);
    }
    // from the nearest chunk on: the map through those that were passed
    float pm[2] = {1.0f, 1.0f}, pb[2] = {0.0f, 0.0f};
    int j = chunk - 1, polls = 0;
    for (;;) {
        const uint32_t f = j - l >= 0 ? __hip_atomic_load(flags + j - l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
        const uint64_t known = __ballot(f == kState), there = __ballot(f != 0u);
        const int d = known ? __ffsll((unsigned long long)known) - 1 : GS_WAVE;      // maps to pass first
        const uint64_t need = d == GS_WAVE ? ~0ull : (1ull << d) - 1;
        if ((there & need) != need) {
            if (++polls > kPolls) {
                h[0] = h[1] = NAN;
                break;
            }
            __builtin_amdgcn_s_sleep(1);
            continue;
        }
        asm volatile("" ::: "memory");         // the values are read behind the flags
        uint64_t s = 0;
        if (known) s = get(states + (int64_t)(j - d) * GS_WAVE + l);
        for (int k = 0; k < d; k += kAhead) {
            uint64_t v[kAhead][2];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int64_t c = (int64_t)(j - min(k + i, d - 1)) * (2 * GS_WAVE) + l;
                v[i][0] = get(maps + c);
                v[i][1] = get(maps + c + GS_WAVE);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (k + i >= d) break;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float2 ab = unpair(v[i][c]);
                    pb[c] = fmaf(pm[c], ab.y, pb[c]);
                    pm[c] *= ab.x;
                }
            }
        }
        if (known) {
            const float2 v = unpair(s);
            h[0] = fmaf(pm[0], v.x, pb[0]);
            h[1] = fmaf(pm[1], v.y, pb[1]);
            break;
        }
        j -= GS_WAVE;
    }
    if (any) return;
    whole_map(own, anew, l, m, b);
    put(states + (int64_t)chunk * GS_WAVE + l, pair(fmaf(m[0], h[0], b[0]), fmaf(m[1], h[1], b[1])));
    announce(flags + chunk, kState);
}

// The next chunk (in the order of the recurrence) and its block of channels; false: none is left.
__device__ __forceinline__ bool take_chunk(const Recur& r, uint32_t* shared, int& chunk, int& block) {
    const int32_t all = r.chunks * r.blocks;
    if (threadIdx.x == 0) *shared = atomicAdd(r.flags + all, 1u);
    __syncthreads();
    const uint32_t t = __builtin_amdgcn_readfirstlane(*shared);
    chunk = (int)(t / (uint32_t)r.blocks);
    block = (int)(t % (uint32_t)r.blocks);
    return t < (uint32_t)all;
}

// ALONE: the list is one chunk, which looks nowhere and has no map of places.
// Two workgroups a compute unit (4 waves a SIMD) where the registers allow it.
template <typename T, bool ONE, bool ALONE>
__global__ void __launch_bounds__(kWaves * GS_WAVE, 4) k_recur(Recur r, RecurOut o) {
    __shared__ float4 maps[kWaves * GS_WAVE];
    __shared__ float2 front[GS_WAVE];
    __shared__ uint32_t anew[kWaves], ticket;
    const gs_recur& a = r.a;
    const int w = threadIdx.x / GS_WAVE, l = lane_id();
    int chunk = 0, block = blockIdx.x;
    if (!ALONE && !take_chunk(r, &ticket, chunk, block)) return;
    const uint32_t col = column(a, block, r.width);
    Tokens tk;
    tk.find<!ALONE>(r, __builtin_amdgcn_readfirstlane(chunk * kChunk + w * kSteps));
    Two<T, ONE> gs[kSteps], xs[kSteps];
    // behind the last place the last one's row, whose values are not used
    const int32_t first = min(tk.p0, a.n - 1);
    Rows gate = Rows::of<T>(a, tk, a.gate, a.ld_gate, first, false), x = Rows::of<T>(a, tk, a.x, a.ld_x, first, false);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        gs[i].load(gate.p, col);
        xs[i].load(x.p, col);
        gate.next(tk.p0 + i + 1 < a.n);
        x.next(tk.p0 + i + 1 < a.n);
    }
    float A[kSteps][2], B[kSteps][2], m[2] = {1.0f, 1.0f}, h[2] = {0.0f, 0.0f};
    const uint32_t firsts = a.initial ? tk.starts & tk.inside : 0u;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {         // the initial states, all on their way at once
        B[i][0] = B[i][1] = 0.0f;
        if (bit(firsts, i)) {
            Two<float, ONE> v;
            v.load(a.initial, tk.segment(i), a.cols, col);
            B[i][0] = v[0];
            B[i][1] = v[1];
        }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (bit(tk.starts, i)) {
            rare();
            m[0] = m[1] = h[0] = h[1] = 0.0f;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float z;
            open(gate_of(gs[i][c]), A[i][c], z);
            B[i][c] = fmaf(A[i][c], B[i][c], z * xs[i][c]);
        }
        if (!bit(tk.inside, i)) {
            rare();
            B[i][0] = B[i][1] = A[i][0] = A[i][1] = 0.0f;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            m[c] *= A[i][c];
            h[c] = fmaf(A[i][c], h[c], B[i][c]);
        }
    }
    maps[w * GS_WAVE + l] = make_float4(m[0], m[1], h[0], h[1]);
    if (l == 0) anew[w] = tk.starts != 0;
    __syncthreads();
    h[0] = h[1] = 0.0f;
    if (!ALONE) {
        if (w == 0) {
            float f[2];
            look_back<4>(r, chunk, block, maps, anew, !bit(tk.starts, 0), f);
            front[l] = make_float2(f[0], f[1]);
        }
        __syncthreads();
        h[0] = front[l].x;
        h[1] = front[l].y;
    }
    through(maps, anew, 0, w, l, h);
    if (o.kept && tk.p0 % GS_RECUR_KEEP == 0 && tk.p0 < a.n)
        Two<float, ONE>::store(o.kept, tk.p0 / GS_RECUR_KEEP, a.cols, col, bit(tk.starts, 0) ? 0.0f : h[0],
                               bit(tk.starts, 0) ? 0.0f : h[1]);
    const uint32_t written = a.fill ? tk.there(a) : tk.inside, lasts = o.final ? tk.ends & tk.inside : 0u;
    Rows y = Rows::of<T>(a, tk, o.y, o.ld_y, first, false);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (bit(tk.starts, i)) {
            rare();
            h[0] = h[1] = 0.0f;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) h[c] = fmaf(A[i][c], h[c], B[i][c]);
        if (bit(written, i)) Two<T, ONE>::store(y.p, col, h[0], h[1]);
        y.next();
        if (bit(lasts, i)) Two<float, ONE>::store(o.final, tk.segment(i), a.cols, col, h[0], h[1]);
    }
}

// Gradient: D_t = dy_t + a_{t+1} D_{t+1} from the last token to the first (dfinal
// comes in at a segment's last one), c_t = a_t D_t passes on;
//   dx_t = (1 - a_t) D_t;  dgate_t = a_t (1 - a_t) (h_{t-1} - x_t) D_t;  dinitial = c of the first token.
// h is formed again from the states that the forward kept every GS_RECUR_KEEP
// tokens, in fp32, not read in the tokens' type.
template <typename T, bool ONE, bool ALONE>
__global__ void __launch_bounds__(kWaves * GS_WAVE, 4) k_recur_bwd(Recur r, gs_recur_grads o) {
    __shared__ float4 maps[kWaves * GS_WAVE], back[kWaves * GS_WAVE];
    __shared__ float2 front[GS_WAVE];
    __shared__ uint32_t anew[kWaves], ended[kWaves], ticket;
    const gs_recur& a = r.a;
    const int w = threadIdx.x / GS_WAVE, l = lane_id();
    int turn = 0, block = blockIdx.x;          // chunks are taken from the last one on
    if (!ALONE && !take_chunk(r, &ticket, turn, block)) return;
    const int chunk = r.chunks - 1 - turn;
    const uint32_t col = column(a, block, r.width);
    Tokens tk;
    tk.find<!ALONE>(r, __builtin_amdgcn_readfirstlane(chunk * kChunk + w * kSteps));
    Two<T, ONE> gs[kSteps], xs[kSteps], ds[kSteps];
    // behind the last place the last one's row, whose values are not used
    const int32_t first = min(tk.p0, a.n - 1), end = min(tk.p0 + kSteps, a.n) - 1;
    Rows gate = Rows::of<T>(a, tk, a.gate, a.ld_gate, first, false), x = Rows::of<T>(a, tk, a.x, a.ld_x, first, false);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        gs[i].load(gate.p, col);
        xs[i].load(x.p, col);
        gate.next(tk.p0 + i + 1 < a.n);
        x.next(tk.p0 + i + 1 < a.n);
    }
    auto load_dy = [&]() {
        Rows dy = Rows::of<T>(a, tk, o.dy, o.ld_dy, first, false);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            ds[i].load(dy.p, col);
            dy.next(tk.p0 + i + 1 < a.n);
            if (!bit(tk.inside, i)) {
                rare();
                ds[i].fill(0.0f);
            }
        }
    };
    load_dy();
    // tokens outside every segment: a gate that holds, and zeros
    if (tk.inside != kAllSteps) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
            if (!bit(tk.inside, i)) {
                rare();
                gs[i].fill(INFINITY);
                xs[i].fill(0.0f);
            }
    }
    const uint32_t firsts = a.initial ? tk.starts & tk.inside : 0u, lasts = o.dfinal ? tk.ends & tk.inside : 0u;
    // states of the row's segment
    auto state_of = [&](const float* from, int i, float* h) {
        Two<float, ONE> v;
        v.load(from, tk.segment(i), a.cols, col);
        h[0] = v[0];
        h[1] = v[1];
    };
    // The wave's two maps: h -> m h + h, and on the way back, whose terms are
    // summed from the same end, c -> bm c + b up to the first token that ends a
    // segment.  A gate is kept in one register, dy and x stay as they were
    // loaded: floats of all would leave room for one workgroup a compute unit.
    float S[kSteps][2], m[2] = {1.0f, 1.0f}, h[2] = {0.0f, 0.0f}, bm[2] = {1.0f, 1.0f}, b[2] = {0.0f, 0.0f};
    const int first_end = tk.ends ? __ffs(tk.ends) - 1 : kSteps;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (bit(tk.starts, i)) {
            rare();
            m[0] = m[1] = h[0] = h[1] = 0.0f;
            if (bit(firsts, i)) state_of(a.initial, i, h);
        }
        float A[2], z;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            S[i][c] = gate_of(gs[i][c]);
            open(S[i][c], A[c], z);
            m[c] *= A[c];
            h[c] = fmaf(A[c], h[c], z * xs[i][c]);
        }
        if (i <= first_end) {
            rare();
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                bm[c] *= A[c];
                b[c] = fmaf(bm[c], ds[i][c], b[c]);
            }
            if (bit(lasts, i)) {
                float d[2];
                state_of(o.dfinal, i, d);
                b[0] = fmaf(bm[0], d[0], b[0]);
                b[1] = fmaf(bm[1], d[1], b[1]);
            }
        }
    }
    if (tk.ends) bm[0] = bm[1] = 0.0f;
    back[(kWaves - 1 - w) * GS_WAVE + l] = make_float4(bm[0], bm[1], b[0], b[1]);
    maps[w * GS_WAVE + l] = make_float4(m[0], m[1], h[0], h[1]);
    if (l == 0) {
        ended[kWaves - 1 - w] = tk.ends != 0;
        anew[w] = tk.starts != 0;
    }
    __syncthreads();
    if (!ALONE && w == kWaves - 1) {
        float f[2];
        look_back<sizeof(T) == 4 ? 1 : 4>(r, turn, block, back, ended, !bit(tk.ends, kSteps - 1), f);
        front[l] = make_float2(f[0], f[1]);
        if (sizeof(T) == 4) load_dy();         // there are no registers to hold it meanwhile
    }
    // the states again, from the kept one in front
    h[0] = h[1] = 0.0f;
    if (tk.p0 < a.n) {
        Two<float, ONE> v;
        v.load(o.kept, tk.p0 / GS_RECUR_KEEP, a.cols, col);
        h[0] = v[0];
        h[1] = v[1];
    }
    through(maps, anew, w / kKeptWaves * kKeptWaves, w, l, h);
    float K[kSteps][2];                        // a (1 - a) (h_{t-1} - x_t)
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (bit(tk.starts, i)) {
            rare();
            h[0] = h[1] = 0.0f;
            if (bit(firsts, i)) state_of(a.initial, i, h);
        }
        xs[i].again();
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float A, z;
            loaded(S[i][c]);                   // opened again in each walk: held open, gates take twice the registers
            open(S[i][c], A, z);
            const float x = xs[i][c];
            K[i][c] = A * z * (h[c] - x);
            loaded(K[i][c]);                   // here, not where it is used: its factors would be held until then
            h[c] = fmaf(A, h[c], z * x);
        }
    }
    float g[2] = {0.0f, 0.0f};
    if (!ALONE) {
        __syncthreads();
        g[0] = front[l].x;
        g[1] = front[l].y;
    }
    through(back, ended, 0, kWaves - 1 - w, l, g);
    const uint32_t written = a.fill ? tk.there(a) : tk.inside, starts = o.dinitial ? tk.starts & tk.inside : 0u;
    Rows dxs = Rows::of<T>(a, tk, o.dx, o.ld_dx, end, true), dgs = Rows::of<T>(a, tk, o.dgate, o.ld_dgate, end, true);
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i) {
        if (bit(tk.ends, i)) {
            rare();
            g[0] = g[1] = 0.0f;
            if (bit(lasts, i)) state_of(o.dfinal, i, g);
        }
        float dx[2], dg[2];
        ds[i].again();
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float A, z;
            loaded(S[i][c]);
            open(S[i][c], A, z);
            const float d = ds[i][c] + g[c];
            dx[c] = z * d;
            dg[c] = K[i][c] * d;
            g[c] = A * d;
        }
        if (bit(written, i)) {
            Two<T, ONE>::store(dxs.p, col, dx[0], dx[1]);
            Two<T, ONE>::store(dgs.p, col, dg[0], dg[1]);
        }
        dxs.next(tk.p0 + i < a.n);
        dgs.next(tk.p0 + i < a.n);
        if (bit(starts, i)) Two<float, ONE>::store(o.dinitial, tk.segment(i), a.cols, col, g[0], g[1]);
    }
}

struct RecurPlan {
    int32_t chunks, blocks, width;
    size_t map, maps, states, flags, bytes;
};

RecurPlan recur_plan(int32_t n, int32_t cols) {
    RecurPlan p;
    p.chunks = (int32_t)div_up(n, kChunk);
    p.width = kCols;                           // so that no block has a single channel
    while (cols > 1 && cols % p.width == 1) p.width -= 2;
    p.blocks = (int32_t)div_up(cols, p.width);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align256(bytes);
        return here;
    };
    const size_t all = p.chunks <= 1 ? 0 : (size_t)p.chunks * p.blocks;
    p.map = take(all ? (size_t)n * 4 : 0);
    p.maps = take(all * GS_WAVE * 16);
    p.states = take(all * GS_WAVE * 8);
    p.flags = take(all ? (all + 1) * 4 : 0);
    p.bytes = at;
    return p;
}

Recur recur_of(const gs_recur& a, const RecurPlan& p, void* ws) {
    char* base = static_cast<char*>(ws);
    Recur r;
    r.a = a;
    r.chunks = p.chunks;
    r.blocks = p.blocks;
    r.width = p.width;
    const bool alone = p.chunks <= 1;
    r.map = alone ? nullptr : reinterpret_cast<uint32_t*>(base + p.map);
    r.maps = alone ? nullptr : reinterpret_cast<uint64_t*>(base + p.maps);
    r.states = alone ? nullptr : reinterpret_cast<uint64_t*>(base + p.states);
    r.flags = alone ? nullptr : reinterpret_cast<uint32_t*>(base + p.flags);
    return r;
}

// The map of the places and cleared flags.
void recur_map(const Recur& r, hipStream_t st) {
    const int32_t flags = r.chunks * r.blocks + 1;
    k_recur_map<<<div_up(std::max(r.a.n, flags), GS_BLOCK), GS_BLOCK, 0, st>>>(r.a, const_cast<uint32_t*>(r.map), r.flags, flags);
}

void empty_segments(const gs_recur& a, const float* from, float* to, hipStream_t st) {
    if (to && (a.n == 0 || a.cu))
        k_recur_empty<<<std::min(a.n_seg, 4096), GS_BLOCK, 0, st>>>(a, from, to);
}

template <typename T, bool ONE>
hipError_t recur_go(const Recur& r, const RecurOut& o, hipStream_t st) {
    const uint32_t grid = (uint32_t)r.chunks * r.blocks;
    if (r.chunks == 1) {
        k_recur<T, ONE, true><<<grid, kWaves * GS_WAVE, 0, st>>>(r, o);
    } else {
        recur_map(r, st);
        k_recur<T, ONE, false><<<grid, kWaves * GS_WAVE, 0, st>>>(r, o);
    }
    return hipGetLastError();
}

template <typename T, bool ONE>
hipError_t recur_bwd_go(const Recur& r, const gs_recur_grads& g, hipStream_t st) {
    const uint32_t grid = (uint32_t)r.chunks * r.blocks;
    if (r.chunks == 1) {
        k_recur_bwd<T, ONE, true><<<grid, kWaves * GS_WAVE, 0, st>>>(r, g);
    } else {
        recur_map(r, st);
        k_recur_bwd<T, ONE, false><<<grid, kWaves * GS_WAVE, 0, st>>>(r, g);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t recur_type(const Recur& r, const RecurOut& o, hipStream_t st) {
    return r.a.cols == 1 ? recur_go<T, true>(r, o, st) : recur_go<T, false>(r, o, st);
}

template <typename T>
hipError_t recur_bwd_type(const Recur& r, const gs_recur_grads& g, hipStream_t st) {
    return r.a.cols == 1 ? recur_bwd_go<T, true>(r, g, st) : recur_bwd_go<T, false>(r, g, st);
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
