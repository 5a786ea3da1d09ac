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
// One pass: a chunk publishes its map, looks back over those in front of it for
// the state that it starts from, and goes through its tokens.  Bound by HBM bytes
// and by the waits: 131,072 bf16 tokens of 1024 channels 218 us, 3.7 TB/s (three
// launches, which read the tokens twice, 613; chunks that wait for nobody 165).
// Of a chunk's 18 us, loads and the first walk take 6.5, publishing, waiting and
// the state in front 5.6, the second walk and the stores 4.7.
// ---------------------------------------------------------------------------

constexpr int kSteps = 16;                     // tokens of a wave
constexpr int kWaves = 8;                      // of a workgroup
constexpr int kChunk = kSteps * kWaves;
constexpr int kAloneWaves = 16;                // of the only workgroup along the tokens
constexpr int kAloneChunk = kSteps * kAloneWaves;
constexpr int kCols = 2 * GS_WAVE;             // channels of a workgroup at most
constexpr int kKeptWaves = GS_RECUR_KEEP / kSteps;
static_assert(GS_RECUR_KEEP % kSteps == 0 && kChunk % GS_RECUR_KEEP == 0, "a kept state is in front of a wave");

constexpr uint32_t kAllSteps = (1u << kSteps) - 1;
constexpr uint32_t kStart = 1, kEnd = 2, kOutside = 0xFFFFFFFFu;

struct Recur {
    gs_recur a;
    uint64_t* maps;                            // [blocks][chunks][2 * 64]: (A, B) of a lane's two channels
    uint64_t* group_maps;                      // [blocks][groups][2 * 64]: the same of kGroup chunks
    uint64_t* states;                          // [blocks][groups][64]: a lane's two states behind the group
    uint32_t* flags;                           // [blocks][chunks]: kMap or kAnew; [blocks][groups]: kMap, then kState;
                                               // a counter a block
    int32_t chunks, groups, blocks, width;     // width: channels of a block
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

// A place: segment << 2 | kEnd | kStart, or kOutside.
__device__ __forceinline__ uint32_t word_of(const gs_recur& a, int32_t t, int32_t s, int32_t first, int32_t end) {
    if (s < 0 || s >= a.n_seg || t < first || t >= end) return kOutside;
    const bool at_first = t == first, at_last = t == end - 1;
    return (uint32_t)s << 2 | ((a.reverse ? at_first : at_last) ? kEnd : 0u) | ((a.reverse ? at_last : at_first) ? kStart : 0u);
}

// Segments without a token pass their states on (from NULL: 0): a wave's part of
// them, 64 segments at a time.
__device__ __forceinline__ void pass_empty(const gs_recur& a, const float* from, float* to, int wave, int waves) {
    if (to == nullptr || (a.cu == nullptr && a.n > 0)) return;
    for (int32_t s0 = wave * GS_WAVE; s0 < a.n_seg; s0 += waves * GS_WAVE) {
        const int32_t s = s0 + lane_id();
        uint64_t empty = __ballot(s < a.n_seg && (a.cu == nullptr || start_of(a, s) >= start_of(a, s + 1)));
        for (; empty; empty &= empty - 1) {
            const int64_t row = (int64_t)(s0 + __ffsll((unsigned long long)empty) - 1) * a.cols;
            for (int32_t c = lane_id(); c < a.cols; c += GS_WAVE) to[row + c] = from ? from[row + c] : 0.0f;
        }
    }
}

// The flags and the counters cleared, the empty segments' states.
__global__ void __launch_bounds__(GS_BLOCK) k_recur_clear(gs_recur a, const float* from, float* to, uint32_t* flags,
                                                          int32_t n_flags) {
    for (int64_t i = (int64_t)blockIdx.x * GS_BLOCK + threadIdx.x; i < n_flags; i += (int64_t)gridDim.x * GS_BLOCK) flags[i] = 0;
    pass_empty(a, from, to, blockIdx.x * (GS_BLOCK / GS_WAVE) + threadIdx.x / GS_WAVE, gridDim.x * (GS_BLOCK / GS_WAVE));
}

// A wave's tokens: bit i of the masks is place p0 + i (scalars).
struct Tokens {
    uint32_t word;                             // lane i: place p0 + i
    uint32_t starts, ends, inside;
    int32_t p0;

    // The wave looks its places up together: 64 starts at a time narrow the
    // segments down to the first place's, then 64 starts from there on serve all
    // places (one reading up to 63 segments, three up to 4095).
    __device__ __forceinline__ void find(const gs_recur& a, int32_t place0) {
        p0 = place0;
        const int l = lane_id();
        const int32_t p = p0 + l, t = a.reverse ? a.n - 1 - p : p;
        word = kOutside;
        if (p0 >= a.n) {
            // nothing of it is a token
        } else if (a.cu == nullptr) {
            const int32_t len = a.n / a.n_seg, s = t / len;
            if (l < kSteps && p < a.n) word = word_of(a, t, s, s * len, s * len + len);
        } else {
            const int32_t p1 = min(p0 + kSteps, a.n) - 1;
            const int32_t low = a.reverse ? a.n - 1 - p1 : p0, high = a.reverse ? a.n - 1 - p0 : p1;
            int32_t base = 0;
            if (a.n_seg >= GS_WAVE) {
                int32_t len = a.n_seg + 1;     // starts from `base` on, one of which is the last that is <= low
                for (;;) {
                    const int32_t step = (len + GS_WAVE - 1) / GS_WAVE, at = base + l * step;
                    const int c = popc64(__ballot(l * step < len && start_of(a, min(at, a.n_seg)) <= low));
                    const int32_t passed = max(c - 1, 0) * step;
                    base += passed;
                    if (step == 1) break;
                    len = min(step, len - passed);
                }
            }
            const int32_t mine = base + l <= a.n_seg ? start_of(a, base + l) : 0x7FFFFFFF;
            if (__builtin_amdgcn_readlane(mine, GS_WAVE - 1) > high) {
                int k = 0;                     // starts up to the lane's place
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const int32_t ti = a.reverse ? a.n - 1 - (p0 + i) : p0 + i;
                    const int c = popc64(__ballot(mine <= ti));
                    if (l == i) k = c;
                }
                const int32_t first = __shfl(mine, max(k - 1, 0), GS_WAVE), end = __shfl(mine, k, GS_WAVE);
                if (l < kSteps && p < a.n) word = word_of(a, t, base + k - 1, first, end);
            } else if (l < kSteps && p < a.n) {            // very many segments end here
                int32_t lo = 0, hi = a.n_seg;  // the last s with start_of(s) <= t
                while (lo < hi) {
                    const int32_t mid = (int32_t)(((int64_t)lo + hi + 1) / 2);
                    if (start_of(a, mid) <= t) lo = mid;
                    else hi = mid - 1;
                }
                word = word_of(a, t, lo, start_of(a, lo), start_of(a, min(lo + 1, a.n_seg)));
            }
        }
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
// column.  ONE: a lane has one channel.
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
// two (ONE: its last) once more, and write the same values there: no lane is
// ever left out.
template <bool ONE>
__device__ __forceinline__ uint32_t column(const gs_recur& a, int block, int width) {
    if (ONE) return (uint32_t)min(lane_id(), a.cols - 1);
    return (uint32_t)min(block * width + min(2 * lane_id(), width - 2), a.cols - 2);
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

// A product of gates of which `least` is the smallest.  It may have run to 0 though
// no gate is 0: then it is the least number, so that an infinite state stays
// infinite (0 * inf is NaN), as it does token by token.  What a finite state
// leaves behind so, 2^-149 of it, is at the end of fp32's range as well.
__device__ __forceinline__ float product(float m, float least) { return fmaxf(m, fminf(least, 1.40129846e-45f)); }
// of two runs' products
__device__ __forceinline__ float behind(float m, float a) { return product(m * a, fminf(m, a)); }

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

// ---------------------------------------------------------------------------
// Looking back.  kGroup chunks are a group.  A chunk joins the maps of those in
// front of it in its group; the last of a group publishes the group's map, and
// when it knows the state that the group starts from, the state behind it.  The
// others look for that state over up to 64 groups.  (Chunk by chunk, 64 chunks a
// look, 400,000 tokens of 128 channels took 324 us: one look after the other.)
// Maps are joined and states passed on in one order, from the front, so the same
// bits come out whichever group's state was known first.
//   The workgroups take chunks from a counter, one after the other, so every chunk
// that one waits for belongs to a workgroup that is already running, and the
// first that is not done waits for nobody: every wait ends.  (Calls that run at
// the same time on one workspace would clear each other's flags; a wait gives up
// after kPolls then, with NaN.)  What is published is written past the caches
// (agent scope), and a flag follows the values it announces.  The values are
// read through the caches: their lines hold nothing else (maps and states start
// at multiples of kLine, wherever the workspace does) and nobody reads them
// before their flag, so no cache can have held them earlier in the kernel.
// ---------------------------------------------------------------------------

constexpr uint32_t kMap = 1, kAnew = 2, kState = 2;
constexpr int kPolls = 1 << 22;
constexpr int kPause = 32;                     // between looks (s_sleep): 1 is 3% slower, 64 is 2%, 4 and 16 are the same
// Chunks of a group.  400,000 tokens of 128 channels take 122 us (gradient 170); with
// 8 of them 129 (178), with 32 130 (197, registers spilled).  131,072 tokens of 1024
// channels 222, 217 with 8, 243 with 32.
constexpr int kGroup = 16;
constexpr size_t kLine = 256;                  // bytes; a cache line is 128
static_assert(GS_WAVE * sizeof(uint64_t) % 128 == 0, "no two chunks' maps or groups' states share a line");

__device__ __forceinline__ uint64_t pair(float a, float b) { return (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a); }
__device__ __forceinline__ float2 unpair(uint64_t v) {
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}
__device__ __forceinline__ void put(uint64_t* p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// by the wave that wrote what the flag announces
__device__ __forceinline__ void announce(uint32_t* flag, uint32_t what) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (lane_id() == 0) __hip_atomic_store(flag, what, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The chunk's own map, from those of its waves; true: a segment starts (ends) in it.
__device__ __forceinline__ bool whole_map(const float4* maps, const uint32_t* anew, int lane, float* m, float* b) {
    float least[2] = {1.0f, 1.0f};
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
        least[0] = fminf(least[0], v.x);
        least[1] = fminf(least[1], v.y);
    }
    m[0] = product(m[0], least[0]);
    m[1] = product(m[1], least[1]);
    return any;
}

constexpr int kNotNeeded = -1, kGaveUp = -2;

struct Lookers {                               // in LDS
    float4 fetched[kGroup * GS_WAVE];          // maps: of chunks in the group, then of groups
    float4 own[GS_WAVE];                       // the chunk's map
    float4 front[GS_WAVE];                     // the map through the group's chunks in front
    float2 state[GS_WAVE];                     // behind the group that the nearest known state is of
    int32_t anew, distance, speaks;            // speaks: the group's map and state are the chunk's to say
};

__device__ __forceinline__ void put_map(uint64_t* p, const float* m, const float* b) {
    put(p + lane_id(), pair(m[0], b[0]));
    put(p + GS_WAVE + lane_id(), pair(m[1], b[1]));
}

// `count` maps from p on, into LDS by all waves together.
__device__ __forceinline__ void fetch(const uint64_t* p, int count, float4* to) {
    constexpr int EACH = kGroup / kWaves;
    const int l = lane_id(), w = threadIdx.x / GS_WAVE;
    uint64_t v[EACH][2];
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (w + i * kWaves < count) {
            const uint64_t* q = p + (int64_t)(w + i * kWaves) * (2 * GS_WAVE) + l;
            v[i][0] = q[0];
            v[i][1] = q[GS_WAVE];
        }
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (w + i * kWaves < count) {
            const float2 a = unpair(v[i][0]), b = unpair(v[i][1]);
            to[(w + i * kWaves) * GS_WAVE + l] = make_float4(a.x, b.x, a.y, b.y);
        }
}

// One wave's part: publishes the chunk's map and waits for those in front of it
// in its group.  In s.anew: the last of them in which a segment starts, -1: none.
// `needed`: someone reads the state in front of the chunk.
__device__ __forceinline__ void publish(const Recur& r, int chunk, int block, const float4* own, const uint32_t* starts,
                                        bool needed, Lookers& s) {
    const int o = chunk % kGroup, l = lane_id();
    const int64_t first = (int64_t)block * r.chunks + chunk - o;
    float m[2], b[2];
    const bool any = whole_map(own, starts, l, m, b);
    put_map(r.maps + (first + o) * (2 * GS_WAVE), m, b);
    announce(r.flags + first + o, any ? kAnew : kMap);
    if (any && o == kGroup - 1) {
        const int64_t g = (int64_t)block * r.groups + chunk / kGroup;
        put(r.states + g * GS_WAVE + l, pair(b[0], b[1]));
        announce(r.flags + (int64_t)r.chunks * r.blocks + g, kState);
    }
    s.own[l] = make_float4(m[0], m[1], b[0], b[1]);
    int from = kNotNeeded - 1;
    if (needed) {
        from = kGaveUp - 1;
        for (int polls = 0; polls < kPolls; ++polls) {
            const uint32_t f = l < o ? __hip_atomic_load(r.flags + first + l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
            const uint32_t there = (uint32_t)__ballot(f != 0u), anew = (uint32_t)__ballot(f == kAnew);
            const int p = anew ? 31 - __clz(anew) : -1;
            const uint32_t front = (1u << o) - 1, known = p < 0 ? 0u : (2u << p) - 1;
            if ((front & ~known & ~there) == 0) {
                from = p;
                break;
            }
            __builtin_amdgcn_s_sleep(kPause);
        }
    }
    if (l == 0) {
        s.anew = from;
        s.speaks = o == kGroup - 1 && !any;
    }
}

// Every wave's part, behind a barrier: the maps of the group's chunks in front,
// back to the last in which a segment starts.
__device__ __forceinline__ void fetch_group(const Recur& r, int chunk, int block, Lookers& s) {
    const int o = chunk % kGroup, from = max(s.anew, 0);
    asm volatile("" ::: "memory");             // read behind the flags
    if (s.anew >= -1) fetch(r.maps + ((int64_t)block * r.chunks + chunk - o + from) * (2 * GS_WAVE), o - from, s.fetched);
}

// One wave's part, behind another: joins them, says the group's map if the chunk
// is its last, and waits until a state is known within the 64 groups in front and
// the maps of those between are there; in s.distance how many those are.
__device__ __forceinline__ void join_and_wait(const Recur& r, int chunk, int block, Lookers& s) {
    const int o = chunk % kGroup, l = lane_id(), p = s.anew, from = max(p, 0);
    float fm[2] = {1.0f, 1.0f}, fb[2] = {0.0f, 0.0f}, least[2] = {1.0f, 1.0f};
    if (p >= -1) {
#pragma unroll 2
        for (int k = 0; k < o - from; ++k) {
            const float4 v = s.fetched[k * GS_WAVE + l];
            const bool whole = k == 0 && p >= 0;           // a segment starts in it: its map is the constant b
            fb[0] = whole ? v.z : fmaf(v.x, fb[0], v.z);
            fb[1] = whole ? v.w : fmaf(v.y, fb[1], v.w);
            fm[0] *= v.x;
            fm[1] *= v.y;
            least[0] = fminf(least[0], v.x);
            least[1] = fminf(least[1], v.y);
        }
        fm[0] = product(fm[0], least[0]);
        fm[1] = product(fm[1], least[1]);
        if (s.speaks) {
            const int64_t g = (int64_t)block * r.groups + chunk / kGroup;
            uint32_t* flag = r.flags + (int64_t)r.chunks * r.blocks + g;
            const float4 own = s.own[l];
            const float gb[2] = {fmaf(own.x, fb[0], own.z), fmaf(own.y, fb[1], own.w)};
            if (p >= 0) {
                put(r.states + g * GS_WAVE + l, pair(gb[0], gb[1]));
                announce(flag, kState);
            } else {
                const float gm[2] = {behind(fm[0], own.x), behind(fm[1], own.y)};
                put_map(r.group_maps + g * (2 * GS_WAVE), gm, gb);
                announce(flag, kMap);
            }
        }
    }
    s.front[l] = make_float4(fm[0], fm[1], fb[0], fb[1]);
    int d = p == kGaveUp - 1 ? kGaveUp : kNotNeeded;
    if (p == -1) {
        const int c = chunk / kGroup - 1 - l;
        const uint32_t* flag = r.flags + (int64_t)r.chunks * r.blocks + (int64_t)block * r.groups + c;
        d = kGaveUp;
        for (int polls = 0; polls < kPolls; ++polls) {
            const uint32_t v = c >= 0 ? __hip_atomic_load(flag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
            const uint64_t known = __ballot(v == kState), there = __ballot(v != 0u);
            if (known && (~there & ((known & -known) - 1)) == 0) {
                d = __ffsll((unsigned long long)known) - 1;
                break;
            }
            __builtin_amdgcn_s_sleep(kPause);
        }
    }
    if (l == 0) s.distance = d;
}

// Every wave's part, behind a barrier: h, the state in front of the chunk; from
// the group's last chunk the state behind the group.
__device__ __forceinline__ void front_state(const Recur& r, int chunk, int block, Lookers& s, float* h) {
    const int l = lane_id(), w = threadIdx.x / GS_WAVE, d = s.distance;
    if (d < 0) {
        h[0] = d == kGaveUp ? NAN : s.front[l].z;
        h[1] = d == kGaveUp ? NAN : s.front[l].w;
        return;
    }
    const int64_t g = (int64_t)block * r.groups + chunk / kGroup;
    asm volatile("" ::: "memory");             // read behind the flags
    if (w == kWaves - 1) s.state[l] = unpair(r.states[(g - 1 - d) * GS_WAVE + l]);
    float q[2] = {0.0f, 0.0f};
    int far = d;
    do {
        const int count = min(far, kGroup);    // groups g - far .. g - far + count - 1
        fetch(r.group_maps + (g - far) * (2 * GS_WAVE), count, s.fetched);
        __syncthreads();
        if (far == d) {
            q[0] = s.state[l].x;
            q[1] = s.state[l].y;
        }
#pragma unroll 2
        for (int k = 0; k < count; ++k) {
            const float4 v = s.fetched[k * GS_WAVE + l];
            q[0] = fmaf(v.x, q[0], v.z);
            q[1] = fmaf(v.y, q[1], v.w);
        }
        far -= count;
        if (far > 0) __syncthreads();
    } while (far > 0);
    const float4 f = s.front[l];
    h[0] = fmaf(f.x, q[0], f.z);
    h[1] = fmaf(f.y, q[1], f.w);
    if (w != 0 || !s.speaks) return;
    const float4 own = s.own[l];               // by the group's map, as the groups behind join it
    put(r.states + g * GS_WAVE + l, pair(fmaf(behind(f.x, own.x), q[0], fmaf(own.x, f.z, own.z)),
                                         fmaf(behind(f.y, own.y), q[1], fmaf(own.y, f.w, own.w))));
    announce(r.flags + (int64_t)r.chunks * r.blocks + g, kState);
}

// The next chunk of the workgroup's block of channels, in the order of the
// recurrence.  A counter a block, each on a line of its own: 768 workgroups that
// start together wait 5 us for one counter.
constexpr int kCounter = 32;                   // words between the counters

// A workgroup's block of channels: each has as many workgroups as chunks, and they
// are spread over the XCDs (workgroups go round those in turn; a block on one of
// them alone took 290 us for the 131,072 tokens that take 212).
__device__ __forceinline__ int block_of(const Recur& r) { return (int)((blockIdx.x + blockIdx.x / r.blocks) % r.blocks); }

__device__ __forceinline__ int take_chunk(const Recur& r, uint32_t* shared, int block) {
    if (threadIdx.x == 0) *shared = atomicAdd(r.flags + (r.chunks + r.groups) * r.blocks + block * kCounter, 1u);
    __syncthreads();
    return (int)__builtin_amdgcn_readfirstlane(*shared);
}

// ALONE: the list is one chunk, which looks nowhere; workgroups behind those of
// the channels see to empty segments.  SHORT: the first states of all segments
// are loaded at once (steps of served sequences start one at every token);
// otherwise where they are used, and 16-bit tokens leave room for three
// workgroups a unit instead of two.
template <typename T, bool ONE, bool ALONE, bool SHORT>
__global__ void __launch_bounds__((ALONE ? kAloneWaves : kWaves) * GS_WAVE, SHORT && !ALONE && sizeof(T) == 4 ? 2 : SHORT || sizeof(T) == 4 ? 4 : 6) k_recur(Recur r, RecurOut o) {
    constexpr int WAVES = ALONE ? kAloneWaves : kWaves;
    __shared__ float4 maps[WAVES * GS_WAVE];
    __shared__ Lookers look;
    __shared__ uint32_t anew[WAVES], ticket;
    const gs_recur& a = r.a;
    const int w = threadIdx.x / GS_WAVE, l = lane_id();
    int chunk = 0, block = ALONE ? blockIdx.x : block_of(r);
    if (ALONE && block >= r.blocks) {
        pass_empty(a, a.initial, o.final, (block - r.blocks) * WAVES + w, (gridDim.x - r.blocks) * WAVES);
        return;
    }
    if (!ALONE) {
        chunk = take_chunk(r, &ticket, block);
        if (chunk >= r.chunks) return;
    }
    const uint32_t col = column<ONE>(a, block, r.width);
    Tokens tk;
    tk.p0 = __builtin_amdgcn_readfirstlane(chunk * kChunk + w * kSteps);
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
    tk.find(a, tk.p0);                         // while the tokens are on their way
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
    const uint32_t firsts = a.initial ? tk.starts & tk.inside : 0u;
    // a segment's first state
    auto first_of = [&](int i, float* h) {
        h[0] = h[1] = 0.0f;
        if (bit(firsts, i)) {
            Two<float, ONE> v;
            v.load(a.initial, tk.segment(i), a.cols, col);
            h[0] = v[0];
            h[1] = v[1];
        }
    };
    float h0[SHORT ? kSteps : 1][2];
    if (SHORT)
#pragma unroll
        for (int i = 0; i < kSteps; ++i) first_of(i, h0[SHORT ? i : 0]);
    auto start = [&](int i, float* h) {
        rare();
        if (SHORT) {
            h[0] = h0[SHORT ? i : 0][0];
            h[1] = h0[SHORT ? i : 0][1];
        } else {
            first_of(i, h);
        }
    };
    // The wave's map.  Gates and x stay as they were loaded, so that three
    // workgroups of 16-bit tokens fit a unit (opened gates: two, 236 us for 214).
    float m[2] = {1.0f, 1.0f}, h[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (bit(tk.starts, i)) {
            m[0] = m[1] = 0.0f;
            start(i, h);
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float A, z;
            open(gate_of(gs[i][c]), A, z);
            m[c] *= A;
            h[c] = fmaf(A, h[c], z * xs[i][c]);
        }
    }
    if (!tk.starts && __any(m[0] == 0.0f || m[1] == 0.0f)) {   // which gates it ran through
        m[0] = m[1] = 1.0f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                gs[i].again();
                float A, z;
                open(gate_of(gs[i][c]), A, z);
                m[c] = behind(m[c], A);
            }
    }
    maps[w * GS_WAVE + l] = make_float4(m[0], m[1], h[0], h[1]);
    if (l == 0) anew[w] = tk.starts != 0;
    __syncthreads();
    h[0] = h[1] = 0.0f;
    if (!ALONE) {
        if (w == 0) publish(r, chunk, block, maps, anew, !bit(tk.starts, 0), look);
        __syncthreads();
        fetch_group(r, chunk, block, look);
        __syncthreads();
        if (w == 0) join_and_wait(r, chunk, block, look);
        __syncthreads();
        front_state(r, chunk, block, look, h);
    }
    through(maps, anew, 0, w, l, h);
    if (o.kept && tk.p0 % GS_RECUR_KEEP == 0 && tk.p0 < a.n)
        Two<float, ONE>::store(o.kept, tk.p0 / GS_RECUR_KEEP, a.cols, col, bit(tk.starts, 0) ? 0.0f : h[0],
                               bit(tk.starts, 0) ? 0.0f : h[1]);
    const uint32_t written = a.fill ? tk.there(a) : tk.inside, lasts = o.final ? tk.ends & tk.inside : 0u;
    Rows y = Rows::of<T>(a, tk, o.y, o.ld_y, first, false);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (bit(tk.starts, i)) start(i, h);
        xs[i].again();
        gs[i].again();
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float A, z;
            open(gate_of(gs[i][c]), A, z);
            h[c] = fmaf(A, h[c], z * xs[i][c]);
        }
        if (bit(written, i)) Two<T, ONE>::store(y.p, col, h[0], h[1]);
        y.next();
        if (bit(lasts, i)) Two<float, ONE>::store(o.final, tk.segment(i), a.cols, col, h[0], h[1]);
    }
}

// Steps of served sequences: a wave walks one segment alone, four tokens' loads on
// the way at a time; the wave behind the last segment's fills the tokens that are
// in none.  Bound by the latency of three loads, one after the other (160 steps
// of 2048 channels in a graph 3.0 us; a chunk, whose waves look for their
// segments and meet, 11.6).  A segment of 1024 tokens beside empty ones takes 157.
template <typename T, bool ONE>
__global__ void __launch_bounds__(GS_BLOCK) k_recur_step(Recur r, RecurOut o) {
    constexpr int AHEAD = 4;
    const gs_recur& a = r.a;
    const int item = __builtin_amdgcn_readfirstlane(blockIdx.x * (GS_BLOCK / GS_WAVE) + threadIdx.x / GS_WAVE);
    const int s = item / r.blocks, block = item % r.blocks;
    if (s > a.n_seg) return;
    const uint32_t col = column<ONE>(a, block, r.width);
    Two<float, ONE> first;
    first.fill(0.0f);
    const bool outside = s == a.n_seg;
    if (!outside && a.initial) first.load(a.initial, s, a.cols, col);
    if (outside) {
        auto zeros = [&](int32_t t, int32_t end) {
            for (; t < end; ++t) Two<T, ONE>::store(o.y, t, o.ld_y, col, 0.0f, 0.0f);
        };
        if (a.fill && a.cu) {
            zeros(0, start_of(a, 0));
            zeros(start_of(a, a.n_seg), a.n);
        }
        return;
    }
    const int32_t t0 = start_of(a, s), t1 = start_of(a, s + 1);
    float h[2] = {first[0], first[1]};
    for (int32_t t = t0; t < t1; t += AHEAD) {
        Two<T, ONE> gs[AHEAD], xs[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int32_t at = min(t + i, t1 - 1), row = a.reverse ? t0 + t1 - 1 - at : at;
            gs[i].load(a.gate, row, a.ld_gate, col);
            xs[i].load(a.x, row, a.ld_x, col);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (t + i >= t1) break;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float A, z;
                open(gate_of(gs[i][c]), A, z);
                h[c] = fmaf(A, h[c], z * xs[i][c]);
                loaded(h[c]);                  // fused with the rounding to fp16, it gives other last bits
            }
            Two<T, ONE>::store(o.y, a.reverse ? t0 + t1 - 1 - t - i : t + i, o.ld_y, col, h[0], h[1]);
        }
    }
    if (o.final) Two<float, ONE>::store(o.final, s, a.cols, col, h[0], h[1]);
}

// Gradient: D_t = dy_t + a_{t+1} D_{t+1} from the last token to the first (dfinal
// comes in at a segment's last one), c_t = a_t D_t passes on;
//   dx_t = (1 - a_t) D_t;  dgate_t = a_t (1 - a_t) (h_{t-1} - x_t) D_t;  dinitial = c of the first token.
// h is formed again from the states that the forward kept every GS_RECUR_KEEP
// tokens, in fp32, not read in the tokens' type.  Nine ragged bf16 segments of up to
// 60,000 tokens, 768 channels: 286 us, 3.9 TB/s.
template <typename T, bool ONE, bool ALONE>
__global__ void __launch_bounds__((ALONE ? kAloneWaves : kWaves) * GS_WAVE, 4) k_recur_bwd(Recur r, gs_recur_grads o) {
    constexpr int WAVES = ALONE ? kAloneWaves : kWaves;
    __shared__ float4 maps[WAVES * GS_WAVE], back[WAVES * GS_WAVE];
    __shared__ Lookers look;
    __shared__ uint32_t anew[WAVES], ended[WAVES], ticket;
    const gs_recur& a = r.a;
    const int w = threadIdx.x / GS_WAVE, l = lane_id();
    int turn = 0, block = ALONE ? blockIdx.x : block_of(r);    // chunks are taken from the last one on
    if (ALONE && block >= r.blocks) {
        pass_empty(a, o.dfinal, o.dinitial, (block - r.blocks) * WAVES + w, (gridDim.x - r.blocks) * WAVES);
        return;
    }
    if (!ALONE) {
        turn = take_chunk(r, &ticket, block);
        if (turn >= r.chunks) return;
    }
    const int chunk = r.chunks - 1 - turn;
    const uint32_t col = column<ONE>(a, block, r.width);
    Tokens tk;
    tk.p0 = __builtin_amdgcn_readfirstlane(chunk * kChunk + w * kSteps);
    Two<T, ONE> gs[kSteps], xs[kSteps], ds[kSteps];
    // behind the last place the last one's row, whose values are not used
    const int32_t first = min(tk.p0, a.n - 1), end = min(tk.p0 + kSteps, a.n) - 1;
    Rows gate = Rows::of<T>(a, tk, a.gate, a.ld_gate, first, false), x = Rows::of<T>(a, tk, a.x, a.ld_x, first, false);
    Rows dy = Rows::of<T>(a, tk, o.dy, o.ld_dy, first, false);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        gs[i].load(gate.p, col);
        xs[i].load(x.p, col);
        ds[i].load(dy.p, col);
        gate.next(tk.p0 + i + 1 < a.n);
        x.next(tk.p0 + i + 1 < a.n);
        dy.next(tk.p0 + i + 1 < a.n);
    }
    tk.find(a, tk.p0);                         // while the tokens are on their way
    // tokens outside every segment: a gate that holds, and zeros
    if (tk.inside != kAllSteps) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
            if (!bit(tk.inside, i)) {
                rare();
                gs[i].fill(INFINITY);
                xs[i].fill(0.0f);
                ds[i].fill(0.0f);
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
    // A product of the gates has run to 0, and may have met an infinite dy: token by
    // token, where it has.
    const bool gone = bm[0] == 0.0f || bm[1] == 0.0f || (!tk.starts && (m[0] == 0.0f || m[1] == 0.0f));
    if (__any(gone)) {
        float c[2] = {0.0f, 0.0f}, p[2] = {1.0f, 1.0f};
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i)
            if (i <= first_end) {
                if (bit(lasts, i)) state_of(o.dfinal, i, c);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float gate = S[i][k], A, z;
                    loaded(gate);              // opened again: held open since the walk above, it would take registers
                    open(gate, A, z);
                    c[k] = A * (ds[i][k] + c[k]);
                    p[k] = behind(p[k], A);
                }
            }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            b[k] = b[k] != b[k] ? c[k] : b[k];
            bm[k] = bm[k] == 0.0f ? p[k] : bm[k];
            m[k] = !tk.starts && m[k] == 0.0f ? p[k] : m[k];           // no start among them: p is of all
        }
    }
    if (tk.ends) bm[0] = bm[1] = 0.0f;
    back[(WAVES - 1 - w) * GS_WAVE + l] = make_float4(bm[0], bm[1], b[0], b[1]);
    maps[w * GS_WAVE + l] = make_float4(m[0], m[1], h[0], h[1]);
    if (l == 0) {
        ended[WAVES - 1 - w] = tk.ends != 0;
        anew[w] = tk.starts != 0;
    }
    __syncthreads();
    if (!ALONE) {
        if (w == kWaves - 1) publish(r, turn, block, back, ended, !bit(tk.ends, kSteps - 1), look);
        __syncthreads();
        fetch_group(r, turn, block, look);
        __syncthreads();
        if (w == kWaves - 1) join_and_wait(r, turn, block, look);
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
        front_state(r, turn, block, look, g);
    }
    through(back, ended, 0, WAVES - 1 - w, l, g);
    if (sizeof(T) == 4) {                      // dy once more: there are no registers to hold it meanwhile
        Rows again = Rows::of<T>(a, tk, o.dy, o.ld_dy, first, false);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            ds[i].load(again.p, col);
            again.next(tk.p0 + i + 1 < a.n);
            if (!bit(tk.inside, i)) {
                rare();
                ds[i].fill(0.0f);
            }
        }
    }
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
    int32_t chunks, groups, blocks, width;
    size_t maps, group_maps, states, flags, bytes;
};

RecurPlan recur_plan(int32_t n, int32_t cols) {
    RecurPlan p;
    p.chunks = n <= kAloneChunk ? 1 : (int32_t)div_up(n, kChunk);
    p.width = kCols;                           // so that no block has a single channel
    while (cols > 1 && cols % p.width == 1) p.width -= 2;
    p.blocks = (int32_t)div_up(cols, p.width);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align256(bytes);
        return here;
    };
    p.groups = (int32_t)div_up(p.chunks, kGroup);
    const size_t many = p.chunks > 1 ? p.blocks : 0, all = many * p.chunks, groups = many * p.groups;
    p.maps = take(all * GS_WAVE * 16);
    p.group_maps = take(groups * GS_WAVE * 16);
    p.states = take(groups * GS_WAVE * 8);
    p.flags = take((all + groups + many * kCounter) * 4);
    p.bytes = at > 0 ? at + kLine - 16 : 0;    // from the first multiple of kLine in a 16-byte aligned workspace
    return p;
}

Recur recur_of(const gs_recur& a, const RecurPlan& p, void* ws) {
    char* base = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(ws) + kLine - 1) & ~(uintptr_t)(kLine - 1));
    Recur r;
    r.a = a;
    r.chunks = p.chunks;
    r.groups = p.groups;
    r.blocks = p.blocks;
    r.width = p.width;
    const bool alone = p.chunks <= 1;
    r.maps = alone ? nullptr : reinterpret_cast<uint64_t*>(base + p.maps);
    r.group_maps = alone ? nullptr : reinterpret_cast<uint64_t*>(base + p.group_maps);
    r.states = alone ? nullptr : reinterpret_cast<uint64_t*>(base + p.states);
    r.flags = alone ? nullptr : reinterpret_cast<uint32_t*>(base + p.flags);
    return r;
}

// Flags cleared for the chunks' workgroups; their number for the only ones'.
void clear_flags(const Recur& r, const float* from, float* to, hipStream_t st) {
    const int32_t flags = (r.chunks + r.groups + kCounter) * r.blocks;
    const uint32_t most = std::max(div_up(flags, GS_BLOCK), to && r.a.cu ? div_up(r.a.n_seg, GS_BLOCK) : 1u);
    k_recur_clear<<<std::min(most, 1024u), GS_BLOCK, 0, st>>>(r.a, from, to, r.flags, flags);
}

constexpr uint32_t kEmptyBlocks = 256;         // that see to empty segments, at most

uint32_t alone_grid(const Recur& r, const float* to) {
    return r.blocks + (to && r.a.cu ? std::min(div_up(r.a.n_seg, kAloneWaves * GS_WAVE), kEmptyBlocks) : 0u);
}

// Whether a wave takes a segment: a token each, as far as the sizes tell (a list
// of more tokens may be one that is being read in beside others' steps, and one
// wave would walk it), or equal segments of a few.
bool steps(const Recur& r, const RecurOut& o) {
    constexpr int32_t kTokens = 1024, kEach = 4;
    const gs_recur& a = r.a;
    if (o.kept || (int64_t)(a.n_seg + 1) * r.blocks >= 1 << 24) return false;
    return a.cu ? a.n <= a.n_seg && a.n <= kTokens : a.n <= (int64_t)a.n_seg * kEach;
}

template <typename T, bool ONE>
hipError_t recur_go(const Recur& r, const RecurOut& o, hipStream_t st) {
    if (steps(r, o)) {
        k_recur_step<T, ONE><<<div_up((r.a.n_seg + 1) * r.blocks, GS_BLOCK / GS_WAVE), GS_BLOCK, 0, st>>>(r, o);
    } else if (r.chunks == 1) {
        k_recur<T, ONE, true, true><<<alone_grid(r, o.final), kAloneWaves * GS_WAVE, 0, st>>>(r, o);
    } else {
        clear_flags(r, r.a.initial, o.final, st);
        const uint32_t grid = (uint32_t)r.chunks * r.blocks;
        // A segment in every four tokens: waiting for one state after the other takes
        // longer than a unit's third workgroup gains (32,768 tokens of 1024 channels
        // in 8192 segments 80 us for 82, in 4096 58 for 52).  And states in place
        // are read once, before anyone can know the segment's last one.
        if (r.a.initial && (r.a.n_seg >= r.a.n / 4 || r.a.initial == o.final)) k_recur<T, ONE, false, true><<<grid, kWaves * GS_WAVE, 0, st>>>(r, o);
        else k_recur<T, ONE, false, false><<<grid, kWaves * GS_WAVE, 0, st>>>(r, o);
    }
    return hipGetLastError();
}

template <typename T, bool ONE>
hipError_t recur_bwd_go(const Recur& r, const gs_recur_grads& g, hipStream_t st) {
    if (r.chunks == 1) {
        k_recur_bwd<T, ONE, true><<<alone_grid(r, g.dinitial), kAloneWaves * GS_WAVE, 0, st>>>(r, g);
    } else {
        clear_flags(r, g.dfinal, g.dinitial, st);
        k_recur_bwd<T, ONE, false><<<(uint32_t)r.chunks * r.blocks, kWaves * GS_WAVE, 0, st>>>(r, g);
    }
    return hipGetLastError();
}

// No tokens at all: the segments' states alone.
hipError_t no_tokens(const gs_recur& a, const float* from, float* to, hipStream_t st) {
    if (to) k_recur_clear<<<std::min(div_up(a.n_seg, GS_BLOCK), 1024u), GS_BLOCK, 0, st>>>(a, from, to, nullptr, 0);
    return hipGetLastError();
}

// A lane takes one channel where there are lanes for all of them: fewer registers,
// more waves (a million fp32 tokens of 64 channels 228 us for 304, of 5 in bf16 190
// for 208); blocks of 64 channels of wider tokens lose (131,072 fp32 tokens of 1024
// 340 us for 305).
template <typename T>
hipError_t recur_type(const Recur& r, const RecurOut& o, hipStream_t st) {
    return r.a.cols <= GS_WAVE ? recur_go<T, true>(r, o, st) : recur_go<T, false>(r, o, st);
}

template <typename T>
hipError_t recur_bwd_type(const Recur& r, const gs_recur_grads& g, hipStream_t st) {
    return r.a.cols <= GS_WAVE ? recur_bwd_go<T, true>(r, g, st) : recur_bwd_go<T, false>(r, g, st);
}

}  // namespace

bool recurrence_fits(const gs_recur& a) {
    const RecurPlan p = recur_plan(a.n, a.cols);
    const uint64_t threads = p.chunks == 1 ? ((uint64_t)p.blocks + kEmptyBlocks) * kAloneWaves * GS_WAVE
                                           : (uint64_t)p.chunks * p.blocks * kWaves * GS_WAVE;
    return threads < 1ull << 32;
}

size_t recurrence_ws_bytes(const gs_recur& a) { return recur_plan(a.n, a.cols).bytes; }

hipError_t launch_recurrence(const gs_recur& a, void* y, int64_t ld_y, float* final, float* kept, void* ws,
                             hipStream_t st) {
    if (a.n == 0) return no_tokens(a, a.initial, final, st);
    const RecurPlan p = recur_plan(a.n, a.cols);
    const Recur r = recur_of(a, p, ws);
    const RecurOut o = {y, final, kept, ld_y};
    if (a.dtype == GS_F32) return recur_type<float>(r, o, st);
    return a.dtype == GS_BF16 ? recur_type<bf16_t>(r, o, st) : recur_type<f16_t>(r, o, st);
}

hipError_t launch_recurrence_bwd(const gs_recur& a, const gs_recur_grads& g, void* ws, hipStream_t st) {
    if (a.n == 0) return no_tokens(a, g.dfinal, g.dinitial, st);
    const RecurPlan p = recur_plan(a.n, a.cols);
    const Recur r = recur_of(a, p, ws);
    if (a.dtype == GS_F32) return recur_bwd_type<float>(r, g, st);
    return a.dtype == GS_BF16 ? recur_bwd_type<bf16_t>(r, g, st) : recur_bwd_type<f16_t>(r, g, st);
}

}  // namespace gsmi
