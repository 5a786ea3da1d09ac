// Lookup of a table's rows by the tokens' ids, and its gradient by sorted tokens.
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace gsmi {

namespace {

// ---------------------------------------------------------------------------
// out[t] = scale * table[id[t]], 0 where id is outside the table.  A thread
// moves 16-byte pieces of the output; bound by HBM bytes (the output, and the
// table's rows that are not in a cache).
// ---------------------------------------------------------------------------

constexpr int kPieces = 4;                     // of a thread, in flight together

template <typename TT, typename T, bool TAIL>
__global__ void __launch_bounds__(GS_BLOCK) k_embedding(gs_embed_args a, int tokens_a_block, int per, float inv_per) {
    constexpr int N = Piece<T>::N, CH = N > Piece<TT>::N ? N / Piece<TT>::N : 1, M = N / CH;
    typedef TT some __attribute__((ext_vector_type(M)));
    typedef some __attribute__((aligned(sizeof(TT)))) loose;
    const int64_t t0 = (int64_t)blockIdx.x * tokens_a_block;
    const int tokens = (int)min((int64_t)tokens_a_block, (int64_t)a.tokens - t0);
    const int items = tokens * per;
    for (int first = threadIdx.x; first < items; first += GS_BLOCK * kPieces) {
        int tok[kPieces], col[kPieces], id[kPieces];
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int i = min(first + k * GS_BLOCK, items - 1);
            // at most 2^12 items: the quotient is off by less than half a step of 1 / per
            tok[k] = (int)(((float)i + 0.5f) * inv_per);
            col[k] = (i - tok[k] * per) * N;
            id[k] = a.ids[t0 + tok[k]];
        }
        float f[kPieces][N];
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const bool in = (uint32_t)id[k] < (uint32_t)a.rows;
            const TT* p = static_cast<const TT*>(a.table) + (int64_t)(in ? id[k] : 0) * a.ld_table + col[k];
            const int there = in ? a.dim - col[k] : 0;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                some v = some{};
                if (there >= (c + 1) * M) {
                    v = *reinterpret_cast<const loose*>(p + c * M);
                } else if (TAIL) {
#pragma unroll
                    for (int i = 0; i < M; ++i)
                        if (c * M + i < there) v[i] = p[c * M + i];
                }
#pragma unroll
                for (int i = 0; i < M; ++i) f[k][c * M + i] = (float)v[i];
            }
        }
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            if (first + k * GS_BLOCK >= items) break;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                f[k][i] = (uint32_t)id[k] < (uint32_t)a.rows ? f[k][i] * a.scale : 0.0f;
                loaded(f[k][i]);               // an fp32 product for every type: fp16's could be fused with its rounding
            }
            Span<T, TAIL>::store(static_cast<T*>(a.out) + (t0 + tok[k]) * a.ld_out + col[k], a.dim - col[k], f[k]);
        }
    }
}

// ---------------------------------------------------------------------------
// Gradient.  The tokens are sorted by id (stable, so that a row's tokens stay in
// their order), and the sorted list is cut into chunks of one length, so that a
// row with very many tokens is shared by many chunks.  A group of lanes walks a
// chunk; rows that lie inside it are written at once, the ends that other chunks
// share go to partial rows, which k_embed_join adds in ascending order.  Nothing
// is summed by atomics: the same call gives the same bits.
//
// The sort: passes of `bits` <= 10 bits, lowest first, each a count of digits by
// block, a scan of the counts, and a scatter whose ranks come from the lanes
// that hold the same digit.  Ids outside the table become `rows`, the last key.
// ---------------------------------------------------------------------------

constexpr int kSortItems = 16;                 // of a thread
constexpr int kSortBlock = GS_BLOCK * kSortItems;
constexpr int kMostBits = 10;
constexpr int kMostBins = 1 << kMostBits;

struct SortPass {
    const int32_t* ids;                        // the first pass reads these,
    const uint2* from;                         // the others (key, token) pairs
    uint2* to;
    uint32_t* counts;                          // [bins][blocks]
    uint32_t* totals;                          // [bins]
    uint8_t* marks;                            // first pass: rows that have tokens (NULL: not wanted)
    int32_t n, rows, shift, bits, blocks;
};

__device__ __forceinline__ uint2 sort_item(const SortPass& s, int64_t i) {
    if (s.from) return s.from[i];
    const int32_t id = s.ids[i];
    return make_uint2((uint32_t)id < (uint32_t)s.rows ? (uint32_t)id : (uint32_t)s.rows, (uint32_t)i);
}

__global__ void __launch_bounds__(GS_BLOCK) k_sort_count(SortPass s) {
    __shared__ uint32_t count[kMostBins];
    const int bins = 1 << s.bits;
    for (int b = threadIdx.x; b < bins; b += GS_BLOCK) count[b] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kSortBlock;
#pragma unroll 4
    for (int k = 0; k < kSortItems; ++k) {
        const int64_t i = first + k * GS_BLOCK + threadIdx.x;
        if (i < s.n) {
            const uint2 v = sort_item(s, i);
            atomicAdd(&count[(v.x >> s.shift) & (bins - 1)], 1u);
            if (s.marks && v.x < (uint32_t)s.rows) s.marks[v.x] = 1;
        }
    }
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += GS_BLOCK) s.counts[(int64_t)b * s.blocks + blockIdx.x] = count[b];
}

// Exclusive prefixes of each bin's counts over the blocks, a wave a bin.
__global__ void __launch_bounds__(GS_BLOCK) k_sort_scan(SortPass s) {
    const int b = blockIdx.x * (GS_BLOCK / GS_WAVE) + threadIdx.x / GS_WAVE;
    if (b >= 1 << s.bits) return;
    uint32_t* c = s.counts + (int64_t)b * s.blocks;
    uint32_t before = 0;
    for (int i = 0; i < s.blocks; i += GS_WAVE) {
        const uint32_t v = i + lane_id() < s.blocks ? c[i + lane_id()] : 0;
        const uint32_t inc = wave_incl_scan(v);
        if (i + lane_id() < s.blocks) c[i + lane_id()] = before + inc - v;
        before += __shfl(inc, GS_WAVE - 1, GS_WAVE);
    }
    if (lane_id() == 0) s.totals[b] = before;
}

// ALONE: the only block, which needs no counts of others.
template <bool ALONE>
__global__ void __launch_bounds__(GS_BLOCK) k_sort_scatter(SortPass s) {
    constexpr int W = GS_BLOCK / GS_WAVE;
    __shared__ uint32_t count[W][kMostBins];
    __shared__ uint32_t scratch[W];
    const int bins = 1 << s.bits, w = threadIdx.x / GS_WAVE;
    for (int b = threadIdx.x; b < W * kMostBins; b += GS_BLOCK) (&count[0][0])[b] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kSortBlock + w * (GS_WAVE * kSortItems) + lane_id();
    uint2 item[kSortItems];
    uint32_t rank[kSortItems];
#pragma unroll
    for (int k = 0; k < kSortItems; ++k)
        item[k] = first + k * GS_WAVE < s.n ? sort_item(s, first + k * GS_WAVE) : make_uint2(0u, 0u);
#pragma unroll
    for (int k = 0; k < kSortItems; ++k) {
        const bool in = first + k * GS_WAVE < s.n;
        const uint32_t d = (item[k].x >> s.shift) & (bins - 1);
        if (s.marks && ALONE && in && item[k].x < (uint32_t)s.rows) s.marks[item[k].x] = 1;
        uint64_t same = __ballot(in);
        for (int i = 0; i < s.bits; ++i) {
            const uint64_t m = __ballot((d >> i) & 1);
            same &= (d >> i) & 1 ? m : ~m;
        }
        // the first lane of a digit takes places for all of them
        const int leader = in ? __ffsll((unsigned long long)same) - 1 : 0;
        uint32_t old = 0;
        if (in && leader == lane_id()) old = atomicAdd(&count[w][d], (uint32_t)popc64(same));
        old = __shfl(old, leader, GS_WAVE);
        rank[k] = old + popc64(same & lanemask_lt());
    }
    __syncthreads();
    // a thread's four bins: where the bin starts, where this block's share of it does, then wave by wave
    uint32_t tot[kMostBins / GS_BLOCK], sum = 0;
#pragma unroll
    for (int j = 0; j < kMostBins / GS_BLOCK; ++j) {
        const int b = threadIdx.x * (kMostBins / GS_BLOCK) + j;
        tot[j] = 0;
        if (b < bins) {
            if (ALONE) {
#pragma unroll
                for (int u = 0; u < W; ++u) tot[j] += count[u][b];
            } else {
                tot[j] = s.totals[b];
            }
        }
        sum += tot[j];
    }
    uint32_t all, before = block_excl_scan(sum, scratch, &all);
#pragma unroll
    for (int j = 0; j < kMostBins / GS_BLOCK; ++j) {
        const int b = threadIdx.x * (kMostBins / GS_BLOCK) + j;
        if (b < bins) {
            uint32_t at = before + (ALONE ? 0u : s.counts[(int64_t)b * s.blocks + blockIdx.x]);
#pragma unroll
            for (int u = 0; u < W; ++u) {
                const uint32_t c = count[u][b];
                count[u][b] = at;
                at += c;
            }
        }
        before += tot[j];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortItems; ++k)
        if (first + k * GS_WAVE < s.n) s.to[count[w][(item[k].x >> s.shift) & (bins - 1)] + rank[k]] = item[k];
}

// -- the touched rows alone: the sorted keys become places among the unique ids ---

__device__ __forceinline__ bool run_starts(const uint2* pairs, int64_t i, uint32_t rows) {
    return pairs[i].x < rows && (i == 0 || pairs[i - 1].x != pairs[i].x);
}

__global__ void __launch_bounds__(GS_BLOCK) k_run_count(const uint2* __restrict__ pairs, int32_t n, uint32_t rows,
                                                        uint32_t* __restrict__ counts) {
    __shared__ uint32_t scratch[GS_BLOCK / GS_WAVE];
    const int64_t first = (int64_t)blockIdx.x * GS_TILE_ITEMS;
    uint32_t c = 0;
    for (int k = 0; k < GS_ITEMS; ++k) {
        const int64_t i = first + k * GS_BLOCK + threadIdx.x;
        if (i < n) c += run_starts(pairs, i, rows);
    }
    c = block_sum_u32(c, scratch);
    if (threadIdx.x == 0) counts[blockIdx.x] = c;
}

__global__ void __launch_bounds__(GS_BLOCK) k_run_place(const uint2* __restrict__ pairs, int32_t n, uint32_t rows,
                                                        const uint32_t* __restrict__ counts, uint2* __restrict__ to,
                                                        int32_t* __restrict__ unique, int32_t* __restrict__ total) {
    __shared__ uint32_t scratch[GS_BLOCK / GS_WAVE];
    uint32_t before = block_sum_prefix(counts, blockIdx.x, scratch);
    const int64_t first = (int64_t)blockIdx.x * GS_TILE_ITEMS;
    for (int k = 0; k < GS_ITEMS; ++k) {
        const int64_t i = first + k * GS_BLOCK + threadIdx.x;
        const bool starts = i < n && run_starts(pairs, i, rows);
        uint32_t all;
        const uint32_t mine = before + block_excl_scan(starts, scratch, &all) + starts;    // runs up to here
        if (i < n) {
            const uint2 v = pairs[i];
            to[i] = make_uint2(v.x < rows ? mine - 1 : rows, v.y);
            if (starts) unique[mine - 1] = (int32_t)v.x;
        }
        before += all;
    }
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) *total = (int32_t)before;
}

// -- the sums --------------------------------------------------------------------

struct EmbedSum {
    const uint2* pairs;                        // (row of grad, token), sorted
    const void* dout;
    int64_t ld_dout, ld_grad;
    float* grad;
    float* parts;                              // [2 * chunks][dim]: a chunk's first and last row
    const uint8_t* marks;                      // rows that are not marked get zeros (NULL: none)
    int64_t rows;
    int32_t n, dim, chunks;
    uint32_t limit;                            // rows from here on are no one's
    float scale;
};

constexpr int kChunk = 32;                     // sorted tokens of a chunk

template <typename T, bool TAIL>
__device__ __forceinline__ void put_row(float* p, int there, const float* f) {
    constexpr int N = Piece<T>::N;
#pragma unroll
    for (int i = 0; i < N; i += 4) Span<float, TAIL>::store(p + i, there - i, f + i);
}

// G lanes a chunk, blockIdx.y: slabs of G * N columns.
template <typename T, bool TAIL, int G>
__global__ void __launch_bounds__(GS_BLOCK) k_embed_sum(EmbedSum a) {
    constexpr int N = Piece<T>::N, AHEAD = 8;
    const int col = blockIdx.y * (G * N) + (threadIdx.x % G) * N, there = a.dim - col;
    const int64_t g = (int64_t)blockIdx.x * (GS_BLOCK / G) + threadIdx.x / G;
    if (g >= a.chunks) return;
    const int64_t p0 = g * kChunk, p1 = min(p0 + kChunk, (int64_t)a.n);
    const uint32_t before = p0 > 0 ? a.pairs[p0 - 1].x : a.limit, after = p1 < a.n ? a.pairs[p1].x : a.limit;
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.0f;
    uint32_t row = a.pairs[p0].x;
    bool shared = row == before;               // with the chunk in front
    auto flush = [&](bool last) {
        if (row >= a.limit) return;
        float v[N];
        float* to = a.grad + (int64_t)row * a.ld_grad + col;
        if (shared) to = a.parts + (2 * g) * a.dim + col;
        else if (last && row == after) to = a.parts + (2 * g + 1) * a.dim + col;
        const bool whole = !shared && !(last && row == after);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = whole ? acc[i] * a.scale : acc[i];
        put_row<T, TAIL>(to, there, v);
    };
    for (int64_t p = p0; p < p1; p += AHEAD) {
        uint2 v[AHEAD];
        Span<T, TAIL> s[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) v[k] = p + k < p1 ? a.pairs[p + k] : make_uint2(a.limit, 0u);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            s[k].load(static_cast<const T*>(a.dout) + (int64_t)v[k].y * a.ld_dout + col, v[k].x < a.limit ? there : 0);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (p + k >= p1) break;
            if (v[k].x != row) {
                flush(false);
                row = v[k].x;
                shared = false;
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] = 0.0f;
            }
            float f[N];
            s[k].floats(f);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] += f[i];
        }
    }
    flush(true);
}

// Sum of the partial rows of one run, from the chunk that holds its start: the
// last row of that chunk, then the first rows of those behind it.  The groups of
// the workgroup take equal slices of them, added in ascending order.
template <typename T, bool TAIL, int G>
__global__ void __launch_bounds__(GS_BLOCK) k_embed_join(EmbedSum a) {
    constexpr int N = Piece<T>::N, GROUPS = GS_BLOCK / G;
    __shared__ float sums[GROUPS][G * N];
    const int64_t g = blockIdx.x, p0 = g * kChunk, p1 = p0 + kChunk;
    if (p1 >= a.n) return;
    const uint32_t row = a.pairs[p1 - 1].x;
    if (row >= a.limit || a.pairs[p1].x != row) return;
    if (p0 > 0 && a.pairs[p0].x == row && a.pairs[p0 - 1].x == row) return;    // it started before
    // the end of the run: the first position behind p1 with another row
    int64_t lo = p1, hi = a.n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (a.pairs[mid].x == row) lo = mid + 1;
        else hi = mid;
    }
    const int64_t last = (lo - 1) / kChunk, m = last - g;      // chunks g + 1 .. last
    const int group = threadIdx.x / G, lane = threadIdx.x % G;
    const int col = blockIdx.y * (G * N) + lane * N, there = a.dim - col;
    const int64_t per = (m + GROUPS - 1) / GROUPS;
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.0f;
    auto add = [&](const float* p) {
        float f[N];
        load_floats<N, TAIL>(p + col, 0, there, f);
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] += f[i];
    };
    if (group == 0) add(a.parts + (2 * g + 1) * a.dim);
#pragma unroll 4
    for (int64_t j = group * per; j < min((group + 1) * per, m); ++j) add(a.parts + 2 * (g + 1 + j) * a.dim);
#pragma unroll
    for (int i = 0; i < N; ++i) sums[group][lane * N + i] = acc[i];
    __syncthreads();
    if (group == 0) {
#pragma unroll
        for (int u = 1; u < GROUPS; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] += sums[u][lane * N + i];
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] *= a.scale;
        put_row<T, TAIL>(a.grad + (int64_t)row * a.ld_grad + col, there, acc);
    }
}

// Zeros for the rows that no token marked.
__global__ void __launch_bounds__(GS_BLOCK) k_embed_zeros(EmbedSum a, int rows_a_block) {
    const int64_t r0 = (int64_t)blockIdx.x * rows_a_block, r1 = min(r0 + rows_a_block, a.rows);
    for (int64_t r = r0 + threadIdx.x / GS_WAVE; r < r1; r += GS_BLOCK / GS_WAVE) {
        if (a.marks && a.marks[r]) continue;
        for (int c = lane_id(); c < a.dim; c += GS_WAVE) a.grad[r * a.ld_grad + c] = 0.0f;
    }
}

__global__ void k_zero_words(uint32_t* p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) p[i] = 0;
}

struct EmbedPlan {
    int32_t bits, passes, digit, blocks, chunks;
    size_t pairs[2], counts, totals, marks, parts, bytes;
};

EmbedPlan embed_plan(int32_t n, int32_t rows, int32_t dim, bool touched) {
    EmbedPlan p;
    p.bits = 1;
    while (p.bits < 31 && (uint32_t)rows >> p.bits) ++p.bits;              // of the key `rows`
    p.passes = (p.bits + kMostBits - 1) / kMostBits;
    p.digit = (p.bits + p.passes - 1) / p.passes;
    p.blocks = (int32_t)div_up(n, kSortBlock);
    p.chunks = (int32_t)div_up(n, kChunk);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align256(bytes);
        return here;
    };
    p.pairs[0] = take((size_t)n * 8);
    p.pairs[1] = take((size_t)n * 8);
    // counts of the sort, then of the runs
    p.counts = take(std::max(((size_t)p.blocks << p.digit) * 4, (size_t)div_up(n, GS_TILE_ITEMS) * 4 + 16));
    p.totals = take((size_t)kMostBins * 4);
    p.marks = take(touched ? 0 : (size_t)rows);
    p.parts = take((size_t)p.chunks * 2 * dim * 4);
    p.bytes = at;
    return p;
}

template <typename T, bool TAIL, int G>
hipError_t sum_go(const EmbedSum& a, hipStream_t st) {
    const uint32_t slabs = div_up(a.dim, G * Piece<T>::N);
    k_embed_sum<T, TAIL, G><<<dim3(div_up(a.chunks, GS_BLOCK / G), slabs), GS_BLOCK, 0, st>>>(a);
    if (a.chunks > 1) k_embed_join<T, TAIL, G><<<dim3(a.chunks, slabs), GS_BLOCK, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T, bool TAIL>
hipError_t sum_lanes(const EmbedSum& a, hipStream_t st) {
    const int pieces = (int)div_up(a.dim, Piece<T>::N);
    if (pieces <= 4) return sum_go<T, TAIL, 4>(a, st);
    if (pieces <= 8) return sum_go<T, TAIL, 8>(a, st);
    if (pieces <= 16) return sum_go<T, TAIL, 16>(a, st);
    if (pieces <= 32) return sum_go<T, TAIL, 32>(a, st);
    return sum_go<T, TAIL, 64>(a, st);
}

template <typename T>
hipError_t sum_type(const EmbedSum& a, hipStream_t st) {
    return a.dim % Piece<T>::N ? sum_lanes<T, true>(a, st) : sum_lanes<T, false>(a, st);
}

template <typename TT, typename T>
hipError_t embed_go(const gs_embed_args& all, hipStream_t st) {
    const int per = (int)div_up(all.dim, Piece<T>::N);
    const int tokens_a_block = std::max(1, GS_BLOCK * kPieces / per);
    const float inv = 1.0f / (float)per;
    // a launch holds fewer than 2^32 threads
    const int64_t most = (int64_t)tokens_a_block << 23;
    for (int64_t first = 0; first < all.tokens; first += most) {
        gs_embed_args a = all;
        a.tokens = (int32_t)std::min<int64_t>(most, all.tokens - first);
        a.ids = all.ids + first;
        a.out = static_cast<T*>(all.out) + first * all.ld_out;
        const uint32_t grid = div_up(a.tokens, tokens_a_block);
        if (a.dim % Piece<T>::N == 0) k_embedding<TT, T, false><<<grid, GS_BLOCK, 0, st>>>(a, tokens_a_block, per, inv);
        else k_embedding<TT, T, true><<<grid, GS_BLOCK, 0, st>>>(a, tokens_a_block, per, inv);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_embedding(const gs_embed_args& a, hipStream_t st) {
    if (a.dtype == GS_F32) return embed_go<float, float>(a, st);
    if (a.table_dtype == GS_F32)
        return a.dtype == GS_BF16 ? embed_go<float, bf16_t>(a, st) : embed_go<float, f16_t>(a, st);
    return a.dtype == GS_BF16 ? embed_go<bf16_t, bf16_t>(a, st) : embed_go<f16_t, f16_t>(a, st);
}

size_t embedding_bwd_ws_bytes(int32_t tokens, int32_t rows, int32_t dim, bool touched) {
    return embed_plan(tokens, rows, dim, touched).bytes;
}

hipError_t launch_embedding_bwd(const gs_embed_bwd_args& g, void* ws, hipStream_t st) {
    const bool touched = g.unique != nullptr;
    const EmbedPlan p = embed_plan(g.tokens, g.rows, g.dim, touched);
    char* base = static_cast<char*>(ws);
    EmbedSum s;
    s.dout = g.dout;
    s.ld_dout = g.ld_dout;
    s.ld_grad = g.ld_grad;
    s.grad = g.grad;
    s.parts = reinterpret_cast<float*>(base + p.parts);
    s.marks = nullptr;
    s.rows = g.rows;
    s.n = g.tokens;
    s.dim = g.dim;
    s.chunks = p.chunks;
    s.limit = (uint32_t)g.rows;
    s.scale = g.scale;
    uint8_t* marks = touched || g.tokens == 0 ? nullptr : reinterpret_cast<uint8_t*>(base + p.marks);
    if (marks) {
        const int64_t words = ((int64_t)g.rows + 3) / 4;
        k_zero_words<<<(uint32_t)std::min<int64_t>(1024, div_up(words, GS_BLOCK)), GS_BLOCK, 0, st>>>(
            reinterpret_cast<uint32_t*>(marks), words);
    }
    if (g.tokens > 0) {
        uint2* buf[2] = {reinterpret_cast<uint2*>(base + p.pairs[0]), reinterpret_cast<uint2*>(base + p.pairs[1])};
        uint32_t* counts = reinterpret_cast<uint32_t*>(base + p.counts);
        int at = 0;
        for (int i = 0; i < p.passes; ++i, at ^= 1) {
            SortPass q;
            q.ids = g.ids;
            q.from = i ? buf[at ^ 1] : nullptr;
            q.to = buf[at];
            q.counts = counts;
            q.totals = reinterpret_cast<uint32_t*>(base + p.totals);
            q.marks = i ? nullptr : marks;
            q.n = g.tokens;
            q.rows = g.rows;
            q.shift = i * p.digit;
            q.bits = std::min(p.digit, p.bits - i * p.digit);
            q.blocks = p.blocks;
            if (p.blocks == 1) {
                k_sort_scatter<true><<<1, GS_BLOCK, 0, st>>>(q);
                continue;
            }
            k_sort_count<<<p.blocks, GS_BLOCK, 0, st>>>(q);
            k_sort_scan<<<div_up(1u << q.bits, GS_BLOCK / GS_WAVE), GS_BLOCK, 0, st>>>(q);
            k_sort_scatter<false><<<p.blocks, GS_BLOCK, 0, st>>>(q);
        }
        s.pairs = buf[at ^ 1];
        if (touched) {
            const uint32_t blocks = div_up(g.tokens, GS_TILE_ITEMS);
            k_run_count<<<blocks, GS_BLOCK, 0, st>>>(s.pairs, g.tokens, (uint32_t)g.rows, counts);
            k_run_place<<<blocks, GS_BLOCK, 0, st>>>(s.pairs, g.tokens, (uint32_t)g.rows, counts, buf[at], g.unique,
                                                     g.count);
            s.pairs = buf[at];
        }
        hipError_t e = g.dtype == GS_F32    ? sum_type<float>(s, st)
                       : g.dtype == GS_BF16 ? sum_type<bf16_t>(s, st)
                                            : sum_type<f16_t>(s, st);
        if (e != hipSuccess) return e;
    } else if (touched) {
        k_zero_words<<<1, 1, 0, st>>>(reinterpret_cast<uint32_t*>(g.count), 1);
    }
    if (!touched) {
        s.marks = marks;
        // about 4096 elements a block, at most 2^23 blocks
        const int64_t per = std::max<int64_t>(std::max<int64_t>(4, 4096 / std::max(1, g.dim)), ((int64_t)g.rows >> 23) + 1);
        k_embed_zeros<<<div_up(g.rows, per), GS_BLOCK, 0, st>>>(s, (int)per);
    }
    return hipGetLastError();
}

}  // namespace gsmi
