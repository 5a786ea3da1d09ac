// Lookup of a table's rows by the tokens' ids, and its gradient by sorted tokens.
#include <algorithm>

#include "internal.h"
#include "rows.h"

namespace gsmi {

namespace {

// ---------------------------------------------------------------------------
// out[t] = scale * table[id[t]], 0 where id is outside the table.  A thread
// moves 16-byte pieces of the output.  400,000 tokens of 256 from an fp32 table of
// 32,768 rows take 75 us, bound by the table's rows, which come out of the
// last-level cache 1 KB at a time; the output is written past the caches so that
// they stay there (83 us otherwise).
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
            Span<T, TAIL>::template store<true>(static_cast<T*>(a.out) + (t0 + tok[k]) * a.ld_out + col[k], a.dim - col[k], f[k]);
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
// The sort: passes of at most kMostBits bits, lowest first, each a count of
// digits by block, a scan of the counts, and a scatter whose ranks come from the
// lanes that hold the same digit; a list of one block needs the scatter alone.
// Ids outside the table become `rows`, the last key.
//   300,001 bf16 tokens of 256 in a table of 20,000 rows take 86 us: the sort 32, its
// six launches bound by their latency, the sum 42 (3.7 TB/s of rows gathered), the
// join with the zeros 13.  120,000 fp32 tokens of 64, touched rows of 2,000,000: 56,
// of which the sort 37.  Many tokens of one row cost more than as many of many rows: a
// single workgroup a slab of columns joins their chunks (400,000 tokens of 200 over
// 20,000 rows 83 us, in three rows 107, in one 201).
// ---------------------------------------------------------------------------

constexpr int kMostBits = 11;
constexpr int kMostBins = 1 << kMostBits;
// Sorted items of a thread.  Few fill the units sooner, many leave fewer blocks to
// scan: 300,000 tokens of 8 take 49 us with 4 and 61 with 16, 2^20 the same, four
// million 252 and 197.
constexpr int kFew = 4, kMany = 16;
constexpr int32_t kManyFrom = 1 << 20;
// At most, of the only block's threads, which needs one launch a pass: 2000 tokens
// take 22 us with 8 and 28 in blocks of 4, 4000 30 with 16 and 28.
constexpr int kAlone = 8;

struct SortPass {
    const int32_t* ids;                        // the first pass reads these,
    const uint2* from;                         // the others (key, token) pairs
    uint2* to;
    uint32_t* counts;                          // [bins][blocks]
    uint32_t* totals;                          // [bins]
    uint32_t* marks;                           // first pass: words to clear (NULL: none)
    int32_t n, rows, shift, bits, blocks;
};

__device__ __forceinline__ uint2 sort_item(const SortPass& s, int64_t i) {
    if (s.from) return s.from[i];
    const int32_t id = s.ids[i];
    return make_uint2((uint32_t)id < (uint32_t)s.rows ? (uint32_t)id : (uint32_t)s.rows, (uint32_t)i);
}

// The marks of the rows that have tokens, cleared on the way (k_embed_sum sets them).
__device__ __forceinline__ void clear_marks(const SortPass& s) {
    if (s.marks == nullptr) return;
    const int64_t words = ((int64_t)s.rows + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * GS_BLOCK + threadIdx.x; i < words; i += (int64_t)gridDim.x * GS_BLOCK) s.marks[i] = 0;
}

template <int ITEMS>
__global__ void __launch_bounds__(GS_BLOCK) k_sort_count(SortPass s) {
    __shared__ uint32_t count[kMostBins];
    const int bins = 1 << s.bits;
    const int64_t first = (int64_t)blockIdx.x * (GS_BLOCK * ITEMS) + threadIdx.x;
    uint32_t key[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
        if (first + k * GS_BLOCK < s.n) key[k] = sort_item(s, first + k * GS_BLOCK).x;
    for (int b = threadIdx.x; b < bins; b += GS_BLOCK) count[b] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
        if (first + k * GS_BLOCK < s.n) atomicAdd(&count[(key[k] >> s.shift) & (bins - 1)], 1u);
    clear_marks(s);
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += GS_BLOCK) s.counts[(int64_t)b * s.blocks + blockIdx.x] = count[b];
}

// Exclusive prefixes of each bin's counts over the blocks, a wave a bin.
__global__ void __launch_bounds__(GS_BLOCK) k_sort_scan(SortPass s) {
    const int b = blockIdx.x * (GS_BLOCK / GS_WAVE) + threadIdx.x / GS_WAVE;
    if (b >= 1 << s.bits) return;
    uint32_t* c = s.counts + (int64_t)b * s.blocks;
    uint32_t before = 0;
    for (int i0 = 0; i0 < s.blocks; i0 += 4 * GS_WAVE) {
        uint32_t v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = i0 + j * GS_WAVE + lane_id();
            v[j] = i < s.blocks ? c[i] : 0;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = i0 + j * GS_WAVE + lane_id();
            const uint32_t inc = wave_incl_scan(v[j]);
            if (i < s.blocks) c[i] = before + inc - v[j];
            before += __shfl(inc, GS_WAVE - 1, GS_WAVE);
        }
    }
    if (lane_id() == 0) s.totals[b] = before;
}

// ALONE: the only block, which needs no counts of others.
template <int ITEMS, bool ALONE>
__global__ void __launch_bounds__(GS_BLOCK) k_sort_scatter(SortPass s) {
    constexpr int W = GS_BLOCK / GS_WAVE, MOST = kMostBins / GS_BLOCK;
    __shared__ uint32_t count[W][kMostBins];
    __shared__ uint32_t scratch[W];
    const int bins = 1 << s.bits, w = threadIdx.x / GS_WAVE;
    const int per = max(1, bins / GS_BLOCK);   // bins of a thread
    const int64_t first = (int64_t)blockIdx.x * (GS_BLOCK * ITEMS) + w * (GS_WAVE * ITEMS) + lane_id();
    uint2 item[ITEMS];
    uint32_t rank[ITEMS], tot[MOST], own[MOST];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
        item[k] = first + k * GS_WAVE < s.n ? sort_item(s, first + k * GS_WAVE) : make_uint2(0u, 0u);
#pragma unroll
    for (int j = 0; j < MOST; ++j) {           // where a bin starts, and this block's share of it
        const int b = threadIdx.x * per + j;
        const bool there = !ALONE && j < per && b < bins;
        tot[j] = there ? s.totals[b] : 0u;
        own[j] = there ? s.counts[(int64_t)b * s.blocks + blockIdx.x] : 0u;
    }
    for (int b = threadIdx.x; b < W * bins; b += GS_BLOCK) count[b >> s.bits][b & (bins - 1)] = 0;
    if (ALONE) clear_marks(s);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const bool in = first + k * GS_WAVE < s.n;
        const uint32_t d = (item[k].x >> s.shift) & (bins - 1);
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
    uint32_t sum = 0;
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
        const int b = threadIdx.x * per + j;
        if (j < per && b < bins) {
            if (ALONE)
#pragma unroll
                for (int u = 0; u < W; ++u) tot[j] += count[u][b];
            sum += tot[j];
        }
    }
    uint32_t all, before = block_excl_scan(sum, scratch, &all);
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
        const int b = threadIdx.x * per + j;
        if (j < per && b < bins) {
            uint32_t at = before + own[j];
#pragma unroll
            for (int u = 0; u < W; ++u) {      // wave by wave
                const uint32_t c = count[u][b];
                count[u][b] = at;
                at += c;
            }
            before += tot[j];
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
        if (first + k * GS_WAVE < s.n) s.to[count[w][(item[k].x >> s.shift) & (bins - 1)] + rank[k]] = item[k];
}

// -- the touched rows alone: the sorted keys become places among the unique ids ---

constexpr int kRunItems = 4;                   // of a thread

__device__ __forceinline__ bool run_starts(const uint2* pairs, int64_t i, int32_t n, uint32_t rows) {
    return i < n && pairs[i].x < rows && (i == 0 || pairs[i - 1].x != pairs[i].x);
}

__global__ void __launch_bounds__(GS_BLOCK) k_run_count(const uint2* __restrict__ pairs, int32_t n, uint32_t rows,
                                                        uint32_t* __restrict__ counts) {
    __shared__ uint32_t part[GS_BLOCK / GS_WAVE];
    const int64_t first = (int64_t)blockIdx.x * (GS_BLOCK * kRunItems) + threadIdx.x;
    uint32_t c = 0;
#pragma unroll
    for (int k = 0; k < kRunItems; ++k) c += popc64(__ballot(run_starts(pairs, first + k * GS_BLOCK, n, rows)));
    if (lane_id() == 0) part[threadIdx.x / GS_WAVE] = c;
    __syncthreads();
    if (threadIdx.x == 0) counts[blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

__global__ void __launch_bounds__(GS_BLOCK) k_run_place(const uint2* __restrict__ pairs, int32_t n, uint32_t rows,
                                                        const uint32_t* __restrict__ counts, uint2* __restrict__ to,
                                                        int32_t* __restrict__ unique, int32_t* __restrict__ total) {
    constexpr int W = GS_BLOCK / GS_WAVE;
    __shared__ uint32_t scratch[W], part[kRunItems * W];
    const int64_t first = (int64_t)blockIdx.x * (GS_BLOCK * kRunItems) + threadIdx.x;
    uint64_t starts[kRunItems];
#pragma unroll
    for (int k = 0; k < kRunItems; ++k) {
        starts[k] = __ballot(run_starts(pairs, first + k * GS_BLOCK, n, rows));
        if (lane_id() == 0) part[k * W + threadIdx.x / GS_WAVE] = popc64(starts[k]);
    }
    uint32_t before = block_sum_prefix(counts, blockIdx.x, scratch);       // synchronizes
    for (int i = 0; i < (int)threadIdx.x / GS_WAVE; ++i) before += part[i];
#pragma unroll
    for (int k = 0; k < kRunItems; ++k) {
        const int64_t i = first + k * GS_BLOCK;
        const bool mine = (starts[k] >> lane_id()) & 1;
        const uint32_t place = before + popc64(starts[k] & lanemask_lt()) + mine;          // runs up to here
        if (i < n) {
            const uint2 v = pairs[i];
            to[i] = make_uint2(v.x < rows ? place - 1 : rows, v.y);
            if (mine) unique[place - 1] = (int32_t)v.x;
        }
        if (i == n - 1) *total = (int32_t)place;
        for (int j = 0; j < W && k + 1 < kRunItems; ++j) before += part[k * W + threadIdx.x / GS_WAVE + j];
    }
}

// -- the sums --------------------------------------------------------------------

struct EmbedSum {
    const uint2* pairs;                        // (row of grad, token), sorted
    const void* dout;
    int64_t ld_dout, ld_grad;
    float* grad;
    float* parts;                              // [2 * chunks][dim]: a chunk's first and last row
    uint8_t* marks;                            // rows that have a token (NULL: not wanted)
    int64_t rows;
    int32_t n, dim, per, chunks;               // per: sorted tokens of a chunk
    uint32_t limit;                            // rows from here on are no one's
    float scale;
};

constexpr int kMostChunk = 64;
constexpr int kSum = 64;                       // threads of a workgroup: few, so that the units share the chunks evenly

template <typename T, bool TAIL>
__device__ __forceinline__ void put_row(float* p, int there, const float* f) {
    constexpr int N = Piece<T>::N;
#pragma unroll
    for (int i = 0; i < N; i += 4) Span<float, TAIL>::store(p + i, there - i, f + i);
}

// G lanes a chunk, blockIdx.y: slabs of G * N columns.  The workgroup's pairs go
// to LDS first, then AHEAD rows are on their way while AHEAD are added.
template <typename T, bool TAIL, int G>
__global__ void __launch_bounds__(kSum) k_embed_sum(EmbedSum a) {
    constexpr int N = Piece<T>::N, AHEAD = 8, GROUPS = kSum / G;
    __shared__ uint2 list[GROUPS * kMostChunk + 2];        // from the position in front of the workgroup's first
    const int64_t base = (int64_t)blockIdx.x * GROUPS * a.per;
    const int count = (int)min((int64_t)GROUPS * a.per, (int64_t)a.n - base);
    for (int i = threadIdx.x; i < count + 2; i += kSum) {
        const int64_t p = base + i - 1;
        list[i] = p >= 0 && p < a.n ? a.pairs[p] : make_uint2(a.limit, 0u);
    }
    __syncthreads();
    const int col = blockIdx.y * (G * N) + (threadIdx.x % G) * N, there = a.dim - col;
    const int64_t g = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G;
    const int p0 = 1 + threadIdx.x / G * a.per, p1 = min(p0 + a.per, count + 1);
    if (p0 >= p1) return;
    const uint32_t before = list[p0 - 1].x, after = list[p1].x;
    uint32_t row = list[p0].x;
    bool shared = row == before;               // with the chunk in front
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.0f;
    auto flush = [&](bool last) {
        if (row >= a.limit) return;
        const bool goes_on = last && row == after, whole = !shared && !goes_on;
        float* to = a.grad + (int64_t)row * a.ld_grad + col;
        if (!whole) to = a.parts + (2 * g + (shared ? 0 : 1)) * a.dim + col;
        if (a.marks && !shared && threadIdx.x % G == 0) a.marks[row] = 1;
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = whole ? acc[i] * a.scale : acc[i];
        put_row<T, TAIL>(to, there, v);
    };
    Span<T, TAIL> now[AHEAD], next[AHEAD];
    auto load = [&](Span<T, TAIL>* s, int p) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const uint2 v = list[min(p + k, p1 - 1)];
            s[k].load(static_cast<const T*>(a.dout) + (int64_t)v.y * a.ld_dout + col,
                      p + k < p1 && v.x < a.limit ? there : 0);
        }
    };
    auto add = [&](const Span<T, TAIL>* s, int p) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const uint32_t mine = list[min(p + k, p1 - 1)].x;          // past the end: the last row, nothing to add
            if (mine != row) {
                flush(false);
                row = mine;
                shared = false;
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] = 0.0f;
            }
            float f[N];
            s[k].floats(f);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] += f[i];
        }
    };
    load(now, p0);
    for (int p = p0; p < p1; p += 2 * AHEAD) {
        load(next, p + AHEAD);
        add(now, p);
        if (p + AHEAD >= p1) break;
        load(now, p + 2 * AHEAD);
        add(next, p + AHEAD);
    }
    flush(true);
}

// Sums of the partial rows of a run, from the chunk that holds its start: the
// last row of that chunk, then the first rows of those behind it.  A group of
// lanes takes a run of few chunks; the workgroup together one of many, in equal
// slices that are added in ascending order.  A slice's sum moves to 64 bits every
// kShort chunks: in 32 throughout, a row's sum loses a bit with every doubling of
// its tokens (400,000 equal numbers came out 8e-6 off, 2^28 would by 0.4%).
// Workgroups behind these write zeros to the rows that have no token.
// Threads of the join.  256 take 330 us for those 201, and 134 for the zeros of
// 1,271,665 rows of 80 (512: 120).
constexpr int kJoin = 512;
constexpr int kShort = 64;                     // chunks of a run that a group joins alone: 32 and 128 are within 1%

template <typename T, bool TAIL, int G>
__global__ void __launch_bounds__(kJoin) k_embed_join(EmbedSum a, int join_blocks, int rows_a_block) {
    constexpr int N = Piece<T>::N, GROUPS = kJoin / G;
    __shared__ double sums[GROUPS][N][G];
    __shared__ int many[GROUPS], n_many, ends;
    if ((int)blockIdx.x >= join_blocks) {
        if (blockIdx.y > 0) return;
        const int64_t r0 = (int64_t)(blockIdx.x - join_blocks) * rows_a_block, r1 = min(r0 + rows_a_block, a.rows);
        // pieces of four floats, each thread its own row's mark
        const int pieces = (a.dim + 3) / 4, items = (int)(r1 - r0) * pieces;
        const float inv = 1.0f / (float)pieces, none[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int i = threadIdx.x; i < items; i += kJoin) {
            const int r = (int)(((float)i + 0.5f) * inv), c = (i - r * pieces) * 4;   // fewer than 2^18 items
            if (a.marks && a.marks[r0 + r]) continue;
            Span<float, TAIL>::template store<true>(a.grad + (r0 + r) * a.ld_grad + c, a.dim - c, none);
        }
        return;
    }
    const int group = threadIdx.x / G, lane = threadIdx.x % G;
    const int col = blockIdx.y * (G * N) + lane * N, there = a.dim - col;
    if (threadIdx.x == 0) n_many = 0;
    __syncthreads();
    const int64_t g = (int64_t)blockIdx.x * GROUPS + group, p0 = g * a.per, p1 = p0 + a.per;
    // whether a run starts here and goes on, and how many chunks behind this one it reaches
    uint32_t row = a.limit;
    bool mine = p1 < a.n;
    if (mine) {
        const uint32_t last = a.pairs[p1 - 1].x, next = a.pairs[p1].x, first = a.pairs[p0].x;
        const uint32_t front = p0 > 0 ? a.pairs[p0 - 1].x : a.limit;
        row = last;
        mine = last < a.limit && next == last && !(first == last && front == last);
    }
    // a run ends in chunk c if the position behind c is another row's
    auto ends_in = [&](int64_t c, uint32_t row) { return (c + 1) * a.per >= a.n || a.pairs[(c + 1) * a.per].x != row; };
    const int lane0 = lane_id() / G * G;
    const uint64_t lanes = G == GS_WAVE ? ~0ull : ((1ull << G) - 1) << lane0;
    int m = 0;
    for (int c = 0; c < kShort; c += G) {
        const bool looks = mine && m == 0;
        if (!__any(looks)) break;
        const uint64_t ending = __ballot(looks && ends_in(g + 1 + c + lane, row)) & lanes;
        if (looks && ending) m = c + __ffsll((unsigned long long)ending) - lane0;
    }
    auto add = [&](float* acc, const float* p) {
        float f[N];
        load_floats<N, TAIL>(p + col, 0, there, f);
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] += f[i];
    };
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.0f;
    if (mine && m > 0) {
        add(acc, a.parts + (2 * g + 1) * a.dim);
#pragma unroll 8
        for (int j = 1; j <= m; ++j) add(acc, a.parts + 2 * (g + j) * a.dim);
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] *= a.scale;
        put_row<T, TAIL>(a.grad + (int64_t)row * a.ld_grad + col, there, acc);
    }
    if (mine && m == 0 && lane == 0) many[atomicAdd(&n_many, 1)] = group;
    __syncthreads();
    const int runs = n_many;
    for (int k = 0; k < runs; ++k) {
        const int64_t c0 = (int64_t)blockIdx.x * GROUPS + many[k];
        const uint32_t run = a.pairs[(c0 + 1) * a.per - 1].x;
        int64_t chunks = 0;                    // behind c0
        for (int64_t c = c0 + 1; chunks == 0; c += kJoin) {
            if (threadIdx.x == 0) ends = kJoin;
            __syncthreads();
            if (ends_in(c + threadIdx.x, run)) atomicMin(&ends, (int)threadIdx.x);
            __syncthreads();
            if (ends < kJoin) chunks = c + ends - c0;
            __syncthreads();
        }
        const int64_t per = (chunks + GROUPS - 1) / GROUPS, last = min((group + 1) * per, chunks);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            acc[i] = 0.0f;
            sums[group][i][lane] = 0.0;
        }
        if (group == 0) add(acc, a.parts + (2 * c0 + 1) * a.dim);
        for (int64_t j0 = group * per; j0 < last; j0 += kShort) {
            const int n = (int)min((int64_t)kShort, last - j0);
            const float* p = a.parts + 2 * (c0 + 1 + j0) * a.dim;
#pragma unroll 8
            for (int j = 0; j < n; ++j, p += 2 * a.dim) add(acc, p);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                sums[group][i][lane] += acc[i];
                acc[i] = 0.0f;
            }
        }
        __syncthreads();
        if (threadIdx.x < G * N) {             // a column each
            double sum = 0.0;
#pragma unroll 8
            for (int u = 0; u < GROUPS; ++u) sum += sums[u][threadIdx.x % N][threadIdx.x / N];
            const int to = blockIdx.y * (G * N) + threadIdx.x;
            if (to < a.dim) a.grad[(int64_t)run * a.ld_grad + to] = (float)sum * a.scale;
        }
        __syncthreads();
    }
}

__global__ void k_zero_words(uint32_t* p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) p[i] = 0;
}

struct EmbedPlan {
    int32_t bits, passes, digit, blocks, per, chunks;
    bool many;
    size_t pairs[2], counts, totals, marks, parts, bytes;
};

// Lanes that walk a chunk together: a power of two that holds the row's 16-byte pieces.
inline int chunk_lanes(int32_t dim, int n) {
    int g = 4;
    while (g < GS_WAVE && g * n < dim) g *= 2;
    return g;
}

EmbedPlan embed_plan(int32_t n, int32_t rows, int32_t dim, int32_t size, bool touched) {
    EmbedPlan p;
    p.bits = 1;
    while (p.bits < 31 && (uint32_t)rows >> p.bits) ++p.bits;              // of the key `rows`
    p.passes = (p.bits + kMostBits - 1) / kMostBits;
    p.digit = (p.bits + p.passes - 1) / p.passes;
    p.many = n >= kManyFrom;
    p.blocks = n <= GS_BLOCK * kAlone ? 1 : (int32_t)div_up(n, GS_BLOCK * (p.many ? kMany : kFew));
    // Chunks as long as leaves 1024 waves: longer ones have fewer ends that others share
    // (120,000 touched rows 57 us; with 512 waves 60, with 2048 56; 400,000 tokens the same).
    const int elements = 16 / size, lanes = chunk_lanes(dim, elements);
    const int64_t waves = (int64_t)n * lanes / GS_WAVE * div_up(dim, lanes * elements);
    p.per = kMostChunk;
    while (p.per > 8 && waves / p.per < 1024) p.per /= 2;
    p.chunks = (int32_t)div_up(n, p.per);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align256(bytes);
        return here;
    };
    p.pairs[0] = take((size_t)n * 8);
    p.pairs[1] = take((size_t)n * 8);
    // counts of the sort, then of the runs
    p.counts = take(std::max(((size_t)p.blocks << p.digit) * 4, (size_t)div_up(n, GS_BLOCK * kRunItems) * 4 + 16));
    p.totals = take((size_t)kMostBins * 4);
    p.marks = take(touched ? 0 : (size_t)rows + 4);
    p.parts = take((size_t)p.chunks * 2 * dim * 4);
    p.bytes = at;
    return p;
}

template <typename T, bool TAIL, int G>
hipError_t sum_go(const EmbedSum& a, int zero_blocks, int rows_a_block, hipStream_t st) {
    const uint32_t slabs = div_up(a.dim, G * Piece<T>::N);
    k_embed_sum<T, TAIL, G><<<dim3(div_up(a.chunks, kSum / G), slabs), kSum, 0, st>>>(a);
    const int join = a.chunks > 1 ? (int)div_up(a.chunks, kJoin / G) : 0;
    if (join + zero_blocks > 0)
        k_embed_join<T, TAIL, G><<<dim3(join + zero_blocks, slabs), kJoin, 0, st>>>(a, join, rows_a_block);
    return hipGetLastError();
}

template <typename T, bool TAIL>
hipError_t sum_lanes(const EmbedSum& a, int zero_blocks, int rows_a_block, hipStream_t st) {
    switch (chunk_lanes(a.dim, Piece<T>::N)) {
        case 4: return sum_go<T, TAIL, 4>(a, zero_blocks, rows_a_block, st);
        case 8: return sum_go<T, TAIL, 8>(a, zero_blocks, rows_a_block, st);
        case 16: return sum_go<T, TAIL, 16>(a, zero_blocks, rows_a_block, st);
        case 32: return sum_go<T, TAIL, 32>(a, zero_blocks, rows_a_block, st);
        default: return sum_go<T, TAIL, 64>(a, zero_blocks, rows_a_block, st);
    }
}

template <typename T>
hipError_t sum_type(const EmbedSum& a, int zero_blocks, int rows_a_block, hipStream_t st) {
    return a.dim % Piece<T>::N ? sum_lanes<T, true>(a, zero_blocks, rows_a_block, st)
                               : sum_lanes<T, false>(a, zero_blocks, rows_a_block, st);
}

void sort_pass(const SortPass& q, bool many, hipStream_t st) {
    if (q.blocks == 1) {
        if (q.n <= GS_BLOCK * kFew) k_sort_scatter<kFew, true><<<1, GS_BLOCK, 0, st>>>(q);
        else k_sort_scatter<kAlone, true><<<1, GS_BLOCK, 0, st>>>(q);
        return;
    }
    if (many) k_sort_count<kMany><<<q.blocks, GS_BLOCK, 0, st>>>(q);
    else k_sort_count<kFew><<<q.blocks, GS_BLOCK, 0, st>>>(q);
    k_sort_scan<<<div_up(1u << q.bits, GS_BLOCK / GS_WAVE), GS_BLOCK, 0, st>>>(q);
    if (many) k_sort_scatter<kMany, false><<<q.blocks, GS_BLOCK, 0, st>>>(q);
    else k_sort_scatter<kFew, false><<<q.blocks, GS_BLOCK, 0, st>>>(q);
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

// For the most that any type's kernels take.
size_t embedding_bwd_ws_bytes(int32_t tokens, int32_t rows, int32_t dim, bool touched) {
    return std::max(embed_plan(tokens, rows, dim, 2, touched).bytes, embed_plan(tokens, rows, dim, 4, touched).bytes);
}

hipError_t launch_embedding_bwd(const gs_embed_bwd_args& g, void* ws, hipStream_t st) {
    const bool touched = g.unique != nullptr;
    const EmbedPlan p = embed_plan(g.tokens, g.rows, g.dim, g.dtype == GS_F32 ? 4 : 2, touched);
    char* base = static_cast<char*>(ws);
    EmbedSum s;
    s.pairs = nullptr;
    s.dout = g.dout;
    s.ld_dout = g.ld_dout;
    s.ld_grad = g.ld_grad;
    s.grad = g.grad;
    s.parts = reinterpret_cast<float*>(base + p.parts);
    s.marks = touched || g.tokens == 0 ? nullptr : reinterpret_cast<uint8_t*>(base + p.marks);
    s.rows = g.rows;
    s.n = g.tokens;
    s.dim = g.dim;
    s.per = p.per;
    s.chunks = p.chunks;
    s.limit = (uint32_t)g.rows;
    s.scale = g.scale;
    // rows without a token: 2^14 elements a workgroup (a row at least; 2^22 workgroups at most)
    const int64_t rows_a_block = std::max<int64_t>(std::max<int64_t>(1, 16384 / g.dim), ((int64_t)g.rows >> 22) + 1);
    const int zero_blocks = touched ? 0 : (int)div_up(g.rows, rows_a_block);
    if (g.tokens == 0) {
        if (touched) k_zero_words<<<1, 1, 0, st>>>(reinterpret_cast<uint32_t*>(g.count), 1);
        else k_embed_join<float, true, 64><<<zero_blocks, kJoin, 0, st>>>(s, 0, (int)rows_a_block);
        return hipGetLastError();
    }
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
        q.marks = i ? nullptr : reinterpret_cast<uint32_t*>(s.marks);
        q.n = g.tokens;
        q.rows = g.rows;
        q.shift = i * p.digit;
        q.bits = std::min(p.digit, p.bits - i * p.digit);
        q.blocks = p.blocks;
        sort_pass(q, p.many, st);
    }
    s.pairs = buf[at ^ 1];
    if (touched) {
        const uint32_t blocks = div_up(g.tokens, GS_BLOCK * kRunItems);
        k_run_count<<<blocks, GS_BLOCK, 0, st>>>(s.pairs, g.tokens, (uint32_t)g.rows, counts);
        k_run_place<<<blocks, GS_BLOCK, 0, st>>>(s.pairs, g.tokens, (uint32_t)g.rows, counts, buf[at], g.unique, g.count);
        s.pairs = buf[at];
    }
    if (g.dtype == GS_F32) return sum_type<float>(s, zero_blocks, (int)rows_a_block, st);
    return g.dtype == GS_BF16 ? sum_type<bf16_t>(s, zero_blocks, (int)rows_a_block, st)
                              : sum_type<f16_t>(s, zero_blocks, (int)rows_a_block, st);
}

}  // namespace gsmi
