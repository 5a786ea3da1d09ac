// Pieces that the attention kernels share (device code; gfx950).
//
// Matrix products run on v_mfma_f32_32x32x16 (16-bit operands, fp32 sums):
//   A [32 x 16]: lane l holds row l & 31, elements 8 (l >> 5) .. +7 of the 16;
//   B [16 x 32]: lane l holds column l & 31, the same 8 of the 16;
//   C [32 x 32]: lane l holds column l & 31; its register r is row
//     8 (r >> 2) + 4 (l >> 5) + (r & 3).
// A sum over the 16 takes them in any order as long as A and B agree.  So
// registers 8u .. 8u+7 of a C tile, rounded to 16 bits, are the B operand (or,
// the tile being its own transpose's A) of a product over the tile's rows
// 16u .. 16u+15, in the order 16u + 8 (i >> 2) + 4 (l >> 5) + (i & 3) for
// element i: softmax probabilities go from one product into the next without
// leaving their lane.
#pragma once

#include "common.h"
#include "internal.h"
#include "vec16.h"

namespace gsmi {

typedef float acc16 __attribute__((ext_vector_type(16)));

template <typename T>
using op8 = T __attribute__((ext_vector_type(8)));
template <typename T>
using op4 = T __attribute__((ext_vector_type(4)));

__device__ __forceinline__ acc16 mfma(op8<bf16_t> a, op8<bf16_t> b, acc16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ acc16 mfma(op8<f16_t> a, op8<f16_t> b, acc16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// The values of the lanes l & 31 and (l & 31) + 32.
__device__ __forceinline__ float2 halves(float v) {
#ifdef __HIP_DEVICE_COMPILE__
    // swaps the upper half of the first with the lower half of the second: of
    // two copies, one is left with the lower half twice, one with the upper
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
#else
    return make_float2(v, v);
#endif
}

// A tile of token rows in LDS: rows of P elements (a power of two), each cut
// into 16-byte pieces that are stored at piece ^ key(row).  Two readers have
// to find their 64 lanes' pieces in different banks: one takes the same piece
// of 32 rows (16 bytes a lane), the other 64 bytes of each of four adjacent
// rows (transposed, 8 bytes a lane).  With 16 pieces a row, row & 3 in the upper
// two bits of the key spreads four adjacent rows over the 256 bytes of all
// banks, and (row >> 2) & 3 below spreads the next ones; with 8 and 4 pieces,
// two and four rows share 256 bytes and fewer bits are left to set.
template <int P>
__device__ __forceinline__ int piece_key(int row) {
    if (P == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
    if (P == 64) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    return (row >> 2) & 3;
}

// Elements between the tile's start and 16-byte piece `piece` of row `row`.
template <int P>
__device__ __forceinline__ int piece_at(int row, int piece) {
    return row * P + ((piece ^ piece_key<P>(row)) << 3);
}

// Transposed read of four rows by sixteen columns for every group of 16 lanes:
// lane l of the group points at four elements of row l >> 2, column 4 (l & 3),
// and gets the four rows' elements of column l.
typedef short s4 __attribute__((ext_vector_type(4)));
template <typename T>
__device__ __forceinline__ op4<T> read_columns(const T* p) {
    const s4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s4*)(const_cast<T*>(p)));
    return __builtin_bit_cast(op4<T>, v);
}

// The same value, of which the compiler knows nothing: what follows from it is
// computed where it is used.  Otherwise the sums of a lane's places and every
// tile's start are kept in a register each over a whole loop, in place of the
// instruction's offset.
__device__ __forceinline__ int fresh(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// Where a lane's pieces of a tile are, in bytes: `rows` for operands made of the
// tile's rows, `cols` for those made of its columns.  The key only moves 16-byte
// pieces within a row, so the other places follow by an exclusive or: 32 t for
// the t-th 16 elements of a row, 64 d for columns 32 d on, 32 for the rows 8
// below.
struct Lanes {
    int rows, cols;

    template <int P>
    __device__ __forceinline__ void init() {
        const int l = lane_id();
        rows = 2 * piece_at<P>(l & 31, l >> 5);
        cols = 2 * piece_at<P>(4 * (l >> 5) + ((l & 15) >> 2), 2 * ((l >> 4) & 1) + ((l & 3) >> 1)) + 8 * (l & 1);
    }
    __device__ __forceinline__ void refresh() {
        rows = fresh(rows);
        cols = fresh(cols);
    }
};

// A operand from the columns of a tile: rows (of the operand) are the tile's
// columns 32 d .. +31, the 16 of the sum are its rows row0 .. row0+15 in the
// order a C tile's registers have.
template <typename T, int P>
__device__ __forceinline__ op8<T> columns_operand(const T* tile, const Lanes& at, int row0, int d) {
    const char* p = reinterpret_cast<const char*>(tile) + row0 * P * 2;
    const op4<T> lo = read_columns(reinterpret_cast<const T*>(p + (at.cols ^ (64 * d))));
    const op4<T> hi = read_columns(reinterpret_cast<const T*>(p + 16 * P + (at.cols ^ (64 * d) ^ 32)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// A or B operand from the rows of a tile: lane l gets row row0 + (l & 31),
// elements 16 t + 8 (l >> 5) .. +7.
template <typename T, int P>
__device__ __forceinline__ op8<T> rows_operand(const T* tile, const Lanes& at, int row0, int t) {
    const char* p = reinterpret_cast<const char*>(tile) + row0 * P * 2;
    return *reinterpret_cast<const op8<T>*>(p + (at.rows ^ (32 * t)));
}

// Registers 8u .. 8u+7 of a C tile as an operand.
template <typename T>
__device__ __forceinline__ op8<T> tile_operand(const acc16& c, int u) {
    op8<T> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (T)c[8 * u + i];
    return o;
}

// The rows of a segment as a buffer: a load outside of it (a row at or past the
// segment's end, or kOutside for a lane that wants nothing) gives zeros.  One
// descriptor serves the rows of 2^29 bytes, then it moves on.
template <typename T>
struct RowBuffer {
    static constexpr int kRange = 0x7FFFFF00, kOutside = 0x7FFFFFF0;
    const T* base;                         // the segment's first row
    const T* from;                         // the descriptor's: row `row0`
    int rows, row0, bytes, ld;             // ld: bytes of a row

    __device__ __forceinline__ void rebase(int row) {
        row0 = row;
        from = base + (int64_t)row * (ld / 2);
        bytes = (int)max((int64_t)0, min((int64_t)kRange, (int64_t)(rows - row) * ld));
    }
    __device__ __forceinline__ void init(const T* first, int n, int64_t row_stride) {
        base = first;
        rows = n;
        ld = (int)row_stride * 2;
        rebase(0);
    }
    // Bytes from the descriptor's start to row `row`.
    __device__ __forceinline__ int place(int row) {
        if ((uint64_t)((int64_t)(row - row0) * ld) >= 1u << 29) rebase(row);
        return (row - row0) * ld;
    }
    // 16 bytes at `at` into registers.
    __device__ __forceinline__ op8<T> piece(int at) const {
#ifdef __HIP_DEVICE_COMPILE__              // the host pass has no buffer descriptors
        typedef uint32_t u4 __attribute__((ext_vector_type(4)));
        const u4 v = __builtin_amdgcn_raw_buffer_load_b128(
            __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(from), 0, bytes, 0x00027000), at, 0, 0);
        return __builtin_bit_cast(op8<T>, v);
#else
        return op8<T>{};
#endif
    }
    // 16 bytes a lane into LDS, in lane order from `to` on.
    __device__ __forceinline__ void piece_to(T* to, int at) const {
#ifdef __HIP_DEVICE_COMPILE__
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(from), 0, bytes, 0x00027000),
            (__attribute__((address_space(3))) void*)to, 16, at, 0, 0, 0);
#endif
    }
};

// Copies tiles of ROWS token rows from memory into LDS without passing through
// registers: each of the LOADS instructions of a wave fills 1 KB, 16 bytes a
// lane in lane order, so the lane that fills a piece's place reads the piece
// that belongs there.  Rows past the segment's end and pieces past the head's
// end arrive as zeros.
template <typename T, int P, int ROWS>
struct TileLoader {
    static constexpr int PIECES = P / 8, LOADS = ROWS * PIECES / GS_BLOCK, STEP = GS_BLOCK / PIECES;
    static_assert(STEP % 16 == 0, "the key repeats every 16 rows: a lane's loads differ by whole rows");
    RowBuffer<T> buf;
    int off;                               // a lane's place from a tile's first row

    __device__ __forceinline__ void init(const T* first, int n, int64_t row_stride, int dim) {
        buf.init(first, n, row_stride);
        const int row = threadIdx.x / PIECES, piece = (threadIdx.x % PIECES) ^ piece_key<P>(row);
        off = 8 * piece < dim ? row * buf.ld + piece * 16 : buf.kOutside;
    }
    // On to another list of as many rows.
    __device__ __forceinline__ void move(const T* first) {
        buf.base = first;
        buf.rebase(0);
    }
    // row: the tile's first; skip: bit u leaves load u's row out (zeros).
    __device__ __forceinline__ void load(T* tile, int row, uint32_t skip) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / GS_WAVE);
        const int at = buf.place(row);
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            // past the range also where `off` is; below 2^32, so the sum is one of unsigned numbers
            const int place = (int)((uint32_t)off + (uint32_t)(at + u * STEP * buf.ld));
            buf.piece_to(tile + (u * GS_BLOCK + wave * GS_WAVE) * 8, (skip >> u) & 1 ? buf.kOutside : place);
        }
    }
};

// 64 words from `base` on into LDS, a lane of the wave each; those at or past
// `n` are zeros.
__device__ __forceinline__ void load_words(float* to, const float* base, int n) {
#ifdef __HIP_DEVICE_COMPILE__
    const __amdgpu_buffer_rsrc_t buf =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(base), 0, min(n, 1 << 16) * 4, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void*)to, 4, lane_id() * 4, 0, 0,
                                             0);
#endif
}

// TileLoader's skip bits from a tile's rows, bit r of `on` for row r (up to 64).
template <int P, int ROWS>
__device__ __forceinline__ uint32_t rows_off(uint64_t on) {
    constexpr int PIECES = P / 8, LOADS = ROWS * PIECES / GS_BLOCK;
    const int first = fresh(threadIdx.x) / PIECES;
    uint32_t skip = 0;
#pragma unroll
    for (int u = 0; u < LOADS; ++u) skip |= (uint32_t)(~(on >> (first + u * (GS_BLOCK / PIECES))) & 1) << u;
    return skip;
}

// Flag of key `key` of a segment whose flags start at `on` (0 past its end).
__device__ __forceinline__ uint8_t key_flag(const uint8_t* on, int key, int n) { return key < n ? on[key] : 0; }

// Bits [lo, hi) of 64, ends clamped.
__device__ __forceinline__ uint64_t bits_between(int lo, int hi) {
    const uint64_t below = hi <= 0 ? 0ull : (hi >= 64 ? ~0ull : (1ull << hi) - 1);
    return lo <= 0 ? below : (lo >= 64 ? 0ull : below & (~0ull << lo));
}

// -inf into a C tile's elements whose row (register e of half h is row 8 (e >> 2)
// + (e & 3) + 4 h) has its bit off in the lane's `seen`: two instructions each.
__device__ __forceinline__ void keep_some(acc16& s, uint32_t seen) {
    const uint32_t mine = seen >> (4 * (lane_id() >> 5));
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const uint32_t m = (int32_t)(mine << (31 - 8 * (e >> 2) - (e & 3))) >> 31;
        s[e] = __uint_as_float((__float_as_uint(s[e]) & m) | (0xFF800000u & ~m));
    }
}

struct AttnArgs {
    const void *q, *k, *v;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;
    const int32_t *cu_q, *cu_k;
    const uint8_t* key_on;
    int32_t n_q, n_k, n_seg, heads, kv_heads, group, dim, left, right;
    float scale;
    int32_t tiles;             // workgroups' tiles per key head
    int32_t fill;              // rows outside every segment are written
};

// Row stride of a tensor of n rows.  The only row of one has no next: any value
// may stand there, and RowBuffer takes a row's bytes from it.
inline int64_t row_stride(const gs_rows& r, int32_t n, int32_t dim) { return n == 1 ? dim : r.ld_row; }

inline AttnArgs attn_args(const gs_attn& a) {
    AttnArgs r;
    r.q = a.q.ptr;
    r.k = a.k.ptr;
    r.v = a.v.ptr;
    r.q_row = row_stride(a.q, a.n_q, a.dim);
    r.q_head = a.q.ld_head;
    r.k_row = row_stride(a.k, a.n_k, a.dim);
    r.k_head = a.k.ld_head;
    r.v_row = row_stride(a.v, a.n_k, a.dim);
    r.v_head = a.v.ld_head;
    r.cu_q = a.cu_q;
    r.cu_k = a.cu_k;
    r.key_on = a.key_on;
    r.n_q = a.n_q;
    r.n_k = a.n_k;
    r.n_seg = a.n_seg;
    r.heads = a.heads;
    r.kv_heads = a.kv_heads;
    r.group = a.heads / a.kv_heads;
    r.dim = a.dim;
    r.left = a.left;
    r.right = a.right;
    r.scale = a.scale;
    r.tiles = 0;
    r.fill = (a.dtype & GS_ATTN_FILL) != 0 && a.cu_q != nullptr;
    return r;
}

// Tiles of `size` rows (or keys) over ragged segments whose lengths only the
// device knows, for rows / size + n_seg tiles at most.
struct Segment {
    int q0, nq, k0, nk;        // first row and rows of the queries and keys
    int tile;                  // the tile's number within the segment
};

__device__ __forceinline__ int cu_at(const int32_t* cu, int s, int n_seg, int n) {
    if (cu == nullptr) return n / n_seg * s;
    return min(max(cu[s], 0), n);
}

__device__ __forceinline__ int of_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// KEYS: the keys are tiled, a token each; otherwise the query rows, `group` of
// them a token.  LAST_FIRST: a segment's last tile comes first (with ordered
// keys it has the most to do).
//   Up to 64 segments: a lane holds each, and the tiles are numbered from the
// segment with the longest other side on, so that the workgroups with the most
// steps start first.  A loop over the segments gives every lane its first tile.
//   More: segment s starts at tile start(s) / size + s, at least as many tiles as
// its rows need (some stay empty), found by a search with 64 probes a round.
// EMPTY_TOO: a segment without any has one tile all the same.
template <bool KEYS, bool LAST_FIRST, bool EMPTY_TOO = false>
__device__ __forceinline__ Segment find_segment(const AttnArgs& a, int size, int tiles, int tile) {
    const int lane = lane_id(), mul = KEYS ? 1 : a.group;
    Segment s;
    if (a.n_seg <= GS_WAVE) {
        const int at = min(lane, a.n_seg - 1);
        const int q0 = cu_at(a.cu_q, at, a.n_seg, a.n_q), k0 = cu_at(a.cu_k, at, a.n_seg, a.n_k);
        const int nq = max(cu_at(a.cu_q, at + 1, a.n_seg, a.n_q) - q0, 0);
        const int nk = max(cu_at(a.cu_k, at + 1, a.n_seg, a.n_k) - k0, 0);
        int has = (int)(((KEYS ? (int64_t)nk : (int64_t)nq * mul) + size - 1) / size);
        if (EMPTY_TOO) has = max(has, 1);
        if (lane >= a.n_seg) has = 0;
        const int work = KEYS ? nq : nk;
        int first = 0;
        for (int t = 0; t < a.n_seg; ++t) {
            const int w = of_lane(work, t), n = of_lane(has, t);
            first += w > work || (w == work && t < lane) ? n : 0;
        }
        const uint64_t hit = __ballot(tile >= first && tile - first < has);
        if (hit == 0) return Segment{0, 0, 0, 0, 0};
        const int l = __builtin_ctzll(hit);
        s.q0 = of_lane(q0, l);
        s.nq = of_lane(nq, l);
        s.k0 = of_lane(k0, l);
        s.nk = of_lane(nk, l);
        s.tile = tile - of_lane(first, l);
        if (LAST_FIRST) s.tile = of_lane(has, l) - 1 - s.tile;
        return s;
    }
    if (LAST_FIRST) tile = tiles - 1 - tile;
    const int32_t* cu = KEYS ? a.cu_k : a.cu_q;
    const int n = KEYS ? a.n_k : a.n_q;
    int lo = 0, hi = a.n_seg - 1;          // the last segment whose first tile is at or before `tile`
    while (lo < hi) {
        const int step = (hi - lo + GS_WAVE - 1) / GS_WAVE;
        const int m = lo + (lane + 1) * step;
        const bool before = m <= hi && (int)((int64_t)cu_at(cu, m, a.n_seg, n) * mul / size) + m <= tile;
        lo += __popcll(__ballot(before)) * step;
        hi = min(hi, lo + step - 1);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);           // the same in every lane: held in scalar registers
    s.q0 = __builtin_amdgcn_readfirstlane(cu_at(a.cu_q, lo, a.n_seg, a.n_q));
    s.nq = __builtin_amdgcn_readfirstlane(max(cu_at(a.cu_q, lo + 1, a.n_seg, a.n_q) - s.q0, 0));
    s.k0 = __builtin_amdgcn_readfirstlane(cu_at(a.cu_k, lo, a.n_seg, a.n_k));
    s.nk = __builtin_amdgcn_readfirstlane(max(cu_at(a.cu_k, lo + 1, a.n_seg, a.n_k) - s.k0, 0));
    s.tile = tile - __builtin_amdgcn_readfirstlane((int)((int64_t)cu_at(cu, lo, a.n_seg, n) * mul / size) + lo);
    return s;
}

// Keys of the segment that a token of the queries is in; -1 for none.
__device__ __forceinline__ int keys_of_token(const AttnArgs& a, int token) {
    int lo = 0, hi = a.n_seg - 1;          // the last segment that starts at or before the token
    while (lo < hi) {
        const int step = (hi - lo + GS_WAVE - 1) / GS_WAVE;
        const int m = lo + (lane_id() + 1) * step;
        lo += __popcll(__ballot(m <= hi && cu_at(a.cu_q, m, a.n_seg, a.n_q) <= token)) * step;
        hi = min(hi, lo + step - 1);
    }
    if (token < cu_at(a.cu_q, lo, a.n_seg, a.n_q) || token >= cu_at(a.cu_q, lo + 1, a.n_seg, a.n_q)) return -1;
    return max(cu_at(a.cu_k, lo + 1, a.n_seg, a.n_k) - cu_at(a.cu_k, lo, a.n_seg, a.n_k), 0);
}

// Zeros into the rows outside every segment of a matrix of n rows (those before
// the first start and from the last on), by all of the launch's workgroups;
// lse, if given, takes -inf.
template <typename T>
__device__ __forceinline__ void fill_rest(const AttnArgs& a, const int32_t* cu, int n, int heads, T* p, int64_t ld_row,
                                          int64_t ld_head, float* lse) {
    const int first = cu_at(cu, 0, a.n_seg, n), held = max(cu_at(cu, a.n_seg, a.n_seg, n) - first, 0), rest = n - held;
    if (rest == 0) return;
    const int per = a.dim / 8;
    const int64_t pieces = (int64_t)rest * heads * per, step = (int64_t)gridDim.x * GS_BLOCK;
#pragma unroll 1
    for (int64_t x = (int64_t)blockIdx.x * GS_BLOCK + threadIdx.x; x < pieces; x += step) {
        const int64_t y = x / per;
        const int c = (int)(x - y * per), i = (int)(y / heads), head = (int)(y - (int64_t)i * heads);
        const int64_t row = i < first ? i : i + held;
        *reinterpret_cast<op8<T>*>(p + row * ld_row + head * ld_head + 8 * c) = op8<T>{};
        if (lse != nullptr && c == 0) lse[row * heads + head] = -INFINITY;
    }
}

// Keys [lo, hi) that any of the places first .. last can admit.
__device__ __forceinline__ void admitted(const AttnArgs& a, int nk, int first, int last, int& lo, int& hi) {
    lo = a.left >= 0 ? max((int64_t)0, (int64_t)first - a.left) : 0;
    hi = a.right >= 0 ? min((int64_t)nk, (int64_t)last + a.right + 1) : nk;
}

// Tokens [lo, hi) that admit any of the keys first .. last.
__device__ __forceinline__ void admitting(const AttnArgs& a, int nq, int shift, int first, int last, int& lo, int& hi) {
    lo = a.right >= 0 ? (int)max((int64_t)0, min((int64_t)nq, (int64_t)first - a.right - shift)) : 0;
    hi = a.left >= 0 ? (int)max((int64_t)0, min((int64_t)nq, (int64_t)last + a.left - shift + 1)) : nq;
}

inline int attn_tiles(int64_t rows, int size, int n_seg) { return (int)(rows / size) + n_seg; }

// Order of the workgroups.  Consecutive ids go to the eight chiplets in turn,
// each with its own L2, so the list of (key head, tile) is cut into eight runs:
// the tiles that read the same keys stay on one chiplet.  Where a run is less
// than a head or not whole heads, a head's tiles are dealt into 8 / gcd(8,
// heads) equal shares, every so many-th tile, so that no chiplet gets all the
// long ones (ordered keys: the last rows; dealt in runs, one chiplet had three
// times another's work).
inline int chiplet_shares(int heads) {
    return heads % 8 == 0 ? 1 : (heads % 4 == 0 ? 2 : (heads % 2 == 0 ? 4 : 8));
}

struct Place {
    int head, tile, split;
};

// tiles: a multiple of the shares; ids: 0 .. tiles * heads * splits - 1.
//   PAIRED, for kernels of which two workgroups fit a compute unit: tiles come
// longest first, and a chiplet's first 32 workgroups go to its 32 units one
// each, so the second 32 are reversed: the unit with the longest tile gets the
// shortest of them beside it (8192 ordered tokens, 16/4 heads of 128: 314 ->
// 300 us forward; with three and more to a unit it cost 3%).
template <bool PAIRED>
__device__ __forceinline__ Place chiplet_place(int id, int tiles, int heads, int splits) {
    const int shares = heads % 8 == 0 ? 1 : (heads % 4 == 0 ? 2 : (heads % 2 == 0 ? 4 : 8));
    const int each = tiles / shares;
    int at = (id & 7) * (each * splits * (heads * shares / 8)) + (id >> 3);
    Place p;
    p.split = at % splits;
    at /= splits;
    const int share = at / each;
    int i = at - share * each;
    if (PAIRED && i >> 5 == 1 && (i | 31) < each) i ^= 31;
    p.head = share / shares;
    p.tile = i * shares + share - p.head * shares;
    return p;
}

inline int whole_shares(int tiles, int heads) {
    const int s = chiplet_shares(heads);
    return (tiles + s - 1) / s * s;
}

}  // namespace gsmi
