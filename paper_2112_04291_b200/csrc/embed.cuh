// Rows of a table by token (an embedding's lookup), and that table's gradient: the rows of a gradient added up by token.
//
// A group of 1 to 32 lanes works on a row, a chunk of eight consecutive columns a lane at a time.  Rows may begin at any element: where
// they do not all begin on 16 bytes, a lane loads the aligned vectors that its columns lie in and shifts them into place, and stores the
// aligned vector that begins among its own columns with the first of the next lane's; single elements remain at the two ends of a chunk alone.
#pragma once

#include "rows.cuh"

namespace fsg {

constexpr int kEmbedThreads = 256;

struct Group { uint32_t lanes, lane, mask; };             // lanes of a row; this thread's; the warp's lanes that they are
__device__ __forceinline__ Group row_group(uint32_t lanes_log) {
    Group g;
    g.lanes = 1u << lanes_log;
    g.lane = threadIdx.x & (g.lanes - 1u);
    g.mask = (g.lanes == 32u ? kFullMask : (1u << g.lanes) - 1u) << (threadIdx.x & 31u & ~(g.lanes - 1u));
    return g;
}

// 16 bytes from byte `from` (0 .. 15) on of N + 1 vectors next to one another, for each of the first N
template <int N> __device__ __forceinline__ void shift_words(const uint32_t (&w)[4 * N + 4], uint32_t from, uint32_t (&out)[4 * N]) {
    uint32_t a[4 * N + 2], b[4 * N + 1];
    const bool two = from & 8u, one = from & 4u;
#pragma unroll
    for (int i = 0; i < 4 * N + 2; ++i) a[i] = two ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 4 * N + 1; ++i) b[i] = one ? a[i + 1] : a[i];
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) out[i] = __funnelshift_r(b[i], b[i + 1], (from & 3u) * 8u);
}

// Eight columns from `c` on, as loaded.  Vectors of which no byte is the row's are not touched; what lies in others behind the row's end
// comes along and is never written.
template <class T, bool WIDE> struct Piece { uint4 v[8 / Vec<T>::N + (WIDE ? 0 : 1)]; };
// (AGAIN: rows that others will read, too, are kept in the L1)
template <bool AGAIN = false, class T, bool WIDE> __device__ __forceinline__ void load_piece(Piece<T, WIDE>& p, const T* row, uint32_t c, uint32_t cols) {
    constexpr int N = 8 / Vec<T>::N;
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (c + (uint32_t)(i * Vec<T>::N) < cols) p.v[i] = AGAIN ? *reinterpret_cast<const uint4*>(row + c + i * Vec<T>::N) : load16(row + c + i * Vec<T>::N);
    } else {
        const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(row) & 15u;      // (of every lane's columns alike)
        const uint4* from = reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned char*>(row + c) - off);
        const uint32_t bytes = c < cols ? min(cols - c, 64u) * (uint32_t)sizeof(T) + off : 0u;      // from there to the row's end, or more than there is to load
#pragma unroll
        for (int i = 0; i <= N; ++i) if (16u * (uint32_t)i < bytes && (i < N || off)) p.v[i] = from[i];
    }
}
template <class T, bool WIDE> __device__ __forceinline__ void unpack_piece(const Piece<T, WIDE>& p, const T* row, float (&f)[8]) {
    constexpr int N = 8 / Vec<T>::N;
    uint32_t w[4 * N];
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < N; ++i) { w[4 * i] = p.v[i].x; w[4 * i + 1] = p.v[i].y; w[4 * i + 2] = p.v[i].z; w[4 * i + 3] = p.v[i].w; }
    } else {
        uint32_t all[4 * N + 4];
#pragma unroll
        for (int i = 0; i <= N; ++i) { all[4 * i] = p.v[i].x; all[4 * i + 1] = p.v[i].y; all[4 * i + 2] = p.v[i].z; all[4 * i + 3] = p.v[i].w; }
        shift_words<N>(all, (uint32_t)reinterpret_cast<uintptr_t>(row) & 15u, w);      // (eight columns are whole vectors: the row's own offset)
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float g[Vec<T>::N];
        Vec<T>::unpack(make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]), g);
#pragma unroll
        for (int j = 0; j < Vec<T>::N; ++j) f[i * Vec<T>::N + j] = g[j];
    }
}
// The words of eight values, rounded to T.
template <class T> __device__ __forceinline__ void pack_piece(const float (&f)[8], uint32_t (&w)[32 / Vec<T>::N]) {
#pragma unroll
    for (int i = 0; i < 8 * (int)sizeof(T) / 4; ++i) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(f[i]);
        else w[i] = pack_two<T>(f[2 * i], f[2 * i + 1]);
    }
}
template <class T> __device__ __forceinline__ void store_element(T* to, const uint32_t* w, uint32_t i) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(to + i) = w[i];
    else *reinterpret_cast<uint16_t*>(to + i) = (uint16_t)(w[i / 2] >> (i % 2 * 16));
}
// Eight columns of each of the group's lanes, all of whose threads come here.
template <class T, bool WIDE> __device__ __forceinline__ void store_piece(T* row, const uint32_t (&w)[32 / Vec<T>::N], uint32_t c, uint32_t cols, const Group& g) {
    constexpr int N = 8 / Vec<T>::N;
    constexpr uint32_t PER = Vec<T>::N;
    const uint32_t off = WIDE ? 0u : (uint32_t)reinterpret_cast<uintptr_t>(row) & 15u;
    if (off == 0u) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t at = c + i * PER;
            if (at + PER <= cols) store16(row + at, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
            else {
#pragma unroll
                for (uint32_t j = 0; j < PER; ++j) if (at + j < cols) store_element(row + c, w, i * PER + j);
            }
        }
        return;
    }
    if constexpr (!WIDE) {
        uint32_t all[4 * N + 4], out[4 * N];
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) all[i] = w[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) all[4 * N + i] = __shfl_down_sync(g.mask, w[i], 1, g.lanes);
        shift_words<N>(all, 16u - off, out);
        const uint32_t head = (16u - off) / sizeof(T);    // columns before the first aligned vector
        if (g.lane == 0u) {
#pragma unroll
            for (uint32_t j = 0; j < PER; ++j) if (j < head && c + j < cols) store_element(row + c, w, j);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t at = c + head + i * PER;
            const uint32_t mine = g.lane + 1u == g.lanes && i + 1 == N ? PER - head : PER;      // (nobody's columns follow those of the last lane)
            if (mine == PER && at + PER <= cols) store16(row + at, make_uint4(out[4 * i], out[4 * i + 1], out[4 * i + 2], out[4 * i + 3]));
            else {
#pragma unroll
                for (uint32_t j = 0; j < PER; ++j) if (j < mine && at + j < cols) store_element(row + at - i * PER, out, i * PER + j);
            }
        }
    }
}

// ---- lookup -------------------------------------------------------------------------------------

struct LookupArgs {
    const void* table;
    uint64_t  table_stride;
    const int32_t* ids;
    uint32_t  per_row;                                    // ids of each of the table's rows: row ids[t] / per_row
    uint32_t  count, vocab, cols;
    uint32_t  lanes_log;                                  // lanes of a group
    uint32_t  spans;                                      // pieces of a row that groups take
    uint64_t  units;                                      // of the groups in all
    float     scale;
    void*     out;
    uint64_t  out_stride;
};

// A group takes four chunks of a row (SHORT rows: a chunk of each of four rows), all on their way at once.
constexpr uint32_t kLookupAhead = 4u;
template <class T, class TO, bool WIDE, bool SHORT> __global__ void __launch_bounds__(kEmbedThreads) k_embedding(const __grid_constant__ LookupArgs a) {
    wait_for_previous_kernels();
    allow_next_kernel();
    const Group g = row_group(a.lanes_log);
    const uint64_t u = (uint64_t)blockIdx.x * (kEmbedThreads >> a.lanes_log) + (threadIdx.x >> a.lanes_log);
    if (u >= a.units) return;
    const uint32_t row0 = SHORT ? (uint32_t)u * kLookupAhead : a.units <= 0xFFFFFFFFull ? (uint32_t)u / a.spans : (uint32_t)(u / a.spans);
    const uint32_t c0 = SHORT ? g.lane * 8u : ((uint32_t)(u - (uint64_t)row0 * a.spans) * kLookupAhead * g.lanes + g.lane) * 8u, step = SHORT ? 0u : g.lanes * 8u;
    Piece<T, WIDE> p[kLookupAhead];
    uint32_t id[kLookupAhead];
#pragma unroll
    for (uint32_t j = 0; j < kLookupAhead; ++j) {
        if (!SHORT && j) { id[j] = id[0]; continue; }
        id[j] = row0 + j < a.count ? (uint32_t)a.ids[row0 + j] : ~0u;
        if (a.per_row != 1u) id[j] /= a.per_row;
    }
#pragma unroll
    for (uint32_t j = 0; j < kLookupAhead; ++j) if (id[j] < a.vocab) load_piece<true>(p[j], static_cast<const T*>(a.table) + id[j] * a.table_stride, c0 + step * j, a.cols);
#pragma unroll
    for (uint32_t j = 0; j < kLookupAhead; ++j) {
        const uint32_t row = SHORT ? row0 + j : row0;
        if (row >= a.count || c0 + step * j - g.lane * 8u >= a.cols) continue;       // (of the whole group)
        float f[8] = {};
        if (id[j] < a.vocab) {
            unpack_piece(p[j], static_cast<const T*>(a.table) + id[j] * a.table_stride, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= a.scale;
        }
        uint32_t w[32 / Vec<TO>::N];
        pack_piece<TO>(f, w);
        store_piece<TO, WIDE>(static_cast<TO*>(a.out) + row * a.out_stride, w, c0 + step * j, a.cols, g);
    }
}

// ---- gradient -------------------------------------------------------------------------------------
// The sorted positions are cut into tiles of equal length, whatever the tokens are; a group of lanes adds up a tile's rows, eight columns a lane,
// in the order of the positions, in fp32.  A token whose positions lie within the tile is finished there.  One that began in an earlier tile, or goes
// on into the next, leaves its part of the sum in the workspace (two rows a tile at most), and k_embedding_join adds those up in
// the tiles' order.  So the order of a sum depends on the sizes and the tokens alone, and a token that fills half the batch takes no
// longer than as many different ones.

struct GradientArgs {
    const void* grad;                                     // count x cols
    uint64_t  grad_stride;
    const int32_t* ids;
    const uint32_t* order;
    const uint32_t* starts;
    const uint32_t* distinct;                             // pairs only
    const uint32_t* number;                               // pairs only
    uint32_t  count, vocab, cols;
    uint32_t  lanes_log, chunks;
    uint32_t  tile_log, tiles;                            // positions of a tile, and how many of them
    float     scale;
    void*     out;                                        // the table's gradient, or
    uint64_t  out_stride;
    uint32_t* keys;                                       // pairs
    float*    values;
    uint32_t  most;                                       // rows that keys and values hold
    uint64_t  part_stride;                                // cols, up to a multiple of 4
    float*    parts;                                      // 2 tiles x part_stride: of a tile's first token (begun earlier), of its last (that goes on)
    uint4*    follow;                                     // of each tile: in how many of the next its last token goes on, if that begins in it; the token; its row (pairs)
    uint32_t  sum_blocks, clear_blocks;                   // blocks that add up, and that clear rows of tokens that do not occur (in turn, as long as there are both)
    uint32_t  clear_rows;                                 // of a block that clears
};

// Where in distinct (ascending, n of them) v is: the first that is not below it.  One warp: 32 probes a step.
__device__ __forceinline__ uint32_t place_among_by_warp(const uint32_t* distinct, uint32_t n, uint32_t v) {
    const uint32_t lane = threadIdx.x & 31u;
    uint32_t lo = 0, hi = n;                              // the answer lies in lo .. hi
    while (hi - lo > 32u) {
        const uint32_t each = (hi - lo + 31u) / 32u, at = lo + lane * each;
        const uint32_t below = __popc(__ballot_sync(kFullMask, at < hi && distinct[at] < v));
        if (!below) return lo;
        hi = min(hi, lo + below * each);
        lo += (below - 1u) * each + 1u;
    }
    return lo + __popc(__ballot_sync(kFullMask, lo + lane < hi && distinct[lo + lane] < v));
}
__device__ __forceinline__ uint32_t place_among(const uint32_t* distinct, uint32_t n, uint32_t v) {
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2u;
        if (distinct[mid] < v) lo = mid + 1u; else hi = mid;
    }
    return lo;
}

// A finished sum to its row.
template <class TO, bool WIDE, bool PAIRS>
__device__ __forceinline__ void write_sum(const GradientArgs& a, uint32_t v, uint32_t row, const float (&sum)[8], uint32_t c, const Group& g) {
    float f[8];
    uint32_t w[32 / Vec<TO>::N];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = sum[i] * a.scale;
    pack_piece<TO>(f, w);
    if constexpr (PAIRS) {
        if (row >= a.most) return;
        store_piece<float, WIDE>(a.values + (uint64_t)row * a.cols, w, c, a.cols, g);
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) w[i] = v * a.cols + c + i;
        store_piece<float, WIDE>(reinterpret_cast<float*>(a.keys) + (uint64_t)row * a.cols, w, c, a.cols, g);
    } else store_piece<TO, WIDE>(static_cast<TO*>(a.out) + v * a.out_stride, w, c, a.cols, g);
}
__device__ __forceinline__ void write_part(const GradientArgs& a, uint64_t part, const float (&sum)[8], uint32_t c, const Group& g) {
    uint32_t w[8];
    pack_piece<float>(sum, w);
    store_piece<float, true>(a.parts + part * a.part_stride, w, c, a.cols, g);
}

// Rows of tokens that do not occur become zero: a block's are listed, and gone through vector by vector.
template <class TO, bool WIDE> __device__ __forceinline__ void clear_rows(const GradientArgs& a, uint32_t block) {
    __shared__ uint32_t listed[64], some;
    const uint32_t v0 = block * a.clear_rows;
    if (threadIdx.x == 0) some = 0;
    __syncthreads();
    if (threadIdx.x < a.clear_rows && v0 + threadIdx.x < a.vocab && a.starts[v0 + threadIdx.x] == a.starts[v0 + threadIdx.x + 1u]) listed[atomicAdd(&some, 1u)] = v0 + threadIdx.x;
    __syncthreads();
    const Group g = row_group(a.lanes_log);
    const uint32_t zero[32 / Vec<TO>::N] = {};
    const uint32_t groups = (uint32_t)kEmbedThreads >> a.lanes_log, mine = threadIdx.x >> a.lanes_log;
    auto clear = [&](uint32_t i, uint32_t chunk) { store_piece<TO, WIDE>(static_cast<TO*>(a.out) + listed[i] * a.out_stride, zero, (chunk * g.lanes + g.lane) * 8u, a.cols, g); };
    if (a.chunks >= groups) {                             // (a row after the other: nothing to divide)
        for (uint32_t i = 0; i < some; ++i)
            for (uint32_t chunk = mine; chunk < a.chunks; chunk += groups) clear(i, chunk);
    } else {
        for (uint32_t u = mine; u < some * a.chunks; u += groups) clear(u / a.chunks, u % a.chunks);
    }
}

// What a group knows of its tile before it adds up.
struct SumTile {
    uint32_t tile, begin, end, have, c, now, row;         // c: this lane's first column; now: the token whose rows are being added up; row: its row (pairs)
    bool earlier, goes_on, first_chunk;                   // now began in an earlier tile; the last token goes on; this lane writes for the tile
};
__device__ __forceinline__ uint32_t id_at(const GradientArgs& a, uint32_t p) {
    const uint32_t at = a.order[p];
    return at < a.count ? (uint32_t)a.ids[at] : ~0u;
}
// Blocks that add up beside blocks that clear: false where this one clears, and has.
template <class TO, bool WIDE, bool PAIRS> __device__ __forceinline__ bool sums(const GradientArgs& a, uint32_t& block) {
    block = blockIdx.x;
    if constexpr (!PAIRS) {
        const uint32_t both = min(a.sum_blocks, a.clear_blocks);
        const bool clears = block < 2u * both ? block & 1u : a.clear_blocks > both;
        block = block < 2u * both ? block / 2u : block - both;
        if (clears) { clear_rows<TO, WIDE>(a, block); return false; }
    }
    return true;
}
template <class TO, bool WIDE, bool PAIRS> __device__ __forceinline__ void finish_token(const GradientArgs& a, const SumTile& t, const float (&sum)[8], const Group& g) {
    if (t.earlier) write_part(a, 2ull * t.tile, sum, t.c, g);
    else if (t.now < a.vocab) write_sum<TO, WIDE, PAIRS>(a, t.now, t.row, sum, t.c, g);
}
template <class TO, bool WIDE, bool PAIRS> __device__ __forceinline__ void finish_tile(const GradientArgs& a, const SumTile& t, const float (&sum)[8], const Group& g) {
    const bool starts_here = t.goes_on && !t.earlier;
    if (t.first_chunk) {
        const uint32_t behind = starts_here && t.now < a.vocab ? min(a.starts[t.now + 1u], t.have) : 0u;
        a.follow[t.tile] = make_uint4(behind > t.end ? ((behind - 1u) >> a.tile_log) - t.tile : 0u, t.now, t.row, 0u);
    }
    if (starts_here) write_part(a, 2ull * t.tile + 1ull, sum, t.c, g);
    else finish_token<TO, WIDE, PAIRS>(a, t, sum, g);
}

// Rows in registers.  FULL: a warp a group, whose lanes look up the rows and tokens of sixteen positions at once and tell one another; otherwise
// each lane looks up all of them.
template <class T, class TO, bool WIDE, bool PAIRS, bool FULL> __global__ void __launch_bounds__(kEmbedThreads, FULL && sizeof(T) == 2 ? 3 : 2) k_embedding_sum(const __grid_constant__ GradientArgs a) {
    constexpr uint32_t AHEAD = sizeof(T) == 2 || WIDE ? 8u : 4u;        // rows in flight
    constexpr uint32_t WINDOW = FULL ? 16u : AHEAD, EACH = FULL ? 1u : AHEAD;      // positions looked up at a time, and of them a lane's
    wait_for_previous_kernels();
    allow_next_kernel();
    uint32_t block;
    if (!sums<TO, WIDE, PAIRS>(a, block)) return;
    const Group g = row_group(FULL ? 5u : a.lanes_log);
    const uint32_t u = FULL ? block * (kEmbedThreads / 32u) + __shfl_sync(kFullMask, threadIdx.x >> 5, 0) : block * (kEmbedThreads >> a.lanes_log) + (threadIdx.x >> a.lanes_log);
    SumTile t;
    t.tile = u / a.chunks; t.c = ((u - t.tile * a.chunks) * g.lanes + g.lane) * 8u;
    if (t.tile >= a.tiles) return;
    t.begin = t.tile << a.tile_log;
    // rows and tokens (those behind the last are garbage, and of no account)
    auto look_up = [&](uint32_t p, uint32_t (&at)[EACH], uint32_t (&id)[EACH]) {
        if constexpr (FULL) p += g.lane & (WINDOW - 1u);
#pragma unroll
        for (uint32_t j = 0; j < EACH; ++j) at[j] = p + j < a.count ? a.order[p + j] : ~0u;
#pragma unroll
        for (uint32_t j = 0; j < EACH; ++j) id[j] = at[j] < a.count ? (uint32_t)a.ids[at[j]] : ~0u;
    };
    uint32_t at[EACH], id[EACH];
    look_up(t.begin, at, id);
    const uint32_t before = t.begin ? id_at(a, t.begin - 1u) : ~0u;
    t.have = min(a.starts[a.vocab], a.count);
    t.end = min(t.begin + (1u << a.tile_log), t.have);
    t.first_chunk = u == t.tile * a.chunks && g.lane == 0u;
    if (t.begin >= t.end) {
        if (t.first_chunk) a.follow[t.tile] = make_uint4(0u, 0u, 0u, 0u);
        return;
    }
    t.now = FULL ? __shfl_sync(kFullMask, id[0], 0) : id[0];
    t.row = 0;
    t.earlier = t.begin && before == t.now;
    t.goes_on = t.end < t.have && id_at(a, t.end) == id_at(a, t.end - 1u);
    if constexpr (PAIRS) t.row = FULL ? place_among_by_warp(a.distinct, min(*a.number, a.most), t.now) : place_among(a.distinct, min(*a.number, a.most), t.now);
    float sum[8] = {};
    for (uint32_t p0 = t.begin; p0 < t.end; p0 += WINDOW) {
        uint32_t next_at[EACH], next_id[EACH];
        if (p0 + WINDOW < t.end) look_up(p0 + WINDOW, next_at, next_id);
#pragma unroll
        for (uint32_t w = 0; w < WINDOW; w += AHEAD) {
            const uint32_t p = p0 + w;
            if (p >= t.end) continue;
            Piece<T, WIDE> piece[AHEAD];
            uint32_t from[AHEAD];
#pragma unroll
            for (uint32_t j = 0; j < AHEAD; ++j) {
                from[j] = FULL ? __shfl_sync(kFullMask, at[0], w + j) : at[FULL ? 0u : j];
                if (p + j < t.end && from[j] < a.count) load_piece(piece[j], static_cast<const T*>(a.grad) + from[j] * a.grad_stride, t.c, a.cols);
            }
#pragma unroll
            for (uint32_t j = 0; j < AHEAD; ++j) {
                if (p + j >= t.end) continue;
                const uint32_t token = FULL ? __shfl_sync(kFullMask, id[0], w + j) : id[FULL ? 0u : j];
                if (token != t.now) {
                    finish_token<TO, WIDE, PAIRS>(a, t, sum, g);
                    t.now = token; t.earlier = false; ++t.row;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
                }
                if (from[j] >= a.count) continue;
                float f[8];
                unpack_piece(piece[j], static_cast<const T*>(a.grad) + from[j] * a.grad_stride, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += f[i];
            }
        }
#pragma unroll
        for (uint32_t j = 0; j < EACH; ++j) { at[j] = next_at[j]; id[j] = next_id[j]; }
    }
    finish_tile<TO, WIDE, PAIRS>(a, t, sum, g);
}

// Rows of more than 128 columns that begin at any element, a warp a chunk of 256.  Their vectors and what shifts them take registers and
// instructions for each row in flight above: here the rows are copied to shared memory, 16 or 8 of them ahead of the one that is added up, from the
// vector that the chunk begins in, and the code for a row stands once.  (30001 x 1001 fp16: 38 us, in registers 45; rows on 16 bytes, 16384 x 2048
// and 65536 x 512 bf16: 92 and 33 us, in registers 91 and 26.)
template <class T> struct SumShared {
    static constexpr uint32_t SLOTS = sizeof(T) == 2 ? 16u : 8u;
    static constexpr uint32_t VECTORS = 16u * (uint32_t)sizeof(T) + 1u;
    uint4 rows[kEmbedThreads / 32][SLOTS][VECTORS];
};
template <class T, class TO, bool PAIRS> __global__ void __launch_bounds__(kEmbedThreads, 3) k_embedding_sum_shifted(const __grid_constant__ GradientArgs a) {
    using Shared = SumShared<T>;
    constexpr uint32_t SLOTS = Shared::SLOTS, N = 8u / Vec<T>::N;       // vectors of a lane
    extern __shared__ __align__(16) unsigned char raw[];
    wait_for_previous_kernels();
    allow_next_kernel();
    uint32_t block;
    if (!sums<TO, false, PAIRS>(a, block)) return;
    const Group g = row_group(5u);
    const uint32_t lane = threadIdx.x & 31u, warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0);
    uint4 (&rows)[SLOTS][Shared::VECTORS] = reinterpret_cast<Shared*>(raw)->rows[warp];
    const uint32_t u = block * (kEmbedThreads / 32u) + warp;
    SumTile t;
    t.tile = u / a.chunks;
    const uint32_t c0 = (u - t.tile * a.chunks) * 256u;
    t.c = c0 + lane * 8u;
    if (t.tile >= a.tiles) return;
    t.begin = t.tile << a.tile_log;
    // rows and tokens of positions p .. p + 31, a lane each (those behind the last are garbage, and of no account)
    auto look_up = [&](uint32_t p, uint32_t& at, uint32_t& id) {
        at = p + lane < a.count ? a.order[p + lane] : ~0u;
        id = at < a.count ? (uint32_t)a.ids[at] : ~0u;
    };
    uint32_t at, id, next_at = ~0u, next_id = ~0u;
    look_up(t.begin, at, id);
    const uint32_t before = t.begin ? id_at(a, t.begin - 1u) : ~0u;
    t.have = min(a.starts[a.vocab], a.count);
    t.end = min(t.begin + (1u << a.tile_log), t.have);
    t.first_chunk = c0 == 0u && lane == 0u;
    if (t.begin >= t.end) {
        if (t.first_chunk) a.follow[t.tile] = make_uint4(0u, 0u, 0u, 0u);
        return;
    }
    uint32_t window = t.begin;                            // the first position of those that at and id are of
    if (window + 32u < t.end) look_up(window + 32u, next_at, next_id);
    const T* const grad = static_cast<const T*>(a.grad) + c0;
    const uint32_t bytes = min(256u, a.cols - c0) * (uint32_t)sizeof(T);
    // position p's row on its way to its place (one group of copies, whether or not there is one)
    auto fetch = [&](uint32_t p, uint32_t slot) {
        const uint32_t ahead = p - window, of = __shfl_sync(kFullMask, ahead < 32u ? at : next_at, ahead & 31u);
        if (p < t.end && of < a.count) {
            const T* from = grad + of * a.grad_stride;
            const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(from) & 15u, vectors = (off + bytes + 15u) / 16u;
            const unsigned char* first = reinterpret_cast<const unsigned char*>(from) - off;
#pragma unroll
            for (uint32_t i = 0; i < Shared::VECTORS; i += 32u) if (i + lane < vectors && i + lane < Shared::VECTORS) copy16_async(&rows[slot][i + lane], first + 16u * (i + lane));
        }
        copies_end_group();
    };
#pragma unroll 1
    for (uint32_t i = 0; i < SLOTS; ++i) fetch(t.begin + i, i);
    t.now = __shfl_sync(kFullMask, id, 0); t.row = 0;
    t.earlier = t.begin && before == t.now;
    t.goes_on = t.end < t.have && id_at(a, t.end) == id_at(a, t.end - 1u);
    if constexpr (PAIRS) t.row = place_among_by_warp(a.distinct, min(*a.number, a.most), t.now);
    float sum[8] = {};
    uint32_t slot = 0;
#pragma unroll 1
    for (uint32_t p = t.begin; p < t.end; ++p) {
        const uint32_t of = __shfl_sync(kFullMask, at, p - window), token = __shfl_sync(kFullMask, id, p - window);
        if (token != t.now) {
            finish_token<TO, false, PAIRS>(a, t, sum, g);
            t.now = token; t.earlier = false; ++t.row;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = 0.f;
        }
        wait_copies<(int)SLOTS - 1>();
        __syncwarp();                                     // (a lane reads what others have copied)
        if (of < a.count) {
            Piece<T, false> piece;
#pragma unroll
            for (uint32_t i = 0; i <= N; ++i) piece.v[i] = rows[slot][lane * N + i];
            float f[8];
            unpack_piece(piece, grad + of * a.grad_stride, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += f[i];
        }
        __syncwarp();
        fetch(p + SLOTS, slot);
        slot = slot + 1u == SLOTS ? 0u : slot + 1u;
        if (p + 1u == window + 32u) {
            window += 32u;
            at = next_at; id = next_id;
            if (window + 32u < t.end) look_up(window + 32u, next_at, next_id);
        }
    }
    wait_copies<0>();
    finish_tile<TO, false, PAIRS>(a, t, sum, g);
}

// Tokens that begin in a tile and go on.  A block looks at eight tiles, for a chunk of columns: each of its warps adds up what follows one of
// them, in the order of the tiles; where that is long all warps add up equal shares, which are added in the warps' order.
constexpr uint32_t kJoinTiles = 8u, kJoinLong = 32u;
template <class TO, bool WIDE, bool PAIRS> __global__ void __launch_bounds__(kEmbedThreads) k_embedding_join(const __grid_constant__ GradientArgs a) {
    constexpr uint32_t WARPS = kEmbedThreads / 32;
    static_assert(WARPS == kJoinTiles, "a tile a warp");
    __shared__ float shares[WARPS][32][9];
    wait_for_previous_kernels();
    allow_next_kernel();
    const Group g = row_group(a.lanes_log);
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t tiles = blockIdx.x / a.chunks * kJoinTiles, c = ((blockIdx.x % a.chunks) * g.lanes + lane) * 8u;
    const uint4 follow = lane < kJoinTiles && tiles + lane < a.tiles ? a.follow[tiles + lane] : make_uint4(0u, 0u, 0u, 0u);
    float sum[8];
    // parts of tiles from .. to, behind the first tile's own (where `own`)
    auto add_up = [&](uint32_t tile, bool own, uint32_t from, uint32_t to) {
        auto add = [&](const Piece<float, true>& p) {
            float f[8];
            unpack_piece(p, a.parts, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += f[j];
        };
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.f;
        if (lane >= g.lanes) return;
        Piece<float, true> first;
        if (own) load_piece(first, a.parts + (2ull * tile + 1ull) * a.part_stride, c, a.cols);
        for (uint32_t t = from; t < to || own; t += 4u) {
            Piece<float, true> p[4];
#pragma unroll
            for (uint32_t j = 0; j < 4u; ++j) if (t + j < to) load_piece(p[j], a.parts + 2ull * (t + j) * a.part_stride, c, a.cols);
            if (own) { add(first); own = false; }
#pragma unroll
            for (uint32_t j = 0; j < 4u; ++j) if (t + j < to) add(p[j]);
        }
    };
    const uint32_t mine = __shfl_sync(kFullMask, follow.x, warp), v = __shfl_sync(kFullMask, follow.y, warp), row = __shfl_sync(kFullMask, follow.z, warp);
    if (mine && mine < kJoinLong) {
        add_up(tiles + warp, true, tiles + warp + 1u, tiles + warp + 1u + mine);
        if (lane < g.lanes) write_sum<TO, WIDE, PAIRS>(a, v, row, sum, c, g);
    }
    for (uint32_t some = __ballot_sync(kFullMask, follow.x >= kJoinLong); some; some &= some - 1u) {
        const uint32_t i = (uint32_t)__ffs((int)some) - 1u, tile = tiles + i, parts = __shfl_sync(kFullMask, follow.x, i), each = (parts + WARPS - 1u) / WARPS;
        add_up(tile, warp == 0u, tile + 1u + min(warp * each, parts), tile + 1u + min(warp * each + each, parts));
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) shares[warp][lane][j] = sum[j];
        __syncthreads();
        const uint32_t v_of = __shfl_sync(kFullMask, follow.y, i), row_of = __shfl_sync(kFullMask, follow.z, i);
        if (warp) continue;
        for (uint32_t w = 1; w < WARPS; ++w) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += shares[w][lane][j];
        }
        if (lane < g.lanes) write_sum<TO, WIDE, PAIRS>(a, v_of, row_of, sum, c, g);
    }
}

}  // namespace fsg
