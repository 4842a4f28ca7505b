// Rows of a table by token (an embedding's lookup), and that table's gradient: the rows of a gradient added up by token.
#pragma once

#include "rows.cuh"

namespace fsg {

constexpr int kEmbedThreads = 256;

// Eight columns of a lane: consecutive ones in vectors of 16 bytes (WIDE: rows begin on 16 bytes), or every G-th of a group of G lanes, one
// element each, so that lanes next to one another still read next to one another.
template <bool WIDE> __device__ __forceinline__ uint32_t column_of(uint32_t chunk, uint32_t lane, uint32_t lanes, int i) {
    return WIDE ? (chunk * lanes + lane) * 8u + (uint32_t)i : chunk * lanes * 8u + (uint32_t)i * lanes + lane;
}
template <class T, bool WIDE> struct Piece {              // as loaded
    static constexpr int WORDS = WIDE ? 8 / Vec<T>::N : 0;
    uint4 raw[WIDE ? WORDS : 1];
    T     one[WIDE ? 1 : 8];
};
// (columns beyond the last are zero)
template <class T, bool WIDE> __device__ __forceinline__ void load_piece(Piece<T, WIDE>& p, const T* row, uint32_t chunk, uint32_t lane, uint32_t lanes, uint32_t cols) {
    if constexpr (WIDE) {
        const uint32_t c = column_of<true>(chunk, lane, lanes, 0);
#pragma unroll
        for (int w = 0; w < Piece<T, WIDE>::WORDS; ++w) {
            const uint32_t at = c + (uint32_t)(w * Vec<T>::N);
            p.raw[w] = make_uint4(0u, 0u, 0u, 0u);
            if (at + Vec<T>::N <= cols) p.raw[w] = load16(row + at);
            else if (at < cols) {                         // (the row's last few)
                T* e = reinterpret_cast<T*>(&p.raw[w]);
#pragma unroll
                for (int i = 0; i < Vec<T>::N; ++i) if (at + (uint32_t)i < cols) e[i] = row[at + (uint32_t)i];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t at = column_of<false>(chunk, lane, lanes, i);
            p.one[i] = at < cols ? row[at] : from_float<T>(0.f);
        }
    }
}
template <class T, bool WIDE> __device__ __forceinline__ void unpack_piece(const Piece<T, WIDE>& p, float (&f)[8]) {
    if constexpr (WIDE) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float g[4];
                Vec<float>::unpack(p.raw[w], g);
#pragma unroll
                for (int i = 0; i < 4; ++i) f[4 * w + i] = g[i];
            }
        } else Vec<T>::unpack(p.raw[0], f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = to_float(p.one[i]);
    }
}
template <class T, bool WIDE> __device__ __forceinline__ void store_piece(T* row, const float (&f)[8], uint32_t chunk, uint32_t lane, uint32_t lanes, uint32_t cols) {
    if (WIDE && column_of<true>(chunk, lane, lanes, 7) < cols) { store_values(row + column_of<true>(chunk, lane, lanes, 0), f, true); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t at = column_of<WIDE>(chunk, lane, lanes, i);
        if (at < cols) row[at] = from_float<T>(f[i]);
    }
}

// ---- lookup -------------------------------------------------------------------------------------

struct LookupArgs {
    const void* table;
    uint64_t  table_stride;
    const int32_t* ids;
    uint32_t  per_row;                                    // ids of each of the table's rows: row ids[t] / per_row
    uint32_t  count, vocab, cols;
    uint32_t  lanes_log;                                  // lanes that share a row's chunk of 8 lanes columns, 1 .. 32
    uint32_t  chunks;
    float     scale;
    void*     out;
    uint64_t  out_stride;
};

// A group of lanes per chunk of a row, kLookupAhead chunks in flight.
constexpr uint32_t kLookupAhead = 4u;
template <class T, class TO, bool WIDE> __global__ void __launch_bounds__(kEmbedThreads) k_embedding(const __grid_constant__ LookupArgs a) {
    wait_for_previous_kernels();
    allow_next_kernel();
    const uint32_t lanes = 1u << a.lanes_log, lane = threadIdx.x & (lanes - 1u);
    const uint64_t groups = (uint64_t)gridDim.x * (kEmbedThreads >> a.lanes_log), all = (uint64_t)a.count * a.chunks;
    for (uint64_t u0 = (uint64_t)blockIdx.x * (kEmbedThreads >> a.lanes_log) + (threadIdx.x >> a.lanes_log); u0 < all; u0 += groups * kLookupAhead) {
        Piece<T, WIDE> p[kLookupAhead];
        uint32_t row[kLookupAhead], chunk[kLookupAhead], id[kLookupAhead];
#pragma unroll
        for (uint32_t j = 0; j < kLookupAhead; ++j) {
            const uint64_t u = u0 + groups * j;
            row[j] = (uint32_t)(u / a.chunks); chunk[j] = (uint32_t)(u - (uint64_t)row[j] * a.chunks);
            id[j] = u < all ? (uint32_t)a.ids[row[j]] / a.per_row : ~0u;
        }
#pragma unroll
        for (uint32_t j = 0; j < kLookupAhead; ++j)
            if (id[j] < a.vocab) load_piece(p[j], static_cast<const T*>(a.table) + id[j] * a.table_stride, chunk[j], lane, lanes, a.cols);
#pragma unroll
        for (uint32_t j = 0; j < kLookupAhead; ++j) {
            if (u0 + groups * j >= all) continue;
            float f[8] = {};
            if (id[j] < a.vocab) {
                unpack_piece(p[j], f);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= a.scale;
            }
            store_piece<TO, WIDE>(static_cast<TO*>(a.out) + row[j] * a.out_stride, f, chunk[j], lane, lanes, a.cols);
        }
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
    uint64_t  sum_blocks;                                 // blocks that add up; the others clear rows of tokens that do not occur
};

// Where in distinct (ascending, n of them) v is: the first that is not below it.
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
__device__ __forceinline__ void write_sum(const GradientArgs& a, uint32_t v, uint32_t row, const float (&sum)[8], uint32_t chunk, uint32_t lane, uint32_t lanes) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = sum[i] * a.scale;
    if constexpr (PAIRS) {
        if (row >= a.most) return;
        store_piece<float, WIDE>(a.values + (uint64_t)row * a.cols, f, chunk, lane, lanes, a.cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v * a.cols + column_of<WIDE>(chunk, lane, lanes, i));
        store_piece<float, WIDE>(reinterpret_cast<float*>(a.keys) + (uint64_t)row * a.cols, f, chunk, lane, lanes, a.cols);
    } else store_piece<TO, WIDE>(static_cast<TO*>(a.out) + v * a.out_stride, f, chunk, lane, lanes, a.cols);
}

template <class T, class TO, bool WIDE, bool PAIRS> __global__ void __launch_bounds__(kEmbedThreads) k_embedding_sum(const __grid_constant__ GradientArgs a) {
    constexpr int AHEAD = sizeof(T) == 2 ? 8 : 4;         // rows in flight
    wait_for_previous_kernels();
    allow_next_kernel();
    const uint32_t lanes = 1u << a.lanes_log, lane = threadIdx.x & (lanes - 1u);
    if (!PAIRS && blockIdx.x >= a.sum_blocks) {           // rows of tokens that do not occur
        const uint64_t groups = (uint64_t)(gridDim.x - a.sum_blocks) * (kEmbedThreads >> a.lanes_log);
        const float zero[8] = {};
        for (uint64_t u = (uint64_t)(blockIdx.x - a.sum_blocks) * (kEmbedThreads >> a.lanes_log) + (threadIdx.x >> a.lanes_log); u < (uint64_t)a.vocab * a.chunks; u += groups) {
            const uint32_t v = (uint32_t)(u / a.chunks), chunk = (uint32_t)(u - (uint64_t)v * a.chunks);
            if (a.starts[v] == a.starts[v + 1u]) store_piece<TO, WIDE>(static_cast<TO*>(a.out) + v * a.out_stride, zero, chunk, lane, lanes, a.cols);
        }
        return;
    }
    const uint32_t have = min(a.starts[a.vocab], a.count);
    const uint64_t u = (uint64_t)blockIdx.x * (kEmbedThreads >> a.lanes_log) + (threadIdx.x >> a.lanes_log);
    const uint32_t tile = (uint32_t)(u / a.chunks), chunk = (uint32_t)(u - (uint64_t)tile * a.chunks);
    const uint32_t begin = min(tile << a.tile_log, have), end = min(begin + (1u << a.tile_log), have);
    if (tile >= a.tiles || begin >= end) return;
    auto id_at = [&](uint32_t p) { const uint32_t at = a.order[p]; return at < a.count ? (uint32_t)a.ids[at] : ~0u; };
    uint32_t now = id_at(begin), row = 0;                 // the token whose rows are being added up; pairs: its row
    bool earlier = begin && id_at(begin - 1u) == now;     // it began in an earlier tile
    const bool goes_on = end < have && id_at(end) == id_at(end - 1u);
    if constexpr (PAIRS) row = place_among(a.distinct, min(*a.number, a.most), now);
    float sum[8] = {};
    auto finish = [&]() {
        if (earlier) store_piece<float, WIDE>(a.parts + 2ull * tile * a.part_stride, sum, chunk, lane, lanes, a.cols);
        else if (now < a.vocab) write_sum<TO, WIDE, PAIRS>(a, now, row, sum, chunk, lane, lanes);
    };
    for (uint32_t p = begin; p < end; p += AHEAD) {
        uint32_t at[AHEAD], id[AHEAD];
        Piece<T, WIDE> piece[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) at[j] = p + (uint32_t)j < end ? a.order[p + (uint32_t)j] : ~0u;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            id[j] = ~0u;
            if (at[j] < a.count) {
                id[j] = (uint32_t)a.ids[at[j]];
                load_piece(piece[j], static_cast<const T*>(a.grad) + at[j] * a.grad_stride, chunk, lane, lanes, a.cols);
            }
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (p + (uint32_t)j >= end) continue;
            if (id[j] != now) {
                finish();
                now = id[j]; earlier = false; ++row;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] = 0.f;
            }
            if (at[j] >= a.count) continue;
            float f[8];
            unpack_piece(piece[j], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += f[i];
        }
    }
    if (goes_on && !earlier) store_piece<float, WIDE>(a.parts + (2ull * tile + 1ull) * a.part_stride, sum, chunk, lane, lanes, a.cols);
    else finish();
}

// Tokens that begin in a tile and go on: a block for each and each chunk of columns (most find nothing to do); its warps each add up an equal
// share of the parts that follow, in their order, and the shares are added in the warps' order.
template <class TO, bool WIDE, bool PAIRS> __global__ void __launch_bounds__(kEmbedThreads) k_embedding_join(const __grid_constant__ GradientArgs a) {
    constexpr uint32_t WARPS = kEmbedThreads / 32;
    __shared__ float shares[WARPS][32][9];
    wait_for_previous_kernels();
    allow_next_kernel();
    const uint32_t lanes = 1u << a.lanes_log, lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t have = min(a.starts[a.vocab], a.count);
    const uint32_t tile = (uint32_t)(blockIdx.x / a.chunks), chunk = (uint32_t)(blockIdx.x - (uint64_t)tile * a.chunks);
    const uint32_t begin = tile << a.tile_log, end = begin + (1u << a.tile_log);
    if (end >= have) return;                              // (the last tile, or behind it)
    const uint32_t first = a.order[end - 1u], next = a.order[end];
    if (first >= a.count || next >= a.count) return;
    const uint32_t v = (uint32_t)a.ids[first];
    if (v >= a.vocab || (uint32_t)a.ids[next] != v || a.starts[v] < begin) return;       // nothing goes on, or it began earlier
    const uint32_t last = (min(a.starts[v + 1u], have) - 1u) >> a.tile_log;              // the tile in which it ends
    const uint32_t parts = last - tile, each = (parts + WARPS - 1u) / WARPS;
    const uint32_t from = tile + 1u + min(warp * each, parts), to = tile + 1u + min(warp * each + each, parts);
    float sum[8] = {};
    if (lane < lanes) {
        if (warp == 0u) {
            Piece<float, WIDE> p;
            load_piece(p, a.parts + (2ull * tile + 1ull) * a.part_stride, chunk, lane, lanes, a.cols);
            unpack_piece(p, sum);
        }
        for (uint32_t t = from; t < to; t += 4u) {
            Piece<float, WIDE> p[4];
#pragma unroll
            for (uint32_t j = 0; j < 4u; ++j) if (t + j < to) load_piece(p[j], a.parts + 2ull * (t + j) * a.part_stride, chunk, lane, lanes, a.cols);
#pragma unroll
            for (uint32_t j = 0; j < 4u; ++j) {
                if (t + j >= to) continue;
                float f[8];
                unpack_piece(p[j], f);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += f[i];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) shares[warp][lane][i] = sum[i];
    __syncthreads();
    if (warp || lane >= lanes) return;
    for (uint32_t w = 1; w < WARPS; ++w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += shares[w][lane][i];
    }
    uint32_t row = 0;
    if constexpr (PAIRS) row = place_among(a.distinct, min(*a.number, a.most), v);
    write_sum<TO, WIDE, PAIRS>(a, v, row, sum, chunk, lane, lanes);
}

}  // namespace fsg
