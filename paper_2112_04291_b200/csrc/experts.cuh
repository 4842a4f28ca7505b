// Matrix products of a router's experts: rows sorted by expert, each expert's rows times its own weights, and the two gradients.
//
//   forward  y[r, :]  = x[source(r), :] W_e^T                          contraction over the ins
//   input    gx[r, :] = gy[r, :] W_e                                   over the outs
//   weights  gW_e     = sum over the expert's rows of gy[r, :]^T x[source(r), :]     over the rows
//
// All three are A B^T of a tile of 128 of the weights' rows (A: the accumulator's lanes) and up to 256 of the ragged side (B: its columns):
// the ragged side is the one whose tiles may have any multiple of 16, so that an expert with few rows costs few instructions, and the weights,
// which bound the time where rows are few, fill whole tiles.
#pragma once

#include "rows.cuh"
#include "tensor.cuh"

namespace fsg {

constexpr uint32_t kProductMaxExperts = 1024u;
constexpr int      kProductThreads    = 256;              // a warp that copies, one that multiplies, two at rest, four that write
constexpr uint32_t kProductM          = 128u;             // of a tile
constexpr uint32_t kProductK          = 64u;              // of a stage
constexpr uint32_t kProductMaxStages  = 8u;
constexpr uint32_t kProductBand       = 16u;              // tiles of weights that are gone through together
constexpr int kForward = 0, kInput = 1, kWeights = 2;

struct alignas(64) ProductArgs {
    CUtensorMap a_map, b_map;
    const uint32_t* starts;
    const uint32_t* order;                                // or nullptr: source(r) = r
    uint32_t  experts, rows, per_row, sources;            // rows: of the sorted side; sources: rows that order may name, times per_row
    uint32_t  m, n, k;                                    // m: A's rows; n: B's (weights only); k: the contraction (forward, input)
    void*     out;
    uint64_t  out_stride, out_expert;
    uint32_t  most_n, box, stages;                        // columns of a tile at most; rows of a copy of B
    uint32_t  kind;
    uint32_t  tries;
};

__host__ __device__ constexpr uint32_t product_stage_bytes(uint32_t most_n) { return kProductM * 128u + most_n * 128u; }

struct ProductShared {
    unsigned long long full[kProductMaxStages], empty[kProductMaxStages], ready[2], taken[2], drained;
    uint32_t tmem, tiles;
    uint32_t first_row[kProductMaxExperts + 1];
    uint32_t first_tile[kProductMaxExperts + 1];
};

struct ProductTile {
    uint32_t expert, m0, n0, n, row, steps;               // n0: first row (weights: in); row, and steps of the contraction
};

template <int MODE> __device__ __forceinline__ ProductTile product_tile(const ProductArgs& a, const ProductShared& s, uint32_t t) {
    ProductTile p;
    const uint32_t mt = (a.m + kProductM - 1u) / kProductM;
    if constexpr (MODE == kWeights) {
        const uint32_t nt = (a.n + a.most_n - 1u) / a.most_n;
        p.expert = t / (mt * nt);
        const uint32_t i = t - p.expert * mt * nt;
        p.m0 = i % mt * kProductM;
        p.n0 = i / mt * a.most_n;
        p.n = min(a.most_n, a.n - p.n0);
        p.row = s.first_row[p.expert];
        p.steps = (s.first_row[p.expert + 1u] - p.row + kProductK - 1u) / kProductK;
    } else {
        uint32_t lo = 0, hi = a.experts;                  // the last expert whose tiles begin at t or before
        while (hi - lo > 1u) {
            const uint32_t mid = (lo + hi) / 2u;
            if (s.first_tile[mid] <= t) lo = mid; else hi = mid;
        }
        p.expert = lo;
        const uint32_t i = t - s.first_tile[lo], rows = s.first_row[lo + 1u] - s.first_row[lo];
        const uint32_t nt = (rows + a.most_n - 1u) / a.most_n, each = ((rows + nt - 1u) / nt + 15u) & ~15u;
        const uint32_t band = i / (nt * kProductBand), j = i - band * nt * kProductBand, wide = min(kProductBand, mt - band * kProductBand);
        p.m0 = (band * kProductBand + j % wide) * kProductM;
        p.n0 = s.first_row[lo] + j / wide * each;
        p.n = min(each, s.first_row[lo + 1u] - p.n0);
        p.row = p.n0;
        p.steps = (a.k + kProductK - 1u) / kProductK;
    }
    return p;
}

// Rows and tiles of each expert, from the starts; every thread of the block.
template <int MODE> __device__ __forceinline__ void product_tables(const ProductArgs& a, ProductShared& s) {
    const uint32_t lane = threadIdx.x & 31u;
    if (threadIdx.x < 32u) {                              // (starts that do not ascend, or lie beyond the rows: no rows)
        const uint32_t mt = (a.m + kProductM - 1u) / kProductM;
        uint32_t row = 0, tiles = 0;
        for (uint32_t e0 = 0; e0 <= a.experts; e0 += 32u) {
            const uint32_t e = e0 + lane;
            uint32_t at = e <= a.experts ? min(a.starts[e], a.rows) : 0u;
#pragma unroll
            for (uint32_t d = 1; d < 32u; d *= 2u) {
                const uint32_t up = __shfl_up_sync(kFullMask, at, d);
                if (lane >= d) at = max(at, up);
            }
            at = max(at, row);
            const uint32_t before = __shfl_up_sync(kFullMask, at, 1);
            // tiles of the expert before: of row .. at
            const uint32_t rows = at - (lane ? before : row);
            uint32_t sum = e && e <= a.experts ? (rows + a.most_n - 1u) / a.most_n * mt : 0u;
#pragma unroll
            for (uint32_t d = 1; d < 32u; d *= 2u) {
                const uint32_t up = __shfl_up_sync(kFullMask, sum, d);
                if (lane >= d) sum += up;
            }
            if (e <= a.experts) { s.first_row[e] = at; s.first_tile[e] = tiles + sum; }
            tiles += __shfl_sync(kFullMask, sum, 31);
            row = __shfl_sync(kFullMask, at, 31);
        }
        if (lane == 0u) {
            const uint32_t nt = MODE == kWeights ? (a.n + a.most_n - 1u) / a.most_n : 1u;
            s.tiles = MODE == kWeights ? a.experts * mt * nt : tiles;
        }
    }
    __syncthreads();
}

// Four sources of sorted rows r .. r + 3, those from `end` on that of the last.
__device__ __forceinline__ int4 product_sources(const ProductArgs& a, uint32_t r, uint32_t end) {
    int x[4];
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) x[i] = (int)(a.order[min(r + i, end - 1u)] / a.per_row);
    return make_int4(x[0], x[1], x[2], x[3]);
}

template <class TO, int MODE> __global__ void __launch_bounds__(kProductThreads, 1) k_product(const __grid_constant__ ProductArgs a) {
    extern __shared__ unsigned char raw[];
    __shared__ ProductShared s;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t stage0 = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t stage_bytes = product_stage_bytes(a.most_n);
    uint32_t columns = 32u;
    while (columns < 2u * a.most_n) columns *= 2u;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < a.stages; ++i) { mbar_init(&s.full[i], 1u); mbar_init(&s.empty[i], 1u); }
        for (uint32_t i = 0; i < 2u; ++i) { mbar_init(&s.ready[i], 1u); mbar_init(&s.taken[i], 4u); }
        mbar_init(&s.drained, 1u);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2u) tmem_alloc(&s.tmem, columns);
    tmem_before_barrier();
    __syncthreads();
    tmem_after_barrier();
    const uint32_t tmem = s.tmem;
    wait_for_previous_kernels();
    allow_next_kernel();
    product_tables<MODE>(a, s);
    const uint32_t tiles = s.tiles;

    if (warp == 0u) {                                     // copies
        uint32_t it = 0;
        bool fine = true;
        for (uint32_t t = blockIdx.x; t < tiles && fine; t += gridDim.x) {
            const ProductTile p = product_tile<MODE>(a, s, t);
            const uint32_t end = p.row + p.n, expert_end = s.first_row[p.expert + 1u];
            const uint32_t groups = (p.n + 3u) / 4u;      // (forward, with an order)
            int4 sources[2];
            if (MODE == kForward && a.order) {
#pragma unroll
                for (uint32_t j = 0; j < 2u; ++j) if (lane + 32u * j < groups) sources[j] = product_sources(a, p.row + 4u * (lane + 32u * j), end);
            }
            const uint32_t boxes = (p.n + a.box - 1u) / a.box, strips = (p.n + 63u) / 64u;
            const uint32_t bytes = kProductM * 128u + (MODE == kWeights ? strips * 8192u : MODE == kForward && a.order ? groups * 512u : boxes * a.box * 128u);
            for (uint32_t step = 0; step < p.steps; ++step, ++it) {
                const uint32_t stage = it % a.stages, round = it / a.stages;
                int4 rows;
                const uint32_t row = p.row + step * kProductK;
                if (MODE == kWeights && a.order) rows = product_sources(a, row + 4u * (lane & 15u), expert_end);
                fine = round == 0u || mbar_wait(&s.empty[stage], (round - 1u) & 1u, a.tries);
                fine = __all_sync(kFullMask, fine);
                if (!fine) break;
                const uint32_t bar = smem_u32(&s.full[stage]), to_a = stage0 + stage * stage_bytes, to_b = to_a + kProductM * 128u;
                const int at = (int)(step * kProductK);
                if (lane == 0u) {
                    mbar_expect_tx(&s.full[stage], bytes);
                    if constexpr (MODE == kForward) tile_load_3d(to_a, &a.a_map, at, (int)p.m0, (int)p.expert, bar);
                    else if constexpr (MODE == kInput) {
                        tile_load_3d(to_a, &a.a_map, (int)p.m0, at, (int)p.expert, bar);
                        tile_load_3d(to_a + 8192u, &a.a_map, (int)p.m0 + 64, at, (int)p.expert, bar);
                    } else {
                        tile_load_2d(to_a, &a.a_map, (int)p.m0, (int)row, bar);
                        tile_load_2d(to_a + 8192u, &a.a_map, (int)p.m0 + 64, (int)row, bar);
                    }
                    if (MODE == kWeights && !a.order) for (uint32_t j = 0; j < strips; ++j) tile_load_2d(to_b + j * 8192u, &a.b_map, (int)(p.n0 + 64u * j), (int)row, bar);
                    if (MODE == kInput || (MODE == kForward && !a.order))
                        for (uint32_t j = 0; j < boxes; ++j) tile_load_2d(to_b + j * a.box * 128u, &a.b_map, at, (int)(p.row + j * a.box), bar);
                }
                __syncwarp();
                if (MODE == kForward && a.order) {
#pragma unroll
                    for (uint32_t j = 0; j < 2u; ++j) if (lane + 32u * j < groups) rows_load(to_b + 512u * (lane + 32u * j), &a.b_map, at, sources[j], bar);
                }
                if (MODE == kWeights && a.order)
                    for (uint32_t j = lane >> 4; j < strips; j += 2u) rows_load(to_b + j * 8192u + 512u * (lane & 15u), &a.b_map, (int)(p.n0 + 64u * j), rows, bar);
            }
        }
        // what is still on its way lands before the block ends, whoever has given up
        for (uint32_t i = it > a.stages ? it - a.stages : 0u; i < it; ++i) mbar_wait(&s.full[i % a.stages], i / a.stages & 1u);
    } else if (warp == 1u) {                              // products
        uint32_t it = 0, turn = 0;
        bool fine = true;
        for (uint32_t t = blockIdx.x; t < tiles && fine; t += gridDim.x) {
            const ProductTile p = product_tile<MODE>(a, s, t);
            if (!p.steps) continue;
            const uint32_t buffer = turn & 1u, acc = tmem + buffer * a.most_n, shape = product_shape(a.kind, kProductM, (p.n + 15u) & ~15u);
            if (turn >= 2u) fine = mbar_wait(&s.taken[buffer], (turn / 2u - 1u) & 1u, a.tries);
            fine = __all_sync(kFullMask, fine);
            if (!fine) break;
            tmem_after_barrier();
            const uint32_t end = s.first_row[p.expert + 1u];
            for (uint32_t step = 0; step < p.steps; ++step, ++it) {
                const uint32_t stage = it % a.stages;
                fine = mbar_wait(&s.full[stage], it / a.stages & 1u, a.tries);
                fine = __all_sync(kFullMask, fine);
                if (!fine) break;
                const uint32_t from_a = stage0 + stage * stage_bytes, from_b = from_a + kProductM * 128u;
                if (MODE == kWeights && p.row + (step + 1u) * kProductK > end) {     // rows behind the expert's last count nothing, whatever they hold
                    const uint32_t left = end - p.row - step * kProductK;
                    const uint32_t strips = 2u + (p.n + 63u) / 64u;
                    for (uint32_t j = 0; j < strips; ++j)
                        for (uint32_t i = left * 8u + lane; i < 512u; i += 32u)
                            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(from_a + j * 8192u + i * 16u), "r"(0u) : "memory");
                    fence_async_reads();
                    __syncwarp();
                }
                tmem_after_barrier();
                if (lane == 0u) {
#pragma unroll
                    for (uint32_t i = 0; i < kProductK / 16u; ++i) {
                        const uint64_t da = MODE == kForward ? operand_at(from_a + 32u * i, 0u) : operand_at(from_a + 2048u * i, 8192u);
                        const uint64_t db = MODE == kWeights ? operand_at(from_b + 2048u * i, 8192u) : operand_at(from_b + 32u * i, 0u);
                        multiply(acc, da, db, shape, step || i);
                    }
                    products_arrive(&s.empty[stage]);
                }
                __syncwarp();
            }
            if (fine && lane == 0u) products_arrive(&s.ready[buffer]);
            __syncwarp();
            ++turn;
        }
        if (lane == 0u) products_arrive(&s.drained);      // no product is under way any more when the accumulators are given back
        __syncwarp();
        mbar_wait(&s.drained, 0u);
    } else if (warp >= 4u) {                              // results
        uint32_t turn = 0;
        bool fine = true;
        for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x) {
            const ProductTile p = product_tile<MODE>(a, s, t);
            const uint32_t buffer = turn & 1u, part = warp & 3u, feature = p.m0 + 32u * part + lane;
            if (p.steps && fine) {
                fine = __all_sync(kFullMask, mbar_wait(&s.ready[buffer], turn / 2u & 1u, a.tries));
                tmem_after_barrier();
            }
            for (uint32_t c0 = 0; c0 < p.n; c0 += 32u) {
                uint32_t r[32];
                if (p.steps && fine) {
                    tmem_load(tmem + (32u * part << 16) + buffer * a.most_n + c0, r);
                    tmem_wait_loads();
                } else {                                  // no rows: zero; a wait ran out: not a number
#pragma unroll
                    for (int i = 0; i < 32; ++i) r[i] = fine ? 0u : 0x7FC00000u;
                }
                if (feature >= a.m) continue;
                if constexpr (MODE == kWeights) {
                    TO* to = static_cast<TO*>(a.out) + p.expert * a.out_expert + feature * a.out_stride + p.n0 + c0;
                    constexpr int V = Vec<TO>::N;
#pragma unroll
                    for (int i = 0; i < 32; i += V) {
                        float f[V];
#pragma unroll
                        for (int j = 0; j < V; ++j) f[j] = __uint_as_float(r[i + j]);
                        if (c0 + (uint32_t)i < p.n) store_values(to + i, f, true);
                    }
                } else {
                    TO* to = static_cast<TO*>(a.out) + (uint64_t)(p.n0 + c0) * a.out_stride + feature;
#pragma unroll
                    for (int i = 0; i < 32; ++i) if (c0 + (uint32_t)i < p.n) to[(uint64_t)i * a.out_stride] = from_float<TO>(__uint_as_float(r[i]));
                }
            }
            if (!p.steps) continue;
            tmem_before_barrier();
            __syncwarp();
            if (lane == 0u) mbar_arrive(&s.taken[buffer]);
            ++turn;
        }
    }
    __syncwarp();
    tmem_before_barrier();
    __syncthreads();
    tmem_after_barrier();
    if (warp == 2u) tmem_free(tmem, columns);
}

}  // namespace fsg
