// Matrix products of a router's experts: rows sorted by expert, each expert's rows times its own weights, and the two gradients.
//
//   forward  y[r, :]  = x[r, :] W_e^T                          contraction over the ins
//   input    gx[r, :] = gy[r, :] W_e                           over the outs
//   weights  gW_e     = sum over the expert's rows of gy[r, :]^T x[r, :]     over the rows
//
// All three are A B^T of a tile of 256 of the weights' rows (A: the accumulator's lanes) and up to 256 of the ragged side (B: its columns):
// the ragged side is the one whose tiles may have any multiple of 32, so that an expert with few rows costs few instructions, and the weights,
// which bound the time where rows are few, fill whole tiles.
//
// A pair of blocks (two SMs) works on a tile: each copies half of A and half of B, so that an operand byte in shared memory serves twice as many
// products as with one block.  In each block a warp copies tiles, a second (the first block's) issues the products; eight write results, while the
// next tile's products go into the other half of the accumulators.  What both blocks copy completes on a barrier of the first block, where the
// products wait.  (A thread that told it what has landed in the second block would have to release at the cluster's scope, which takes a microsecond
// a stage: 16384 x 4096 x 14336 in 3290 us.)  Only where rows behind an expert's last are cleared, once a tile of the weights' gradients, do two
// further warps of each block so (with one, 40 rows, 8 experts, 14336 x 4096: 249 us, with two 163; 512 rows, nothing to clear, 160).  Waits for what
// the other block's threads, copies or products signal are of the cluster's scope; that costs nothing that could be measured.  Where there are few tiles of a long
// contraction, up to eight pairs of a cluster share each, and add up what they have through their shared memory.  A single thread issues copies and
// products: what bounds the rate is then the tensor cores (and the GPU's power) alone.  Measured, with sorted rows, by the GPU and its clocks:
//   16384 x 4096 x 14336 bf16, 8 experts: 1160 to 1460 us each way (1320 to 1650 TFLOP/s; a library's product of one matrix of that size, 1590)
//   49152 x 2048 x 1408, 64 experts: 205 to 286 us (990 to 1390 TFLOP/s; 19 rounds of tiles, the last partly filled, 5.5 tiles of 256 outs); to fp32 273 to 290
//   32 x 4096 x 14336, 8 experts: 142 to 156 us, the weights' 940 MB at a copy's rate
//   gradients of 64 experts' 1408 x 2048 weights of 49152 rows, fp32: 281 to 384 us, 738 MB written while 340 MB are read; bf16 234 to 302, fp16 277 to 340
//
// The tensor cores cut off what an addition to an accumulator has beyond 32 bits, always towards zero.  Measured, in proportion to the contraction's
// length, of the sum of magnitudes: 5.9e-9 for each value where all have one sign (512 values 2.4e-6, 8192 4.8e-5, 65536 3.9e-4), up to 2.6 times
// that where the first values outweigh the others (512 6.4e-6, 1.1e-5 at most; 8192 1.0e-4); 1e-9 of the result where signs are random (512 5.5e-7, 8192
// 8.4e-6).  So accumulators begin anew after a while, and the warps that write add them up in registers, rounding to nearest (SUMS): results of 32 bits
// every 512 values, whatever the length (plain sums in fp32 of 4096 values of random signs: 6.1e-7).  Results of 16 bits may lose a quarter of half
// a step on average, which just below a power of two is 2^-12 of the value in fp16, 2^-9 in bf16: contractions that may have more than 2^12 values
// (fp16) or 2^15 (bf16) are added up every 2^12.
#pragma once

#include "rows.cuh"
#include "tensor.cuh"

namespace fsg {

constexpr uint32_t kProductMaxExperts = 1024u;
constexpr int      kProductThreads    = 384;              // four warps that feed, eight that write
constexpr uint32_t kProductM          = 256u;             // of a tile; half of it a block's
constexpr uint32_t kProductK          = 64u;              // of a stage
constexpr uint32_t kProductMaxStages  = 12u;
constexpr uint32_t kProductSorted     = 256u;             // experts that are put in order of their rows (weights)
constexpr uint32_t kProductBand       = 8u;               // tiles of weights that are gone through together
constexpr uint32_t kProductSum        = 8u;               // stages between two additions in registers: results of 32 bits, and shared contractions
constexpr uint32_t kProductLongSum    = 64u;              // ... results of 16 bits, of contractions that may have more values than
constexpr uint64_t kProductLongF16    = 1ull << 12, kProductLongBF16 = 1ull << 15;
// Bytes of a box of a gradient of weights; each warp that writes has one.  With two or three, which it would wait for less, or with boxes of rows of
// 128 bytes, there is room for five or four stages instead of six: 49152 x 2048 x 1408 of 64 experts 239 us as it is, 246, 245 (128) and 259 (two of
// 128); to fp32 288, 298, 297, 319; 8192 x 2048 x 2048 of 8 52, 54, 54.5, 58; 4096 x 1016 x 680 of 60 30.6, 31.2, 29.8, 30.0.
constexpr uint32_t kProductTurned     = 2048u;
constexpr int kForward = 0, kInput = 1, kWeights = 2;

struct alignas(64) ProductArgs {
    CUtensorMap a_map, b_map, out_map;                    // (the last: weights)
    const uint32_t* starts;
    uint32_t  experts, rows;                              // rows: of the sorted side
    uint32_t  m, n, k;                                    // m: A's rows; n: B's (weights only); k: the contraction (forward, input)
    void*     out;
    uint64_t  out_stride, out_expert;
    uint32_t  most_n, box, stages;                        // columns of a tile at most; rows of a copy of B
    uint32_t  sum_stages;                                 // (SUMS) of an accumulator
    uint32_t  splits;                                     // pairs of blocks that share a tile's contraction (a cluster; then a tile each)
    uint32_t  kind;
    uint32_t  tries;
};

// of one block: half of A's rows and half of B's (weights: in strips of 64)
template <int MODE> __host__ __device__ constexpr uint32_t product_stage_bytes(uint32_t most_n) {
    return kProductM / 2u * 128u + (MODE == kWeights ? (most_n / 2u + 63u) / 64u * 8192u : most_n / 2u * 128u);
}

struct ProductShared {
    unsigned long long landed[kProductMaxStages];         // (weights) this block's copies of a stage whose last rows are to be cleared
    unsigned long long full[kProductMaxStages];           // (first block) both blocks' operands
    unsigned long long empty[kProductMaxStages];          // the products that read them are done
    unsigned long long ready[2];                          // an accumulator's products are done
    unsigned long long taken[2];                          // (first block) ... and have been read, by both blocks
    unsigned long long drained;
    uint32_t tmem, tiles, lost;                           // lost: (a shared contraction) a wait of this block's has run out
    uint32_t gave_up;                                     // a thread of the pair's that copies or multiplies has
    uint32_t issued[2], cleared[2];                       // of each block: stages copied; those whose last copies are its own `landed`'s (bits)
    uint32_t first_row[kProductMaxExperts + 1];
    uint32_t first_tile[kProductMaxExperts];              // (forward, input) of the experts in their order
    uint16_t expert_at[kProductMaxExperts];               // that order
};

// The stages in turn, and the parity of the round.
struct ProductRing {
    uint32_t stage = 0, round = 0;
    __device__ __forceinline__ void next(uint32_t stages) { if (++stage == stages) { stage = 0; round ^= 1u; } }
};

struct ProductTile {
    uint32_t expert, m0, n0, n, half, row, end;           // n0: first row (weights: in); half: columns of a block's B; rows row .. end
    uint32_t step0, steps, all_steps;                     // of the contraction: this pair's, and all
    bool     clears;                                      // (weights) the last of this pair's stages holds rows behind `end`
};

// columns of each of the tiles that an expert's rows make (forward, input): as few tiles as hold them, of equal length
__device__ __forceinline__ uint32_t product_columns(uint32_t rows, uint32_t most_n) {
    const uint32_t nt = (rows + most_n - 1u) / most_n;
    return nt ? ((rows + nt - 1u) / nt + 31u) & ~31u : 0u;
}

template <int MODE, bool SPLIT> __device__ __forceinline__ ProductTile product_tile(const ProductArgs& a, const ProductShared& s, uint32_t t, uint32_t share) {
    ProductTile p;
    const uint32_t mt = (a.m + kProductM - 1u) / kProductM;
    if constexpr (MODE == kWeights) {
        const uint32_t nt = (a.n + a.most_n - 1u) / a.most_n;
        const uint32_t place = t / (mt * nt), i = t - place * mt * nt;
        p.expert = s.expert_at[place];
        const uint32_t band = i / (nt * kProductBand), j = i - band * nt * kProductBand, wide = min(kProductBand, mt - band * kProductBand);
        p.m0 = (band * kProductBand + j % wide) * kProductM;
        p.n0 = j / wide * a.most_n;
        p.n = min(a.most_n, a.n - p.n0);
        p.row = s.first_row[p.expert];
        p.end = s.first_row[p.expert + 1u];
        p.all_steps = (p.end - p.row + kProductK - 1u) / kProductK;
    } else {
        uint32_t lo = 0, hi = a.experts;                  // the last expert whose tiles begin at t or before
        while (hi - lo > 1u) {
            const uint32_t mid = (lo + hi) / 2u;
            if (s.first_tile[mid] <= t) lo = mid; else hi = mid;
        }
        p.expert = s.expert_at[lo];
        const uint32_t first_row = s.first_row[p.expert], end = s.first_row[p.expert + 1u], rows = end - first_row, i = t - s.first_tile[lo];
        // (no tile is empty, since all but one of the fewest tiles that hold the rows do not)
        const uint32_t nt = (rows + a.most_n - 1u) / a.most_n, each = product_columns(rows, a.most_n);
        const uint32_t band = i / (nt * kProductBand), j = i - band * nt * kProductBand, wide = min(kProductBand, mt - band * kProductBand);
        p.m0 = (band * kProductBand + j % wide) * kProductM;
        p.n0 = first_row + j / wide * each;
        p.n = min(each, end - p.n0);
        p.row = p.n0;
        p.end = p.n0 + p.n;
        p.all_steps = (a.k + kProductK - 1u) / kProductK;
    }
    p.half = ((p.n + 31u) & ~31u) / 2u;
    p.step0 = 0; p.steps = p.all_steps;
    if constexpr (SPLIT) {
        p.step0 = (uint32_t)((uint64_t)p.all_steps * share / a.splits);
        p.steps = (uint32_t)((uint64_t)p.all_steps * (share + 1u) / a.splits) - p.step0;
    }
    p.clears = MODE == kWeights && p.steps && p.step0 + p.steps == p.all_steps && (p.end - p.row) % kProductK != 0u;
    return p;
}

// Rows and tiles of each expert, from the starts; every thread of the block.
template <int MODE> __device__ __forceinline__ void product_tables(const ProductArgs& a, ProductShared& s) {
    const uint32_t lane = threadIdx.x & 31u, mt = (a.m + kProductM - 1u) / kProductM;
    if (threadIdx.x < 32u) {                              // (starts that do not ascend, or lie beyond the rows: no rows)
        uint32_t row = 0;
        for (uint32_t e0 = 0; e0 <= a.experts; e0 += 32u) {
            const uint32_t e = e0 + lane;
            uint32_t at = e <= a.experts ? min(a.starts[e], a.rows) : 0u;
#pragma unroll
            for (uint32_t d = 1; d < 32u; d *= 2u) {
                const uint32_t up = __shfl_up_sync(kFullMask, at, d);
                if (lane >= d) at = max(at, up);
            }
            at = max(at, row);
            if (e <= a.experts) s.first_row[e] = at;
            row = __shfl_sync(kFullMask, at, 31);
        }
    }
    __syncthreads();
    // (weights) The experts in descending order of their rows, so that pairs of blocks, which take tiles in turn (there and back), have about as much
    // to do.  (Of more experts each pair has many tiles, whose sums differ little.)
    for (uint32_t e = threadIdx.x; e < a.experts; e += kProductThreads) {
        uint32_t place = e;
        if (MODE == kWeights && a.experts <= kProductSorted) {
            auto rows = [&](uint32_t i) { return s.first_row[i + 1u] - s.first_row[i]; };
            const uint32_t mine = rows(e);
            place = 0;
            for (uint32_t i = 0; i < a.experts; ++i) { const uint32_t other = rows(i); place += other > mine || (other == mine && i < e); }
        }
        s.expert_at[place] = (uint16_t)e;
    }
    __syncthreads();
    if constexpr (MODE == kWeights) {
        if (threadIdx.x == 0) s.tiles = a.experts * mt * ((a.n + a.most_n - 1u) / a.most_n);
    } else if (threadIdx.x < 32u) {
        uint32_t tiles = 0;
        for (uint32_t i0 = 0; i0 < a.experts; i0 += 32u) {
            const uint32_t i = i0 + lane, e = i < a.experts ? s.expert_at[i] : 0u;
            const uint32_t mine = i < a.experts ? (s.first_row[e + 1u] - s.first_row[e] + a.most_n - 1u) / a.most_n * mt : 0u;
            uint32_t sum = mine;
#pragma unroll
            for (uint32_t d = 1; d < 32u; d *= 2u) {
                const uint32_t up = __shfl_up_sync(kFullMask, sum, d);
                if (lane >= d) sum += up;
            }
            if (i < a.experts) s.first_tile[i] = tiles + sum - mine;
            tiles += __shfl_sync(kFullMask, sum, 31);
        }
        if (lane == 0u) s.tiles = tiles;
    }
    __syncthreads();
}
// The tile of a pair's round.
__device__ __forceinline__ uint32_t product_turn(uint32_t round, uint32_t pair, uint32_t pairs) { return round * pairs + (round & 1u ? pairs - 1u - pair : pair); }

// Rows of a stage's strips from `left` on become zero: what lies behind an expert's last row counts nothing, whatever it holds.  One warp; the
// products may be issued by the other block, which learns of it by an arrival that releases at the cluster's scope.
__device__ __forceinline__ void product_clear(uint32_t from, uint32_t strips, uint32_t left) {
    for (uint32_t j = 0; j < strips; ++j)
        for (uint32_t c = left * 8u + (threadIdx.x & 31u); c < kProductK * 8u; c += 32u)
            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(from + j * 8192u + c * 16u), "r"(0u) : "memory");
    fence_async_reads();
    __syncwarp();
}

// A shared contraction: a block keeps its sums in lines that lie as those of the result do, a line a column of the tile (forward, input) or a row of it.
// Words of a line (weights: a vector more than 256, which keeps rows off one another's banks).
template <int MODE> __device__ __forceinline__ constexpr uint32_t product_line() { return MODE == kWeights ? 260u : kProductM / 2u; }
// Each of the cluster's blocks adds up every splits-th line of its half of the tile, in the order of the shares: a warp a line, four values a lane.  The
// eight warps that write (they have the registers).
template <class TO, int MODE> __device__ __forceinline__ void product_join(const ProductArgs& a, ProductShared& s, const ProductTile& p, uint32_t stage0, uint32_t share, uint32_t block) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32u - 4u;
    bool lost = lane < 2u * a.splits && load_from(address_in(&s.lost, lane % (2u * a.splits))) != 0u;
    lost = __any_sync(kFullMask, lost);
    const uint32_t along = MODE == kWeights ? p.n : kProductM / 2u, lines = MODE == kWeights ? kProductM / 2u : p.n, row0 = p.m0 + block * (kProductM / 2u);
    for (uint32_t line = share + a.splits * warp; line < lines; line += a.splits * 8u)
        for (uint32_t i = 4u * lane; i < along; i += 128u) {
            if (MODE == kWeights ? row0 + line >= a.m : row0 + i >= a.m) continue;      // (a.m is a multiple of 8)
            float4 part[8];
            float sum[4] = {};
#pragma unroll
            for (uint32_t j = 0; j < 8u; ++j) if (j < a.splits) part[j] = load_four_from(address_in_cluster(stage0 + 4u * (line * product_line<MODE>() + i), 2u * j + block));
#pragma unroll
            for (uint32_t j = 0; j < 8u; ++j) if (j < a.splits) { sum[0] += part[j].x; sum[1] += part[j].y; sum[2] += part[j].z; sum[3] += part[j].w; }
#pragma unroll
            for (int j = 0; j < 4; ++j) if (lost) sum[j] = __uint_as_float(0x7FC00000u);
            TO* to = static_cast<TO*>(a.out) + (MODE == kWeights ? p.expert * a.out_expert + (row0 + line) * a.out_stride + p.n0 + i : (uint64_t)(p.n0 + line) * a.out_stride + row0 + i);
            if constexpr (sizeof(TO) == 4) *reinterpret_cast<float4*>(to) = make_float4(sum[0], sum[1], sum[2], sum[3]);
            else *reinterpret_cast<uint2*>(to) = make_uint2(pack_two<TO>(sum[0], sum[1]), pack_two<TO>(sum[2], sum[3]));
        }
}

template <class TO, int MODE, bool SUMS, bool SPLIT> __global__ void __launch_bounds__(kProductThreads, 1) k_product(const __grid_constant__ ProductArgs a) {
    extern __shared__ unsigned char raw[];
    __shared__ ProductShared s;
    const uint32_t warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31u;
    // the pair's first block, this one of the two, the pair's share of a contraction (pairs of a cluster), and the pair, or cluster, among all
    const uint32_t leader = SPLIT ? cluster_block() & ~1u : 0u, block = blockIdx.x & 1u, share = leader / 2u, both = 3u << leader;
    const uint32_t splits = SPLIT ? a.splits : 1u, pair = blockIdx.x / (2u * splits), pairs = gridDim.x / (2u * splits);
    const uint32_t stage0 = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t stage_bytes = product_stage_bytes<MODE>(a.most_n);
    uint32_t columns = 32u;
    while (columns < 2u * a.most_n) columns *= 2u;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < a.stages; ++i) { mbar_init(&s.landed[i], 1u); mbar_init(&s.full[i], 2u); mbar_init(&s.empty[i], 1u); }
        for (uint32_t i = 0; i < 2u; ++i) { mbar_init(&s.ready[i], 1u); mbar_init(&s.taken[i], 16u); }
        mbar_init(&s.drained, 1u);
        s.lost = 0u; s.gave_up = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (warp == 3u) tmem_alloc(&s.tmem, columns);
    tmem_before_barrier();
    __syncthreads();
    cluster_meet();
    tmem_after_barrier();
    const uint32_t tmem = s.tmem;
    wait_for_previous_kernels();
    allow_next_kernel();
    product_tables<MODE>(a, s);
    const uint32_t tiles = s.tiles;
    // (SUMS: of 168 registers a thread at launch 96 x 128 + 200 x 256 are less than 168 x 384)
    if (warp >= 4u) {                                     // results
        if constexpr (SUMS) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        uint32_t turn = 0;
        bool fine = true;
        const uint32_t part = warp & 3u, side = (warp - 4u) >> 2;         // lanes; every other 32 columns
        const uint32_t turned = stage0 + a.stages * stage_bytes + (warp - 4u) * kProductTurned;      // (weights)
        for (uint32_t t = pair, turns = 0; turns * pairs < tiles; t = product_turn(++turns, pair, pairs)) {
            if (t >= tiles) continue;
            const ProductTile p = product_tile<MODE, SPLIT>(a, s, t, share);
            const uint32_t row0 = p.m0 + block * kProductM / 2u + 32u * part;
            const uint32_t from = tmem + (32u * part << 16);
            auto write = [&](const float (&f)[32], uint32_t c0) {
                if constexpr (SPLIT) {                    // (a shared contraction: this pair's sums, where its operands were, for all to add up)
                    const uint32_t row = 32u * part + lane;
                    if constexpr (MODE == kWeights) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(stage0 + 4u * (row * product_line<MODE>() + c0 + (uint32_t)i)), "f"(f[i]), "f"(f[i + 1]), "f"(f[i + 2]), "f"(f[i + 3]) : "memory");
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (c0 + (uint32_t)i < p.n) asm volatile("st.shared.f32 [%0], %1;" ::"r"(stage0 + 4u * ((c0 + (uint32_t)i) * product_line<MODE>() + row)), "f"(f[i]) : "memory");
                    }
                    if (!fine) s.lost = 1u;
                } else if constexpr (MODE == kWeights) {
                    // A lane holds 32 columns of a row of its own: 64 bytes of each of 32 rows at a time go through shared memory (in
                    // the order of vectors that a copy of 64-byte rows has, which keeps rows off one another's banks) and from there by a copy.
                    constexpr uint32_t V = Vec<TO>::N, COLS = 4u * V;
#pragma unroll
                    for (uint32_t h = 0; h < 32u; h += COLS) {
                        if (c0 + h >= p.n || row0 >= a.m) continue;
                        if (elect_one()) wait_stores_read<0>();      // (the copy before has read it)
                        __syncwarp();
#pragma unroll
                        for (uint32_t v = 0; v < 4u; ++v) {
                            const uint32_t i = h + v * V;
                            uint4 x;
                            if constexpr (sizeof(TO) == 4) x = make_uint4(__float_as_uint(f[i]), __float_as_uint(f[i + 1]), __float_as_uint(f[i + 2]), __float_as_uint(f[i + 3]));
                            else x = make_uint4(pack_two<TO>(f[i], f[i + 1]), pack_two<TO>(f[i + 2], f[i + 3]), pack_two<TO>(f[i + 4], f[i + 5]), pack_two<TO>(f[i + 6], f[i + 7]));
                            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(turned + lane * 64u + ((v ^ (lane >> 1 & 3u)) << 4)), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
                        }
                        fence_async_reads();
                        __syncwarp();
                        if (elect_one()) {
                            tile_store_3d(&a.out_map, (int)(p.n0 + c0 + h), (int)row0, (int)p.expert, turned);
                            stores_end_group();
                        }
                    }
                } else {
                    if (row0 + lane < a.m) {
                        TO* to = static_cast<TO*>(a.out) + (uint64_t)(p.n0 + c0) * a.out_stride + row0 + lane;
#pragma unroll
                        for (int i = 0; i < 32; ++i) if (c0 + (uint32_t)i < p.n) to[(uint64_t)i * a.out_stride] = from_float<TO>(f[i]);
                    }
                }
            };
            auto wait = [&]() {
                if (fine) fine = __all_sync(kFullMask, mbar_wait_cluster(&s.ready[turn & 1u], turn / 2u & 1u, a.tries));
                __syncwarp();
                tmem_after_barrier();
            };
            auto give_back = [&]() {
                tmem_before_barrier();
                __syncwarp();
                if (lane == 0u) mbar_tell(&s.taken[turn & 1u], leader);
                ++turn;
            };
            // (no rows: zero; a wait that ran out: not a number)
            auto not_a_number = [&](float (&f)[32]) {
#pragma unroll
                for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(0x7FC00000u);
            };
            if constexpr (SUMS) {
                float sum[4][32];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) sum[j][i] = 0.f;
                }
                for (uint32_t step = 0; step < p.steps; step += a.sum_stages) {
                    wait();
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t c0 = 64u * (uint32_t)j + 32u * side;
                        if (c0 >= p.n) continue;
                        uint32_t r[16], q[16];
                        tmem_load(from + (turn & 1u) * a.most_n + c0, r);
                        tmem_wait(r);
                        tmem_load(from + (turn & 1u) * a.most_n + c0 + 16u, q);
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[j][i] += __uint_as_float(r[i]);
                        tmem_wait(q);
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[j][16 + i] += __uint_as_float(q[i]);
                    }
                    give_back();
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t c0 = 64u * (uint32_t)j + 32u * side;
                    if (!fine) not_a_number(sum[j]);
                    if (c0 < p.n) write(sum[j], c0);
                }
            } else {
                // 64 columns at a time; the accumulator is given back before the last of them are written
                if (p.steps) wait();
                const uint32_t at = from + (turn & 1u) * a.most_n + 32u * side;
                for (uint32_t c0 = 32u * side; c0 < p.n || c0 == 32u * side; c0 += 128u) {
                    float f[2][32] = {};
                    if (p.steps) {
                        __syncwarp();                     // (a warp reads an accumulator as one: its lanes, or the one that copies, may have written apart)
#pragma unroll
                        for (uint32_t j = 0; j < 2u; ++j) if (c0 + 64u * j < p.n) tmem_load(at + (c0 - 32u * side) + 64u * j, reinterpret_cast<uint32_t (&)[32]>(f[j]));
#pragma unroll
                        for (uint32_t j = 0; j < 2u; ++j) tmem_wait(reinterpret_cast<uint32_t (&)[32]>(f[j]));
                        if (c0 + 128u >= p.n) give_back();
                    }
#pragma unroll
                    for (uint32_t j = 0; j < 2u; ++j) {
                        if (!fine) not_a_number(f[j]);
                        if (c0 + 64u * j < p.n) write(f[j], c0 + 64u * j);
                    }
                }
            }
        }
        if constexpr (MODE == kWeights && !SPLIT) if (elect_one()) wait_stores();
    } else {
        if constexpr (SUMS) asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
        auto give_up = [&]() {                            // (both blocks of the pair know before they meet at the end)
            for (uint32_t i = 0; i < 2u; ++i) store_word_to(address_in(&s.gave_up, leader + i), 1u);
        };
        if (warp == 0u) {                                     // copies of tiles
            if (elect_one()) {
                ProductRing ring;
                uint32_t issued = 0, cleared = 0, parity = 0;         // (weights, a bit a stage) its last copies are `landed`'s; of that barrier
                bool fine = true;
                const uint32_t full0 = address_in(s.full, leader), landed0 = address_in(s.landed, leader + block);
                for (uint32_t t = pair, turns = 0; turns * pairs < tiles && fine; t = product_turn(++turns, pair, pairs)) {
                    if (t >= tiles) continue;
                    const ProductTile p = product_tile<MODE, SPLIT>(a, s, t, share);
                    const uint32_t boxes = (p.half + a.box - 1u) / a.box, strips = (p.half + 63u) / 64u;
                    const uint32_t bytes = kProductM / 2u * 128u + (MODE == kWeights ? strips * 8192u : boxes * a.box * 128u);
                    const int m0 = (int)(p.m0 + block * kProductM / 2u);
                    const int n0 = (int)((MODE == kWeights ? p.n0 : p.row) + block * p.half);
                    int at = (int)((MODE == kWeights ? p.row : 0u) + p.step0 * kProductK);      // in the contraction
                    for (uint32_t step = 0; step < p.steps; ++step, at += (int)kProductK) {
                        fine = mbar_wait_cluster(&s.empty[ring.stage], ring.round ^ 1u, a.tries);
                        if (!fine) break;
                        const uint32_t to_a = stage0 + ring.stage * stage_bytes, to_b = to_a + kProductM / 2u * 128u;
                        // Both blocks' copies complete on the first block's barrier, for the products that read them; where rows are to be
                        // cleared, on one of their own block's.
                        uint32_t bar = full0 + 8u * ring.stage;
                        if constexpr (MODE == kWeights) {
                            const uint32_t bit = 1u << ring.stage;
                            cleared &= ~bit;
                            if (p.clears && step + 1u == p.steps) { bar = landed0 + 8u * ring.stage; cleared |= bit; parity ^= bit; }
                        }
                        mbar_expect_tx_at(bar, bytes);
                        if constexpr (MODE == kForward) tile_load_3d(to_a, &a.a_map, at, m0, (int)p.expert, bar);
                        else if constexpr (MODE == kInput) {
                            tile_load_3d(to_a, &a.a_map, m0, at, (int)p.expert, bar);
                            tile_load_3d(to_a + 8192u, &a.a_map, m0 + 64, at, (int)p.expert, bar);
                        } else {
                            tile_load_2d(to_a, &a.a_map, m0, at, bar);
                            tile_load_2d(to_a + 8192u, &a.a_map, m0 + 64, at, bar);
                        }
                        if constexpr (MODE == kWeights) {
                            tile_load_2d(to_b, &a.b_map, n0, at, bar);
                            if (strips > 1u) tile_load_2d(to_b + 8192u, &a.b_map, n0 + 64, at, bar);
                        } else for (uint32_t j = 0; j < boxes; ++j) tile_load_2d(to_b + j * a.box * 128u, &a.b_map, at, n0 + (int)(j * a.box), bar);
                        ring.next(a.stages);
                        ++issued;
                    }
                }
                // what is still on its way to a barrier of this block's alone lands before it ends
                for (uint32_t i = 0; i < a.stages; ++i) if (cleared >> i & 1u) mbar_wait(&s.landed[i], (parity >> i & 1u) ^ 1u);
                for (uint32_t i = 0; i < 2u; ++i) {
                    store_word_to(address_in(&s.issued[block], leader + i), issued);
                    store_word_to(address_in(&s.cleared[block], leader + i), cleared);
                }
                if (!fine) give_up();
            }
        } else if (warp == 1u && block == 0u) {               // products
            if (elect_one()) {
                ProductRing ring;
                uint32_t turn = 0;
                bool fine = true;
                for (uint32_t t = pair, turns = 0; turns * pairs < tiles && fine; t = product_turn(++turns, pair, pairs)) {
                    if (t >= tiles) continue;
                    const ProductTile p = product_tile<MODE, SPLIT>(a, s, t, share);
                    const uint32_t shape = product_shape(a.kind, kProductM, 2u * p.half);
                    uint32_t acc = 0, piece = 0;
                    for (uint32_t step = 0; step < p.steps; ++step) {
                        const bool begins = SUMS ? piece == 0u : step == 0u, ends = step + 1u == p.steps || (SUMS && piece + 1u == a.sum_stages);
                        piece = ends ? 0u : piece + 1u;
                        if (begins) {
                            fine = mbar_wait_cluster(&s.taken[turn & 1u], (turn >> 1 & 1u) ^ 1u, a.tries);
                            acc = tmem + (turn & 1u) * a.most_n;
                        }
                        fine = fine && mbar_wait_cluster(&s.full[ring.stage], ring.round, a.tries);
                        if (!fine) { give_up(); break; }
                        tmem_after_barrier();
                        const uint32_t from_a = stage0 + ring.stage * stage_bytes, from_b = from_a + kProductM / 2u * 128u;
                        const uint32_t da = operand_at(from_a, MODE == kForward ? 0u : 8192u), db = operand_at(from_b, MODE == kWeights ? 8192u : 0u);
                        constexpr uint32_t STEP_A = (MODE == kForward ? 32u : 2048u) >> 4, STEP_B = (MODE == kWeights ? 2048u : 32u) >> 4;
#pragma unroll
                        for (uint32_t i = 0; i < kProductK / 16u; ++i) multiply(acc, da + STEP_A * i, db + STEP_B * i, shape, !begins || i);
                        products_arrive(&s.empty[ring.stage], both);
                        if (ends) { products_arrive(&s.ready[turn & 1u], both); ++turn; }
                        ring.next(a.stages);
                    }
                }
                products_arrive(&s.drained, both);                  // no product is under way any more when the accumulators are given back
                mbar_wait(&s.drained, 0u);
            }
        } else if (warp == 1u) {
            mbar_wait(&s.drained, 0u);                        // (every signal of the other block's products has come)
        } else if (MODE == kWeights && warp >= 2u) {          // rows behind an expert's last: two warps, each with stages of its own
            uint32_t issued = 0, parity = 0;
            for (uint32_t t = pair, turns = 0; turns * pairs < tiles; t = product_turn(++turns, pair, pairs)) {
                if (t >= tiles) continue;
                const ProductTile p = product_tile<MODE, SPLIT>(a, s, t, share);
                issued += p.steps;
                if (!p.clears) continue;
                const uint32_t stage = (issued - 1u) % a.stages;
                // a warp's stages: of six or eight, and of every other one of them, about half (whoever waits for a barrier waits for each of its
                // rounds: a parity tells no more than two apart)
                if ((stage ^ stage / 2u ^ warp) & 1u) continue;
                if (!__all_sync(kFullMask, mbar_wait(&s.landed[stage], parity >> stage & 1u, a.tries))) break;
                parity ^= 1u << stage;
                product_clear(stage0 + stage * stage_bytes, kProductM / 128u + (p.half + 63u) / 64u, (p.end - p.row) % kProductK);
                if (lane == 0u) mbar_arrive_at(&s.full[stage], leader);
            }
        }
    }
    __syncwarp();
    tmem_before_barrier();
    __syncthreads();
    cluster_meet();                                       // (neither block ends, or frees its accumulators, while the other's products or signals may need it)
    tmem_after_barrier();
    if (warp == 3u) tmem_free(tmem, columns);
    // Where a thread gave up, copies may still be on their way to either block: the first block waits for the last of each stage, in the place of a
    // block that did not come so far.  (One that did has seen the products of the round before, so the other was there, too.)
    const bool gave_up = s.gave_up != 0u;
    if (gave_up && warp == 0u && block == 0u && elect_one()) {
        const uint32_t most = max(s.issued[0], s.issued[1]), least = min(s.issued[0], s.issued[1]), cleared = s.cleared[s.issued[0] < s.issued[1]];
        for (uint32_t i = 0; i < min(most, a.stages); ++i) {
            const uint32_t round = (most - 1u - i) / a.stages;
            if (cleared >> i & 1u) continue;
            if (least <= i + round * a.stages) mbar_arrive(&s.full[i]);
            mbar_wait_cluster(&s.full[i], round & 1u);
        }
    }
    if constexpr (SPLIT) {
        if (warp >= 4u && pair < tiles) product_join<TO, MODE>(a, s, product_tile<MODE, SPLIT>(a, s, pair, share), stage0, share, block);
    }
    if (SPLIT || gave_up) cluster_meet();                 // (no block ends while others read its sums, or its copies are on their way)
}

}  // namespace fsg
