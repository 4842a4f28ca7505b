// Ids put in order: positions by (id, position), where each id's begin, and the ids that occur.  What the gradient of an embedding
// and a router's experts are both worked by.
//
// A stable sort by digits, lowest first, of 10 bits at most: one digit for a router's experts, two for a vocabulary.  Ids outside the
// range become the range itself, the largest key, and are sorted like the others but not written.  Within a warp equal digits find one
// another by a vote on each of their bits; each warp counts its digits in shared memory, so that an element's place is the sum of four numbers: elements of lower
// digits, of its digit in earlier blocks, in earlier warps, and before it in its warp.  No place depends on the order in which threads run.
//
// Up to 2^16 ids are sorted by one cluster of sixteen blocks in its shared memory (k_order): no launch between digits and no
// workspace; up to 2^11 are each compared with all others instead.  More take three launches a digit (k_order_tile counts, k_order_offsets, k_order_tile places), with keys and positions in the workspace.
#pragma once

#include "async.cuh"

namespace fsg {

constexpr int      kOrderThreads  = 1024;
constexpr int      kOrderWarps    = kOrderThreads / 32;
constexpr uint32_t kOrderBlocks   = 16u;                  // of the cluster
constexpr uint32_t kOrderMaxBins  = 1024u;
constexpr uint32_t kOrderRounds   = 4u;                   // elements of a thread of the cluster, at most
constexpr uint32_t kOrderTile     = kOrderThreads * kOrderRounds;
constexpr uint32_t kOrderMaxFew   = kOrderTile * kOrderBlocks;      // ids that the cluster takes
constexpr uint32_t kOrderMaxPairs = 2048u;                // ... by comparing each with all others
constexpr uint32_t kOrderTileRounds = 8u;                 // elements of a thread of a tile (many ids), at most
constexpr uint32_t kOrderMaxRange = 1u << 20;

struct OrderArgs {
    const int32_t* ids;
    uint32_t  count, range;
    uint32_t* order;
    uint32_t* starts;                                     // range + 1
    uint32_t* distinct;                                   // or nullptr
    uint32_t* number;                                     // or nullptr
    uint32_t  passes, bits;                               // digits and their width
    uint32_t  pass;                                       // (many ids) this launch's
    uint32_t  blocks, tile;                               // (many ids) tiles, and ids of each
    uint32_t* keys[2];                                    // (many ids) between passes
    uint32_t* places[2];
    uint32_t* table;                                      // (many ids) bins x blocks: counts, then elements of that digit in earlier tiles
    uint32_t* totals;                                     // (many ids) bins
};

__device__ __forceinline__ uint32_t order_key(const OrderArgs& a, uint32_t i) {
    const uint32_t id = (uint32_t)a.ids[i];
    return id < a.range ? id : a.range;
}
__device__ __forceinline__ uint32_t digit_of(const OrderArgs& a, uint32_t key, uint32_t pass) { return (key >> (pass * a.bits)) & ((1u << a.bits) - 1u); }

// The exclusive sum of one value a thread over the block, and the sum of all; every thread calls it.
__device__ __forceinline__ uint32_t order_scan(uint32_t x, uint32_t* warp_sums, uint32_t* total) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    uint32_t y = x;
#pragma unroll
    for (uint32_t d = 1; d < 32u; d *= 2u) {
        const uint32_t up = __shfl_up_sync(kFullMask, y, d);
        if (lane >= d) y += up;
    }
    if (lane == 31u) warp_sums[warp] = y;
    __syncthreads();
    if (warp == 0u) {
        uint32_t w = warp_sums[lane];
#pragma unroll
        for (uint32_t d = 1; d < 32u; d *= 2u) {
            const uint32_t up = __shfl_up_sync(kFullMask, w, d);
            if (lane >= d) w += up;
        }
        warp_sums[lane] = w;
    }
    __syncthreads();
    const uint32_t before = warp ? warp_sums[warp - 1u] : 0u;
    *total = warp_sums[31];
    __syncthreads();
    return before + y - x;
}

// Each warp's elements of a tile lie next to each other.  Counts the warp's digits in `mine` (bins, zero before) and gives each element the
// number of those of its digit before it in the warp.  `have` elements of this warp; digits beyond are of no account.
template <uint32_t ROUNDS, class Key>
__device__ __forceinline__ void order_rank(uint16_t* mine, uint32_t have, uint32_t bits, Key key_at, uint32_t (&digit)[ROUNDS], uint32_t (&rank)[ROUNDS]) {
    const uint32_t lane = threadIdx.x & 31u;
#pragma unroll
    for (uint32_t j = 0; j < ROUNDS; ++j) digit[j] = 32u * j + lane < have ? key_at(j) : ~0u;
#pragma unroll
    for (uint32_t j = 0; j < ROUNDS; ++j) {
        if (32u * j >= have) continue;
        const bool in = digit[j] != ~0u;
        uint32_t same = __ballot_sync(kFullMask, in);
#pragma unroll
        for (uint32_t b = 0; b < 10u; ++b) {
            if (b >= bits) break;
            const uint32_t set = __ballot_sync(kFullMask, digit[j] >> b & 1u);
            same &= digit[j] >> b & 1u ? set : ~set;
        }
        const uint32_t before = __popc(same & ((1u << lane) - 1u));
        uint32_t old = 0;
        if (in) old = mine[digit[j]];
        __syncwarp();
        if (in && before == 0u) mine[digit[j]] = (uint16_t)(old + __popc(same));
        __syncwarp();
        rank[j] = old + before;
    }
}

// Over the block's warps: counts become the numbers of the same digit in earlier warps; sums[bin]: in all.
__device__ __forceinline__ void order_over_warps(uint16_t* counts, uint32_t bins, uint32_t* sums) {
    if (threadIdx.x < bins) {
        uint32_t sum = 0;
#pragma unroll 8
        for (int w = 0; w < kOrderWarps; ++w) {
            uint16_t* c = counts + (uint32_t)w * bins + threadIdx.x;
            const uint32_t n = *c;
            *c = (uint16_t)sum;
            sum += n;
        }
        sums[threadIdx.x] = sum;
    }
}

__device__ __forceinline__ void store_to(uint32_t at, uint32_t v, uint32_t w) { asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(at), "r"(v), "r"(w) : "memory"); }

struct OrderShared {
    uint32_t sums[kOrderMaxBins];                         // this block's, by digit
    uint32_t base[kOrderMaxBins];                         // places of its first element of each digit
    uint32_t warp_sums[32];
    unsigned long long pair_sums[32];
    unsigned long long of_block;                          // occurrences and ids that occur in this block's part of the range
    uint32_t pad[2];
    uint2    entries[2][kOrderTile];                      // keys and places
    uint16_t counts[kOrderWarps * kOrderMaxBins];         // by warp and digit (as many digits as there are)
};

// The same of two values that are below 2^32, the second in the upper half.
__device__ __forceinline__ unsigned long long order_scan_pair(unsigned long long x, unsigned long long* warp_sums, unsigned long long* total) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    unsigned long long y = x;
#pragma unroll
    for (uint32_t d = 1; d < 32u; d *= 2u) {
        const unsigned long long up = __shfl_up_sync(kFullMask, y, d);
        if (lane >= d) y += up;
    }
    if (lane == 31u) warp_sums[warp] = y;
    __syncthreads();
    unsigned long long w = warp_sums[lane], before = 0, all = 0;
#pragma unroll
    for (uint32_t d = 16; d; d /= 2u) {                   // (every warp sums for itself what lies before it, and all)
        all = d == 16u ? w : all;
        all += __shfl_xor_sync(kFullMask, all, d);
    }
    before = lane < warp ? w : 0ull;
#pragma unroll
    for (uint32_t d = 16; d; d /= 2u) before += __shfl_xor_sync(kFullMask, before, d);
    *total = all;
    __syncthreads();
    return before + y - x;
}

// Where each id's positions begin, from its number of occurrences in starts (one cluster; a slice of the range a block, sixteen ids a thread at a
// time), and the ids that occur: first each block's totals, then, once the cluster has met, the rest.
constexpr uint32_t kOrderEach = 16u;
struct OrderSlice {
    static constexpr uint32_t ROUND = kOrderThreads * kOrderEach;
    uint32_t lo, hi;
    bool aligned, once;                                   // once: what a thread has loaded it keeps
    uint32_t n[kOrderEach];
    unsigned long long before;                            // of the block's, before this thread's

    __device__ __forceinline__ unsigned long long load(const OrderArgs& a, uint32_t v) {
        if (aligned && v + kOrderEach <= hi) {
#pragma unroll
            for (uint32_t i = 0; i < kOrderEach; i += 4u) {
                const uint4 x = __ldcg(reinterpret_cast<const uint4*>(a.starts + v + i));
                n[i] = x.x; n[i + 1] = x.y; n[i + 2] = x.z; n[i + 3] = x.w;
            }
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kOrderEach; ++i) n[i] = v + i < hi ? __ldcg(a.starts + v + i) : 0u;
        }
        unsigned long long sum = 0;
#pragma unroll
        for (uint32_t i = 0; i < kOrderEach; ++i) sum += n[i] + ((unsigned long long)(n[i] != 0u) << 32);
        return sum;
    }
    __device__ __forceinline__ void add_up(const OrderArgs& a, OrderShared& s, uint32_t block) {
        const uint32_t entries = a.range + 1u, slice = ((entries + kOrderBlocks - 1u) / kOrderBlocks + kOrderEach - 1u) / kOrderEach * kOrderEach;
        lo = min(block * slice, entries);
        hi = min(lo + slice, entries);
        aligned = (reinterpret_cast<uintptr_t>(a.starts) & 15u) == 0u;
        once = slice <= ROUND;
        unsigned long long mine = 0, total = 0;
        for (uint32_t v = lo; v < hi; v += ROUND) mine += load(a, v + threadIdx.x * kOrderEach);
        before = order_scan_pair(mine, s.pair_sums, &total);
        if (threadIdx.x == 0) s.of_block = total;
    }
    __device__ __forceinline__ void finish(const OrderArgs& a, OrderShared& s, uint32_t block) {
        // (a warp a block: loads of one instruction from different blocks would come one after the other)
        const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
        if (lane == 0u && warp < kOrderBlocks) {
            const uint32_t from = address_in(&s.of_block, warp);
            s.pair_sums[warp] = load_from(from) | (unsigned long long)load_from(from + 4u) << 32;
        }
        __syncthreads();
        unsigned long long all = lane < kOrderBlocks ? s.pair_sums[lane] : 0ull, at = lane < block ? all : 0ull, total = 0;
#pragma unroll
        for (uint32_t d = 16; d; d /= 2u) { all += __shfl_xor_sync(kFullMask, all, d); at += __shfl_xor_sync(kFullMask, at, d); }
        if (!once) __syncthreads();
        for (uint32_t v0 = lo; v0 < hi; v0 += ROUND) {
            const uint32_t v = v0 + threadIdx.x * kOrderEach;
            unsigned long long here = at + before;
            if (!once) {
                here = at + order_scan_pair(load(a, v), s.pair_sums, &total);
                at += total;
            }
            uint32_t first = (uint32_t)here, rank = (uint32_t)(here >> 32);
            uint32_t first_of[kOrderEach];
#pragma unroll
            for (uint32_t i = 0; i < kOrderEach; ++i) {
                first_of[i] = first;
                first += n[i];
                if (n[i]) { if (a.distinct) a.distinct[rank] = v + i; ++rank; }
            }
            if (aligned && v + kOrderEach <= hi) {
#pragma unroll
                for (uint32_t i = 0; i < kOrderEach; i += 4u)
                    *reinterpret_cast<uint4*>(a.starts + v + i) = make_uint4(first_of[i], first_of[i + 1], first_of[i + 2], first_of[i + 3]);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < kOrderEach; ++i) if (v + i < hi) a.starts[v + i] = first_of[i];
            }
        }
        if (a.number && block == 0u && threadIdx.x == 0) *a.number = (uint32_t)(all >> 32);
    }
};

// One cluster: everything.  Its blocks meet four times for two digits: what does not depend on the others' is done between the same two meetings.
__global__ void __launch_bounds__(kOrderThreads, 1) k_order(const __grid_constant__ OrderArgs a) {
    extern __shared__ __align__(16) unsigned char raw[];
    OrderShared& s = *reinterpret_cast<OrderShared*>(raw);
    const uint32_t block = cluster_block(), lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t bins = 1u << a.bits;
    // slices of a power of two of elements, from 32 a warp on
    uint32_t per_log = 5;                                 // log2 of a warp's
    while ((kOrderBlocks * kOrderWarps << per_log) < a.count) ++per_log;
    const uint32_t slice_log = per_log + 5u, slice = 1u << slice_log;
    const uint32_t begin = min(a.count, block << slice_log), end = min(a.count, begin + slice);
    const uint32_t first = begin + (warp << per_log);
    const uint32_t have = first < end ? min(end - first, 1u << per_log) : 0u;
    const bool several = a.passes > 1u;                   // (one digit: its counts are the ids')
    const bool pairs = several && a.count <= kOrderMaxPairs;
    OrderSlice of;
    if (!pairs) for (uint32_t i = threadIdx.x; i < kOrderWarps * bins / 2u; i += kOrderThreads) reinterpret_cast<uint32_t*>(s.counts)[i] = 0u;
    wait_for_previous_kernels();
    allow_next_kernel();
    if (several) {                                        // (the last entry counts nothing)
        const uint32_t vectors = (reinterpret_cast<uintptr_t>(a.starts) & 15u) == 0u ? (a.range + 1u) / 4u : 0u, thread = block * kOrderThreads + threadIdx.x;
        for (uint32_t i = thread; i < vectors; i += kOrderBlocks * kOrderThreads) reinterpret_cast<uint4*>(a.starts)[i] = make_uint4(0u, 0u, 0u, 0u);
        for (uint32_t v = 4u * vectors + thread; v <= a.range; v += kOrderBlocks * kOrderThreads) a.starts[v] = 0u;
    }
    if (pairs) {                                          // eight threads an element, each an eighth of the others
        uint32_t* keys = reinterpret_cast<uint32_t*>(s.entries);
        for (uint32_t i = threadIdx.x; i < a.count; i += kOrderThreads) keys[i] = order_key(a, i);
        __syncthreads();
        const uint32_t i = block * (kOrderThreads / 8u) + threadIdx.x / 8u, part = threadIdx.x & 7u;
        const uint32_t key = i < a.count ? keys[i] : ~0u;
        uint32_t before = 0;
        for (uint32_t j = part; j < a.count; j += 8u) before += keys[j] < key || (keys[j] == key && j < i);
#pragma unroll
        for (uint32_t d = 1; d < 8u; d *= 2u) before += __shfl_xor_sync(kFullMask, before, d);
        cluster_meet();
        if (part == 0u && key < a.range) {
            atomicAdd(a.starts + key, 1u);
            a.order[before] = i;
        }
        cluster_meet();
        of.add_up(a, s, block);
        cluster_meet();
        of.finish(a, s, block);
        cluster_meet();                                   // (no block ends while others read its shared memory)
        return;
    }
    for (uint32_t i = threadIdx.x; i < end - begin; i += kOrderThreads) s.entries[0][i] = make_uint2(order_key(a, begin + i), begin + i);
    __syncthreads();
    uint32_t from = 0;
    for (uint32_t pass = 0; pass < a.passes; ++pass) {
        const bool last = pass + 1u == a.passes;
        uint16_t* mine = s.counts + warp * bins;
        uint32_t digit[kOrderRounds], rank[kOrderRounds];
        const uint32_t local = warp << per_log;
        order_rank<kOrderRounds>(mine, have, a.bits, [&](uint32_t j) { return digit_of(a, s.entries[from][local + 32u * j + lane].x, pass); }, digit, rank);
        __syncthreads();
        order_over_warps(s.counts, bins, s.sums);
        if (several && last) of.add_up(a, s, block);      // (all occurrences have been counted: the cluster has met since)
        cluster_meet();
        if (several && pass == 0u)                        // occurrences, equal ids of a warp together (all have been cleared)
            for (uint32_t i0 = 0; i0 < end - begin; i0 += kOrderThreads) {
                const uint32_t i = i0 + threadIdx.x;
                const uint32_t key = i < end - begin ? s.entries[0][i].x : a.range;
                const uint32_t same = __match_any_sync(kFullMask, key);
                if (key < a.range && lane == (uint32_t)__ffs((int)same) - 1u) atomicAdd(a.starts + key, (uint32_t)__popc(same));
            }
        uint32_t all = 0, before = 0, total = 0;
        if (threadIdx.x < bins) {
            uint32_t n[kOrderBlocks];
#pragma unroll
            for (uint32_t b = 0; b < kOrderBlocks; ++b) n[b] = load_from(address_in(s.sums + threadIdx.x, b));
#pragma unroll
            for (uint32_t b = 0; b < kOrderBlocks; ++b) {
                all += n[b];
                if (b < block) before += n[b];
            }
        }
        const uint32_t lower = order_scan(all, s.warp_sums, &total);
        if (threadIdx.x < bins) s.base[threadIdx.x] = lower + before;
        __syncthreads();
        if (!several && block == 0u) {
            if (threadIdx.x <= a.range) a.starts[threadIdx.x] = lower;
            const bool occurs = threadIdx.x < a.range && all != 0u;
            const uint32_t rank_of = order_scan(occurs, s.warp_sums, &total);
            if (occurs && a.distinct) a.distinct[rank_of] = threadIdx.x;
            if (a.number && threadIdx.x == 0) *a.number = total;
        }
#pragma unroll
        for (uint32_t j = 0; j < kOrderRounds; ++j) {
            if (digit[j] == ~0u) continue;
            const uint2 x = s.entries[from][local + 32u * j + lane];
            const uint32_t to = s.base[digit[j]] + mine[digit[j]] + rank[j];
            if (last) {
                if (x.x < a.range) a.order[to] = x.y;
            } else store_to(address_in(&s.entries[from ^ 1u][to & (slice - 1u)], to >> slice_log), x.x, x.y);
        }
        from ^= 1u;
        if (several && last) of.finish(a, s, block);
        if (!last) {
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < kOrderWarps * bins / 2u; i += kOrderThreads) reinterpret_cast<uint32_t*>(s.counts)[i] = 0u;
        }
        cluster_meet();                                   // (also: what others read of this block's has been read before it is formed anew, or the block ends)
    }
}

struct OrderTileShared {
    uint32_t sums[kOrderMaxBins];
    uint32_t warp_sums[32];
    uint16_t counts[kOrderWarps * kOrderMaxBins];
};

__device__ __forceinline__ uint32_t many_key(const OrderArgs& a, uint32_t i) { return a.pass ? a.keys[a.pass & 1u][i] : order_key(a, i); }

// Counts of a tile's digits (MODE 0), or its elements to their places (MODE 1).
template <int PLACE> __global__ void __launch_bounds__(kOrderThreads, 1) k_order_tile(const __grid_constant__ OrderArgs a) {
    extern __shared__ __align__(16) unsigned char raw[];
    OrderTileShared& s = *reinterpret_cast<OrderTileShared*>(raw);
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, bins = 1u << a.bits;
    const uint32_t each = a.tile / kOrderWarps, first = blockIdx.x * a.tile + warp * each;
    const uint32_t have = first < a.count ? min(a.count - first, each) : 0u;
    for (uint32_t i = threadIdx.x; i < kOrderWarps * bins / 2u; i += kOrderThreads) reinterpret_cast<uint32_t*>(s.counts)[i] = 0u;
    wait_for_previous_kernels();
    allow_next_kernel();
    __syncthreads();
    uint16_t* mine = s.counts + warp * bins;
    uint32_t digit[kOrderTileRounds], rank[kOrderTileRounds], key[kOrderTileRounds];
    order_rank<kOrderTileRounds>(mine, have, a.bits, [&](uint32_t j) { key[j] = many_key(a, first + 32u * j + lane); return digit_of(a, key[j], a.pass); }, digit, rank);
    __syncthreads();
    order_over_warps(s.counts, bins, s.sums);
    if constexpr (PLACE == 0) {
        if (threadIdx.x < bins) a.table[(uint64_t)threadIdx.x * a.blocks + blockIdx.x] = s.sums[threadIdx.x];
        return;
    }
    uint32_t total = 0;
    const uint32_t lower = order_scan(threadIdx.x < bins ? __ldcg(a.totals + threadIdx.x) : 0u, s.warp_sums, &total);
    if (threadIdx.x < bins) s.sums[threadIdx.x] = lower + __ldcg(a.table + (uint64_t)threadIdx.x * a.blocks + blockIdx.x);
    __syncthreads();
    const bool last = a.pass + 1u == a.passes;
    const uint32_t to_buffer = (a.pass + 1u) & 1u;
#pragma unroll
    for (uint32_t j = 0; j < kOrderTileRounds; ++j) {
        if (digit[j] == ~0u) continue;
        const uint32_t i = first + 32u * j + lane;
        const uint32_t place = a.pass ? a.places[a.pass & 1u][i] : i;
        const uint32_t to = s.sums[digit[j]] + mine[digit[j]] + rank[j];
        a.keys[to_buffer][to] = key[j];
        if (!last) a.places[to_buffer][to] = place;
        else if (key[j] < a.range) a.order[to] = place;
    }
}

// A warp a digit: counts of its tiles become the numbers in earlier tiles.
__global__ void __launch_bounds__(256) k_order_offsets(const __grid_constant__ OrderArgs a) {
    wait_for_previous_kernels();
    allow_next_kernel();
    const uint32_t bin = blockIdx.x * 8u + (threadIdx.x >> 5), lane = threadIdx.x & 31u;
    if (bin >= 1u << a.bits) return;
    uint32_t* row = a.table + (uint64_t)bin * a.blocks;
    uint32_t sum = 0;
    for (uint32_t b0 = 0; b0 < a.blocks; b0 += 32u) {
        const uint32_t b = b0 + lane, n = b < a.blocks ? row[b] : 0u;
        uint32_t y = n;
#pragma unroll
        for (uint32_t d = 1; d < 32u; d *= 2u) {
            const uint32_t up = __shfl_up_sync(kFullMask, y, d);
            if (lane >= d) y += up;
        }
        if (b < a.blocks) row[b] = sum + y - n;
        sum += __shfl_sync(kFullMask, y, 31);
    }
    if (lane == 0u) a.totals[bin] = sum;
}

// Where each id's positions begin: the first place whose key is not below it.
__global__ void __launch_bounds__(256) k_order_starts(const __grid_constant__ OrderArgs a) {
    wait_for_previous_kernels();
    allow_next_kernel();
    const uint32_t* keys = a.keys[a.passes & 1u];
    const uint32_t v = blockIdx.x * 256u + threadIdx.x;
    if (v > a.range) return;
    uint32_t lo = 0, hi = a.count;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2u;
        if (keys[mid] < v) lo = mid + 1u; else hi = mid;
    }
    a.starts[v] = lo;
}

// The ids that occur, from the starts (one cluster).
__global__ void __launch_bounds__(kOrderThreads, 1) k_order_distinct(const __grid_constant__ OrderArgs a) {
    __shared__ uint32_t warp_sums[32], of_block;
    wait_for_previous_kernels();
    allow_next_kernel();
    const uint32_t block = cluster_block(), slice = (a.range + kOrderBlocks - 1u) / kOrderBlocks;
    const uint32_t lo = min(block * slice, a.range), hi = min(lo + slice, a.range);
    uint32_t occur = 0, total = 0;
    for (uint32_t v = lo + threadIdx.x; v < hi; v += kOrderThreads) occur += a.starts[v + 1u] != a.starts[v];
    order_scan(occur, warp_sums, &total);
    if (threadIdx.x == 0) of_block = total;
    cluster_meet();
    uint32_t at = 0, all = 0;
#pragma unroll
    for (uint32_t b = 0; b < kOrderBlocks; ++b) {
        const uint32_t n = load_from(address_in(&of_block, b));
        if (b < block) at += n;
        all += n;
    }
    for (uint32_t v0 = lo; v0 < hi; v0 += kOrderThreads) {
        const uint32_t v = v0 + threadIdx.x;
        const bool occurs = v < hi && a.starts[v + 1u] != a.starts[v];
        const uint32_t rank = order_scan(occurs, warp_sums, &total);
        if (occurs && a.distinct) a.distinct[at + rank] = v;
        at += total;
    }
    if (a.number && block == 0u && threadIdx.x == 0) *a.number = all;
    cluster_meet();
}

}  // namespace fsg
