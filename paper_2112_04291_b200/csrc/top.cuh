// The k largest of a row of logits as (key, value) pairs, in descending order and, among equals, in ascending order of their keys;
// with them log sum_j exp(z_j / T) and the share of that sum outside of the pairs.
//
// Values are compared by their rank, a word that ascends with them (NaN above all, -0 equal to +0); a candidate is its rank and the
// complement of its key in 64 bits, so that no two are equal and the order in which they are found does not matter.
#pragma once

#include <cooperative_groups.h>

#include "rows.cuh"

namespace fsg {

constexpr int kTopThreads = 512;
constexpr int kTopWarps   = kTopThreads / 32;
constexpr uint32_t kTopMaxPairs = 1024u;

struct TopArgs {
    const void* z; int32_t* keys; void* values; float* lse; float* tail;
    uint64_t rows, z_stride;
    uint32_t cols, k, slice;                               // columns of a row that a block takes (a cluster takes the row)
    float temperature, c, slack;                           // c = log2(e) / T
};

// The rank of a value of T: the fp32 word that ascends with it, without the bits that T never sets.
template <class T> struct Rank;
template <> struct Rank<float> { static constexpr int kBits = 32; };
template <> struct Rank<__nv_bfloat16> { static constexpr int kBits = 16; };
template <> struct Rank<__half> { static constexpr int kBits = 19; };      // (1 + 8 + 10 bits as fp32)
template <class T> __device__ __forceinline__ uint32_t rank_of(float x) {
    const uint32_t b = __float_as_uint(__fadd_rn(x, 0.f));
    return (x != x ? 0xFFC00000u : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) >> (32 - Rank<T>::kBits);
}
template <class T> __device__ __forceinline__ float value_of_rank(uint32_t r) {
    constexpr int S = 32 - Rank<T>::kBits;
    const uint32_t b = r << S | (r >> (Rank<T>::kBits - 1) ? 0u : (1u << S) - 1u);
    return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ __forceinline__ unsigned long long candidate(uint32_t rank, uint32_t key) { return (unsigned long long)rank << 32 | (uint32_t)~key; }

// ---- few columns: a warp per row, all of it in registers -----------------------------------------
// k rounds of a maximum over the lane's values and over the warp, and of the least key that has it.
constexpr int kTopRowsThreads = 256;
constexpr uint32_t kTopRowsMaxCols = 1024u, kTopRowsMaxPairs = 32u;

template <class T, int PER>
__global__ void __launch_bounds__(kTopRowsThreads) k_top_rows(TopArgs a) {
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t row = (uint64_t)blockIdx.x * (kTopRowsThreads / 32) + (threadIdx.x >> 5);
    wait_for_previous_kernels();
    if (row >= a.rows) return;
    const T* z = static_cast<const T*>(a.z) + row * a.z_stride;
    uint32_t r[PER];                                       // rank + 1; 0: taken, or no column
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t j = lane + 32u * i;
        r[i] = j < a.cols ? rank_of<float>(to_float(z[j])) + 1u : 0u;
    }
    uint32_t mine = 0u, my_key = 0u;                       // lane i: the i-th pair
    for (uint32_t n = 0; n < a.k; ++n) {
        uint32_t best = 0u, key = 0xFFFFFFFFu;
#pragma unroll
        for (int i = 0; i < PER; ++i) best = max(best, r[i]);
        best = __reduce_max_sync(kFullMask, best);
#pragma unroll
        for (int i = PER - 1; i >= 0; --i) if (r[i] == best) key = lane + 32u * i;
        key = __reduce_min_sync(kFullMask, key);
#pragma unroll
        for (int i = 0; i < PER; ++i) if (lane + 32u * i == key) r[i] = 0u;
        if (lane == n) { mine = best; my_key = key; }
    }
    if (a.lse || a.tail) {
        const float m = value_of_rank<float>(__shfl_sync(kFullMask, mine, 0) - 1u);
        float in = lane < a.k ? exp2_fast((value_of_rank<float>(mine - 1u) - m) * a.c) : 0.f, rest = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) if (r[i]) rest += exp2_fast((value_of_rank<float>(r[i] - 1u) - m) * a.c);
        in = warp_sum(in);
        rest = warp_sum(rest);
        if (lane == 0) {
            const bool none = m == -INFINITY;
            if (a.lse) a.lse[row] = none ? m : m / a.temperature + logf(rest + in);
            if (a.tail) a.tail[row] = none ? 0.f : rest / (rest + in);
        }
    }
    if (lane < a.k) {
        a.keys[row * a.k + lane] = (int32_t)my_key;
        static_cast<T*>(a.values)[row * a.k + lane] = z[my_key];
    }
}

// ---- many columns: a block or a cluster of blocks per row -----------------------------------------
// One pass over the row in tiles.  A vector of 16 bytes whose maximum is below the bar `lo` (a lower bound of the row's k-th
// largest rank) cannot hold a pair: its exponentials are summed and it is forgotten.  Other vectors are kept as they are in shared
// memory; when they are many, and at the end, the k largest of what is kept are found by histograms of eight bits of their ranks
// (and, among equals, of their keys), the bar rises above the k-th, and what is not among them joins the sum.  The first bar is the k-th
// largest of the maxima of the first tile's vectors.  A row that ascends keeps every vector: slower, never wrong, never out of room.
constexpr int kTopTile = 4;                                // vectors a thread takes per tile
constexpr uint32_t kTopTileVecs = kTopTile * kTopThreads;
constexpr uint32_t kTopKeep = 512u;                        // vectors kept before they are gone through
constexpr uint32_t kTopRoom = kTopKeep + kTopTileVecs + 2u;

struct TopShared {
    unsigned long long cand[2][kTopMaxPairs];
    uint4    raw[kTopRoom];
    uint32_t base[kTopRoom];                               // key of the first element (of the row's first, unaligned ones: modulo 2^32)
    uint32_t hist[256];
    uint32_t kept, taken, total, bin, above, equal;
    float2   join[kTopWarps];
    float    sums[kTopWarps];
    float4   cluster[8];                                   // in the first block: m, rest and in of every block
    uint32_t count;                                        // for the neighbours: candidates of this block | which half << 16
};

// The bin that holds the `need`-th entry counted from the last bin down, how many lie in later bins and in it; the total.  One warp.
__device__ __forceinline__ void find_bin(TopShared& s, uint32_t need) {
    const int lane = threadIdx.x & 31;
    uint32_t h[8], sum = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += h[i] = s.hist[255 - (8 * lane + i)];
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(kFullMask, upto, o); if (lane >= o) upto += y; }
    uint32_t at = upto - sum;
    if (lane == 31) s.total = upto;
    if (at < need && need <= upto) {                       // at most one lane
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (at < need && need <= at + h[i]) { s.bin = 255u - (uint32_t)(8 * lane + i); s.above = at; s.equal = h[i]; }
            at += h[i];
        }
    }
}

// The need-th largest of the words that `each` hands out (BITS significant bits), how many of those equal to it belong to the
// first `need` and how many there are.  False if there are fewer than `need` (no more than that: all of them).
struct Selected { uint32_t word, need, equal; bool found; };
template <int BITS, class EACH>
__device__ __forceinline__ Selected select_word(TopShared& s, uint32_t need, EACH each) {
    Selected r{0u, need, 0u, true};
    constexpr int kPasses = (BITS + 7) / 8;
#pragma unroll 1
    for (int pass = kPasses - 1; pass >= 0; --pass) {
        const int shift = 8 * pass;
        const uint32_t fixed = pass == kPasses - 1 ? 0u : ~0u << (shift + 8);
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < 256u; i += kTopThreads) s.hist[i] = 0u;
        __syncthreads();
        each([&](uint32_t w) { if ((w & fixed) == r.word) atomicAdd(&s.hist[w >> shift & 255u], 1u); });
        __syncthreads();
        if (threadIdx.x < 32u) find_bin(s, r.need);
        __syncthreads();
        if (s.total < r.need) { r.found = false; return r; }        // (first pass only)
        r.word |= s.bin << shift; r.need -= s.above; r.equal = s.equal;
    }
    return r;
}

// f(rank, key, value) for each element of the kept vectors that lies in the slice [begin, end).
template <class T, class F>
__device__ __forceinline__ void each_kept(const TopShared& s, uint32_t kept, uint32_t begin, uint32_t end, F f) {
    constexpr int N = Vec<T>::N;
    for (uint32_t h = threadIdx.x; h < kept; h += kTopThreads) {
        float x[N];
        Vec<T>::unpack(s.raw[h], x);
        const uint32_t base = s.base[h];
#pragma unroll
        for (int i = 0; i < N; ++i) if (base + i - begin < end - begin) f(rank_of<T>(x[i]), base + i, x[i]);
    }
}

// The k largest of the candidates and the kept vectors' elements of rank >= lo become the candidates (all of them, if there are no
// more); the others join the sum.  Returns the new bar.
template <class T>
__device__ __forceinline__ uint32_t go_through(TopShared& s, uint32_t& have, int& from, uint32_t k, uint32_t lo, uint32_t begin, uint32_t end, ExpSum& e, float c, float slack) {
    const uint32_t tid = threadIdx.x, kept = s.kept, n = have;
    const unsigned long long* old = s.cand[from];
    unsigned long long* now = s.cand[from ^ 1];
    const Selected r = select_word<Rank<T>::kBits>(s, k, [&](auto put) {
        for (uint32_t i = tid; i < n; i += kTopThreads) put((uint32_t)(old[i] >> 32));
        each_kept<T>(s, kept, begin, end, [&](uint32_t rank, uint32_t, float) { if (rank >= lo) put(rank); });
    });
    unsigned long long cut = 0ull;                         // candidates from here on belong to the first k
    if (r.found) {
        cut = (unsigned long long)r.word << 32;
        if (r.need < r.equal) {                            // of the equals, those of the least keys
            const Selected q = select_word<32>(s, r.need, [&](auto put) {
                for (uint32_t i = tid; i < n; i += kTopThreads) if ((uint32_t)(old[i] >> 32) == r.word) put((uint32_t)old[i]);
                each_kept<T>(s, kept, begin, end, [&](uint32_t rank, uint32_t key, float) { if (rank == r.word) put(~key); });
            });
            cut |= q.word;
        }
    }
    if (tid == 0) s.taken = 0u;
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kTopThreads) {
        if (old[i] >= cut) now[atomicAdd(&s.taken, 1u)] = old[i];
        else e.add(value_of_rank<T>((uint32_t)(old[i] >> 32)), c, slack);
    }
    each_kept<T>(s, kept, begin, end, [&](uint32_t rank, uint32_t key, float x) {
        const unsigned long long w = candidate(rank, key);
        if (rank >= lo && w >= cut) now[atomicAdd(&s.taken, 1u)] = w;
        else e.add(x, c, slack);
    });
    __syncthreads();
    have = s.taken; from ^= 1;
    __syncthreads();
    if (tid == 0) s.kept = 0u;
    __syncthreads();
    return r.found ? r.word + 1u : lo;
}

// Descending order of n candidates, from cand[from] to the other half: up to 256 by counting the larger ones, more by a bitonic network.
__device__ __forceinline__ void sort_candidates(TopShared& s, uint32_t n, int& from) {
    const uint32_t tid = threadIdx.x;
    unsigned long long* a = s.cand[from];
    if (n <= 256u) {
        constexpr uint32_t kParts = 8u;                    // threads of a candidate, next to each other
        for (uint32_t i0 = 0; i0 < n; i0 += kTopThreads / kParts) {
            const uint32_t i = i0 + tid / kParts, part = tid % kParts;
            const unsigned long long x = i < n ? a[i] : 0ull;
            uint32_t before = 0u;
            for (uint32_t j = part; j < n; j += kParts) before += a[j] > x;
#pragma unroll
            for (uint32_t o = 1u; o < kParts; o <<= 1) before += __shfl_xor_sync(kFullMask, before, o);
            if (i < n && part == 0u) s.cand[from ^ 1][before] = x;
        }
        from ^= 1;
    } else {
        uint32_t size2 = 512u;
        while (size2 < n) size2 <<= 1;
        for (uint32_t i = n + tid; i < size2; i += kTopThreads) a[i] = 0ull;
        for (uint32_t size = 2u; size <= size2; size <<= 1)
            for (uint32_t step = size >> 1; step; step >>= 1) {
                __syncthreads();
                for (uint32_t i = tid; i < size2 / 2u; i += kTopThreads) {
                    const uint32_t p = 2u * i - (i & (step - 1u)), q = p + step;
                    const unsigned long long x = a[p], y = a[q];
                    if ((x < y) == ((p & size) == 0u)) { a[p] = y; a[q] = x; }
                }
            }
    }
    __syncthreads();
}

template <class T>
__global__ void __launch_bounds__(kTopThreads, 2) k_top(TopArgs a) {
    extern __shared__ __align__(16) unsigned char top_smem[];
    TopShared& s = *reinterpret_cast<TopShared*>(top_smem);
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    constexpr int N = Vec<T>::N;
    const uint32_t tid = threadIdx.x, k = a.k, blocks = cluster.num_blocks(), rank = cluster.block_rank();
    const bool sums = a.lse || a.tail;
    const uint32_t begin = rank * a.slice < a.cols ? rank * a.slice : a.cols, end = begin + a.slice < a.cols ? begin + a.slice : a.cols;
    wait_for_previous_kernels();
    if (tid == 0) s.kept = 0u;
    __syncthreads();
    for (uint64_t row = blockIdx.x / blocks; row < a.rows; row += gridDim.x / blocks) {
        const T* z = static_cast<const T*>(a.z) + row * a.z_stride;
        const Span sp = span_of(z + begin, end - begin);
        const T* body = z + begin + sp.head;
        const uint32_t tiles = sp.vecs ? (sp.vecs + kTopTileVecs - 1u) / kTopTileVecs : 1u;
        uint32_t lo = 0u, have = 0u;
        int from = 0;
        float bar = __uint_as_float(0x7FC00000u);          // (nothing is below NaN)
        ExpSum e;
        for (uint32_t t = 0; t < tiles; ++t) {
            const uint32_t v0 = t * kTopTileVecs + tid;
            uint4 raw[kTopTile];
            float top[kTopTile];
#pragma unroll
            for (int u = 0; u < kTopTile; ++u) if (v0 + u * kTopThreads < sp.vecs) raw[u] = load16(body + (uint64_t)(v0 + u * kTopThreads) * N);
#pragma unroll
            for (int u = 0; u < kTopTile; ++u) top[u] = v0 + u * kTopThreads < sp.vecs ? Vec<T>::max_nan(raw[u]) : 0.f;
            if (t == 0) {
                if (sp.vecs >= k) {
                    const Selected r = select_word<Rank<T>::kBits>(s, k, [&](auto put) {
#pragma unroll
                        for (int u = 0; u < kTopTile; ++u) if (v0 + u * kTopThreads < sp.vecs) put(rank_of<T>(top[u]));
                    });
                    lo = r.word;
                    bar = value_of_rank<T>(lo);
                }
                if (tid < 2u && (tid ? tiles == 1u && sp.tail : sp.head)) {
                    // the elements before the first vector, and behind the last (those come with the last tile)
                    T x[N];
                    const uint32_t base = tid ? end - sp.tail : begin + sp.head - N;
#pragma unroll
                    for (int i = 0; i < N; ++i) x[i] = base + i >= begin && base + i < end ? z[base + i] : from_float<T>(0.f);
                    const uint32_t h = atomicAdd(&s.kept, 1u);
                    s.raw[h] = *reinterpret_cast<const uint4*>(x); s.base[h] = base;
                }
            } else if (t == tiles - 1u && tid == 0 && sp.tail) {
                T x[N];
                const uint32_t base = end - sp.tail;
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = base + i < end ? z[base + i] : from_float<T>(0.f);
                const uint32_t h = atomicAdd(&s.kept, 1u);
                s.raw[h] = *reinterpret_cast<const uint4*>(x); s.base[h] = base;
            }
#pragma unroll
            for (int u = 0; u < kTopTile; ++u) {
                const uint32_t v = v0 + u * kTopThreads;
                if (v >= sp.vecs) break;
                if (!(top[u] < bar)) {
                    const uint32_t h = atomicAdd(&s.kept, 1u);
                    s.raw[h] = raw[u]; s.base[h] = begin + sp.head + v * N;
                } else if (sums) {
                    float x[N];
                    Vec<T>::unpack(raw[u], x);
                    e.raise(top[u], a.c, a.slack);
#pragma unroll
                    for (int i = 0; i < N; ++i) e.s += exp2_fast((x[i] - e.m) * a.c);
                }
            }
            __syncthreads();
            if (s.kept > kTopKeep || t == tiles - 1u) {
                lo = go_through<T>(s, have, from, k, lo, begin, end, e, a.c, a.slack);
                bar = lo > rank_of<T>(INFINITY) ? INFINITY : value_of_rank<T>(lo);
            }
        }
        sort_candidates(s, have, from);

        // ---- the pairs: a candidate's place is how many of the whole row's are larger -----------------
        if (tid == 0) s.count = have | (uint32_t)from << 16;
        if (blocks > 1u) cluster.sync();
        const unsigned long long* mine = s.cand[from];
        ExpSum in;
        for (uint32_t i = tid; i < have; i += kTopThreads) {
            const unsigned long long w = mine[i];
            uint32_t place = i;
            for (uint32_t b = 0; b < blocks; ++b) {
                if (b == rank) continue;
                const TopShared& o = *cluster.map_shared_rank(&s, b);
                const uint32_t n = o.count & 0xFFFFu;
                const unsigned long long* other = o.cand[o.count >> 16];
                uint32_t l = 0u, h = n;
                while (l < h) { const uint32_t mid = (l + h) >> 1; if (other[mid] > w) l = mid + 1u; else h = mid; }
                place += l;
            }
            const float x = value_of_rank<T>((uint32_t)(w >> 32));
            if (place < k) {
                const uint32_t key = ~(uint32_t)w;
                a.keys[row * k + place] = (int32_t)key;
                static_cast<T*>(a.values)[row * k + place] = z[key];
                in.add(x, a.c, a.slack);
            } else e.add(x, a.c, a.slack);
        }
        if (sums) {
            e = block_join<kTopWarps>(e, s.join, a.c);
            in = block_join<kTopWarps>(in, s.join, a.c);
            const float top = fmaxf(e.m, in.m);
            const float4 sum = make_float4(top, e.s * exp2_fast((e.m - top) * a.c), in.s * exp2_fast((in.m - top) * a.c), 0.f);
            if (tid == 0) cluster.map_shared_rank(&s, 0)->cluster[rank] = sum;
        }
        if (blocks > 1u) cluster.sync(); else __syncthreads();
        if (sums && rank == 0u && tid == 0) {
            float m = kLowest, rest = 0.f, inside = 0.f;
            for (uint32_t b = 0; b < blocks; ++b) m = fmaxf(m, s.cluster[b].x);
            for (uint32_t b = 0; b < blocks; ++b) {
                const float f = exp2_fast((s.cluster[b].x - m) * a.c);
                rest += s.cluster[b].y * f; inside += s.cluster[b].z * f;
            }
            const bool none = rest + inside == 0.f;        // every logit is -inf
            if (a.lse) a.lse[row] = none ? -INFINITY : m / a.temperature + logf(rest + inside);
            if (a.tail) a.tail[row] = none ? 0.f : rest / (rest + inside);
        }
    }
}

}  // namespace fsg
