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
// One pass over the row in tiles.  A vector of 16 bytes whose maximum is below the bar cannot hold one of the k pairs: its
// exponentials are summed and it is forgotten.  The others are kept as they are in shared memory; when they are many, and at the
// end, their elements above the bar become candidates, and the rest of them joins the sum.  When there are many candidates, the k-th largest
// is found by histograms of eight bits, the smaller ones join the sum and the bar rises to it.
//
// The first tile is a sample of the row (its 512-byte pieces lie apart as many pieces as there are tiles).  The first bar is the
// maximum of one of its vectors, of the place from above that the k-th of the row has in the sample, five standard deviations
// lower.  Where that turns out too high (fewer than k candidates at the end: values in an order that the sample does not
// meet), the row is gone through again with a bar that is a lower bound for sure: the k-th largest maximum of the first tile.
constexpr int kTopTile = 4;                                // vectors a thread takes per tile
constexpr uint32_t kTopTileVecs = kTopTile * kTopThreads;
constexpr uint32_t kTopKeep = 256u;                        // vectors kept before they are gone through
constexpr uint32_t kTopRoom = kTopKeep + kTopTileVecs + 2u;
constexpr uint32_t kTopHead = 0xFFFFFFFEu, kTopTail = 0xFFFFFFFFu;
constexpr uint32_t kTopStep = 256u;                        // kept vectors gone through at a time
constexpr uint32_t kTopBurst = 8u * kTopStep;              // candidates that they can add
constexpr uint32_t kTopCands = kTopMaxPairs + kTopBurst;
constexpr uint32_t kTopByCount = 384u;                     // candidates that are sorted by counting the larger ones

struct TopShared {
    unsigned long long cand[kTopCands];
    unsigned long long sorted[kTopMaxPairs];
    uint4    ring[2][kTopTile][kTopThreads];               // the tile at hand and the next one
    uint32_t vec[kTopRoom];                                // vectors that are kept, by number; kTopHead, kTopTail: the elements around them
    unsigned long long head[2], tail[2];                   // those elements, as vectors
    uint32_t hist[256];
    uint32_t kept, cands, taken, bin, above, equal;
    float2   join[kTopWarps];
    float4   cluster[8];                                   // in the first block: m, rest and in of every block
    uint32_t count;                                        // for the neighbours: entries of `sorted`
};

// The bin that holds the `need`-th entry counted from the last bin down, how many lie in later bins and in it.  One warp; there are
// at least `need`.
__device__ __forceinline__ void find_bin(TopShared& s, uint32_t need) {
    const int lane = threadIdx.x & 31;
    uint32_t h[8], sum = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += h[i] = s.hist[255 - (8 * lane + i)];
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(kFullMask, upto, o); if (lane >= o) upto += y; }
    uint32_t at = upto - sum;
    if (at < need && need <= upto) {                       // one lane
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (at < need && need <= at + h[i]) { s.bin = 255u - (uint32_t)(8 * lane + i); s.above = at; s.equal = h[i]; }
            at += h[i];
        }
    }
}

// One step of a selection: the histogram of the eight bits at `shift` of the words whose bits above are those of `word`.  Afterwards the
// need-th largest word begins with `word`; true when as many begin with it as are still needed.
template <class W, class EACH>
__device__ __forceinline__ bool select_step(TopShared& s, W& word, uint32_t& need, int shift, W fixed, EACH each) {
    __syncthreads();
    if (threadIdx.x < 256u) s.hist[threadIdx.x] = 0u;
    __syncthreads();
    each([&](W w) { if ((w & fixed) == word) atomicAdd(&s.hist[(uint32_t)(w >> shift) & 255u], 1u); });
    __syncthreads();
    if (threadIdx.x < 32u) find_bin(s, need);
    __syncthreads();
    word |= (W)s.bin << shift;
    need -= s.above;
    return need == s.equal;
}

// The k largest of the n candidates (more than k of them) stay; the others join the sum.  Returns a lower bound of them all: the bar.
template <class T>
__device__ __noinline__ unsigned long long cut_candidates(TopShared& s, uint32_t n, uint32_t k, uint32_t cols, ExpSum* sum, float c, float slack) {
    const uint32_t tid = threadIdx.x;
    unsigned long long word = 0ull;
    uint32_t need = k;
    auto each = [&](auto put) { for (uint32_t i = tid; i < n; i += kTopThreads) put(s.cand[i]); };
    bool done = false;
    for (int shift = 32 + 8 * ((Rank<T>::kBits - 1) / 8); shift >= 32 && !done; shift -= 8)
        done = select_step(s, word, need, shift, shift + 8 > 63 ? 0ull : ~0ull << (shift + 8), each);
    if (!done) {                                           // of the equals, those of the least keys (the bits that no key has are all set)
        const int passes = cols > 1u << 24 ? 4 : cols > 1u << 16 ? 3 : cols > 1u << 8 ? 2 : 1;
        if (passes < 4) word |= 0xFFFFFFFFull & ~0ull << (8 * passes);
        for (int shift = 8 * passes - 8; shift >= 0 && !done; shift -= 8) done = select_step(s, word, need, shift, ~0ull << (shift + 8), each);
    }
    if (tid == 0) s.taken = 0u;
    __syncthreads();
    ExpSum e = *sum;
    for (uint32_t i = tid; i < n; i += kTopThreads) {
        const unsigned long long w = s.cand[i];
        if (w >= word) s.sorted[atomicAdd(&s.taken, 1u)] = w;
        else e.add(value_of_rank<T>((uint32_t)(w >> 32)), c, slack);
    }
    *sum = e;
    __syncthreads();
    for (uint32_t i = tid; i < k; i += kTopThreads) s.cand[i] = s.sorted[i];
    if (tid == 0) s.cands = k;
    __syncthreads();
    return word;
}

// The kept vectors' elements above the bar become candidates, the others join the sum.
template <class T>
__device__ __noinline__ unsigned long long go_through(TopShared& s, const T* z, uint32_t k, unsigned long long cut, uint32_t first_key, uint32_t begin, uint32_t end, uint32_t cols,
                                                      ExpSum* sum, float c, float slack) {
    constexpr int N = Vec<T>::N;
    const uint32_t tid = threadIdx.x, kept = s.kept;
    uint32_t n = s.cands;
    __syncthreads();
    for (uint32_t h0 = 0; h0 < kept; h0 += kTopStep) {
        if (n > kTopMaxPairs) cut = cut_candidates<T>(s, n, k, cols, sum, c, slack);
        const uint32_t h = h0 + tid / 2u, part = tid & 1u;      // two threads a vector
        if (h < kept) {
            ExpSum e = *sum;
            const uint32_t v = s.vec[h];
            uint32_t base = v == kTopHead ? first_key - N : v == kTopTail ? end - (end - first_key) % N : first_key + v * N;
            unsigned long long raw = v == kTopHead ? s.head[part] : v == kTopTail ? s.tail[part] : *(reinterpret_cast<const unsigned long long*>(z + base) + part);
            const T* x = reinterpret_cast<const T*>(&raw);
            base += part * (N / 2);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                if (base + i - begin >= end - begin) continue;
                const unsigned long long w = candidate(rank_of<T>(to_float(x[i])), base + i);
                if (w >= cut) s.cand[atomicAdd(&s.cands, 1u)] = w;
                else e.add(to_float(x[i]), c, slack);
            }
            *sum = e;
        }
        __syncthreads();
        n = s.cands;
        __syncthreads();
    }
    if (n > 2u * k + 256u) cut = cut_candidates<T>(s, n, k, cols, sum, c, slack);
    if (tid == 0) s.kept = 0u;
    __syncthreads();
    return cut;
}

// The k largest of n candidates (all, if there are no more) in descending order to `sorted`; the others join the sum.
template <class T>
__device__ __noinline__ uint32_t sort_candidates(TopShared& s, uint32_t n, uint32_t k, uint32_t cols, ExpSum* sum, float c, float slack) {
    const uint32_t tid = threadIdx.x;
    if (n > kTopByCount && n > k) { cut_candidates<T>(s, n, k, cols, sum, c, slack); n = k; }
    if (n <= kTopByCount) {                                // a candidate's place is the number of larger ones
        constexpr uint32_t kParts = 8u;                    // threads of a candidate, next to each other
        for (uint32_t i0 = 0; i0 < n; i0 += kTopThreads / kParts) {
            const uint32_t i = i0 + tid / kParts, part = tid % kParts;
            const unsigned long long x = i < n ? s.cand[i] : 0ull;
            uint32_t before = 0u;
            for (uint32_t j = part; j < n; j += kParts) before += s.cand[j] > x;
#pragma unroll
            for (uint32_t o = 1u; o < kParts; o <<= 1) before += __shfl_xor_sync(kFullMask, before, o);
            if (i < n && part == 0u) {
                if (before < k) s.sorted[before] = x;
                else sum->add(value_of_rank<T>((uint32_t)(x >> 32)), c, slack);
            }
        }
    } else {                                               // n <= k: a bitonic network
        uint32_t size2 = 512u;
        while (size2 < n) size2 <<= 1;
        for (uint32_t i = tid; i < size2; i += kTopThreads) s.sorted[i] = i < n ? s.cand[i] : 0ull;
        for (uint32_t size = 2u; size <= size2; size <<= 1)
            for (uint32_t step = size >> 1; step; step >>= 1) {
                __syncthreads();
                for (uint32_t i = tid; i < size2 / 2u; i += kTopThreads) {
                    const uint32_t p = 2u * i - (i & (step - 1u)), q = p + step;
                    const unsigned long long x = s.sorted[p], y = s.sorted[q];
                    if ((x < y) == ((p & size) == 0u)) { s.sorted[p] = y; s.sorted[q] = x; }
                }
            }
    }
    __syncthreads();
    return n < k ? n : k;
}

// The elements of a slice that lie before its first vector or behind its last: kept as a vector whose other elements lie outside.
template <class T>
__device__ __forceinline__ void keep_edge(TopShared& s, const T* z, uint32_t which, uint32_t base, uint32_t begin, uint32_t end) {
    T* x = reinterpret_cast<T*>(which == kTopHead ? s.head : s.tail);
    for (int i = 0; i < Vec<T>::N; ++i) x[i] = base + i - begin < end - begin ? z[base + i] : from_float<T>(0.f);
    s.vec[atomicAdd(&s.kept, 1u)] = which;
}

template <class T>
__global__ void __launch_bounds__(kTopThreads, 2) k_top(TopArgs a) {
    extern __shared__ __align__(16) unsigned char top_smem[];
    TopShared& s = *reinterpret_cast<TopShared*>(top_smem);
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    constexpr int N = Vec<T>::N;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5, k = a.k, blocks = cluster.num_blocks(), rank = cluster.block_rank();
    const bool sums = a.lse || a.tail;
    const uint32_t begin = rank * a.slice < a.cols ? rank * a.slice : a.cols, end = begin + a.slice < a.cols ? begin + a.slice : a.cols;
    const uint64_t stride = gridDim.x / blocks;
    // The slice of a row as vectors: in pieces of 32, piece p in tile p % tiles.
    struct Slice { const T* z; const T* body; Span sp; uint32_t pieces, tiles; };
    auto slice_of = [&](uint64_t row) {
        Slice q;
        q.z = static_cast<const T*>(a.z) + row * a.z_stride;
        q.sp = span_of(q.z + begin, end - begin);
        q.body = q.z + begin + q.sp.head;
        q.pieces = (q.sp.vecs + 31u) / 32u;
        q.tiles = q.pieces ? (q.pieces + kTopTileVecs / 32u - 1u) / (kTopTileVecs / 32u) : 1u;
        return q;
    };
    // vector u of this thread's in tile t
    auto place_of = [&](const Slice& q, uint32_t t, int u) { return ((warp + (uint32_t)u * kTopWarps) * q.tiles + t) * 32u + lane; };
    auto fetch = [&](const Slice& q, uint32_t t, uint32_t slot) {
#pragma unroll
        for (int u = 0; u < kTopTile; ++u) {
            const uint32_t v = place_of(q, t, u);
            if (v < q.sp.vecs) copy16_async(&s.ring[slot][u][tid], q.body + (uint64_t)v * N);
        }
        copies_end_group();
    };
    wait_for_previous_kernels();
    uint32_t slot = 0u;
    uint64_t row = blockIdx.x / blocks;
    Slice q = slice_of(row < a.rows ? row : 0);
    if (row < a.rows) fetch(q, 0u, slot);
    for (; row < a.rows; row += stride) {
        if (row != blockIdx.x / blocks) q = slice_of(row);
        const T* z = q.z;
        const uint32_t first_key = begin + q.sp.head;
        // vectors in the first tile: of its pieces all but the row's last are whole
        const uint32_t there = q.pieces ? (q.pieces + q.tiles - 1u) / q.tiles * 32u - ((q.pieces - 1u) % q.tiles ? 0u : q.pieces * 32u - q.sp.vecs) : 0u;
        const float expect = (float)k * (float)there / (float)max(q.sp.vecs, 1u);
        const uint32_t guess = (uint32_t)(expect + 5.f * sqrtf(expect) + 3.f);
        ExpSum e;
        for (bool sure = guess >= k, again = false;; sure = again = true) {
            ExpSums es;
            e = ExpSum();
            unsigned long long cut = 0ull;
            float bar = 0.f;
            uint32_t key_bar = 0u;
            auto vector_at = [&](uint32_t t, int u) { return again ? load16(q.body + (uint64_t)place_of(q, t, u) * N) : s.ring[slot][u][tid]; };
            auto set_bar = [&]() {
                const uint32_t lo = (uint32_t)(cut >> 32);
                bar = lo > rank_of<T>(INFINITY) ? INFINITY : value_of_rank<T>(lo);      // (nothing is below NaN, the value of 0)
                key_bar = ~(uint32_t)cut;
            };
            __syncthreads();
            if (tid == 0) { s.kept = 0u; s.cands = 0u; }
            for (uint32_t t = 0; t < q.tiles; ++t) {
                if (!again) {
                    if (t + 1u < q.tiles) fetch(q, t + 1u, slot ^ 1u);
                    else if (row + stride < a.rows) fetch(slice_of(row + stride), 0u, slot ^ 1u);
                    else copies_end_group();
                    wait_copies<1>();
                }
                if (t == 0u) {
                    uint32_t need = sure ? k : guess;
                    if (need <= there) {
                        uint32_t word = 0u;
                        for (int shift = 8 * ((Rank<T>::kBits - 1) / 8); shift >= 0; shift -= 8) {
                            if (select_step(s, word, need, shift, shift == 24 ? 0u : ~0u << (shift + 8), [&](auto put) {
#pragma unroll 1
                                    for (int u = 0; u < kTopTile; ++u) if (place_of(q, 0u, u) < q.sp.vecs) put(rank_of<T>(Vec<T>::max_nan(vector_at(0u, u))));
                                })) break;
                        }
                        cut = (unsigned long long)word << 32;
                    } else __syncthreads();
                    set_bar();
                    if (tid == 0 && q.sp.head) keep_edge(s, z, kTopHead, first_key - N, begin, end);
                    if (tid == 1 && q.sp.tail) keep_edge(s, z, kTopTail, end - q.sp.tail, begin, end);
                }
                bool many = false;
#pragma unroll
                for (int u = 0; u < kTopTile; ++u) {
                    const uint32_t v = place_of(q, t, u), key = first_key + v * N;
                    if (v >= q.sp.vecs) break;
                    const uint4 raw = vector_at(t, u);
                    const float top = Vec<T>::max_nan(raw);
                    if (!(top < bar) && !(top == bar && key > key_bar)) {
                        const uint32_t h = atomicAdd(&s.kept, 1u);
                        s.vec[h] = v;
                        many |= h >= kTopKeep;
                    } else if (sums) {
                        float x[N];
                        Vec<T>::unpack(raw, x);
                        es.add(x, top, a.c, a.slack);
                    }
                }
                if (!again) slot ^= 1u;
                if (__syncthreads_or(many) || t == q.tiles - 1u) {
                    cut = go_through<T>(s, z, k, cut, first_key, begin, end, a.cols, &e, a.c, a.slack);
                    set_bar();
                }
            }
            const ExpSum w = es.whole();
            e.join(w.m, w.s, a.c);
            if (s.cands >= k || sure) break;
        }
        const uint32_t have = sort_candidates<T>(s, s.cands, k, a.cols, &e, a.c, a.slack);

        // ---- the pairs: a candidate's place is how many of the whole row's are larger -----------------
        if (tid == 0) s.count = have;
        if (blocks > 1u) cluster.sync();
        ExpSum in;
        for (uint32_t i = tid; i < have; i += kTopThreads) {
            const unsigned long long w = s.sorted[i];
            uint32_t place = i;
            for (uint32_t b = 0; b < blocks; ++b) {
                if (b == rank) continue;
                const TopShared& o = *cluster.map_shared_rank(&s, b);
                uint32_t l = 0u, h = o.count;
                while (l < h) { const uint32_t mid = (l + h) >> 1; if (o.sorted[mid] > w) l = mid + 1u; else h = mid; }
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
