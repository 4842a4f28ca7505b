// The k largest of a row of logits as (key, value) pairs, in descending order and, among equals, in ascending order of their keys;
// with them log sum_j exp(z_j / T) and the share of that sum outside of the pairs.
//
// Values are compared by their rank, a word that ascends with them (NaN above all, -0 equal to +0); a candidate is its rank and the
// complement of its key in 64 bits, so that no two are equal and the order in which they are found does not matter.
#pragma once

#include <cooperative_groups.h>

#include "async.cuh"
#include "rows.cuh"

namespace fsg {

constexpr int kTopThreads = 256;
constexpr int kTopWarps   = kTopThreads / 32;
constexpr uint32_t kTopMaxPairs = 1024u;

struct TopArgs {
    const void* z; int32_t* keys; void* values; float* lse; float* tail;
    uint64_t rows, z_stride;
    uint32_t cols, k, slice;                               // columns of a row that a block takes (a cluster takes the row)
    uint32_t claims;                                       // there are more rows than blocks at a time (no clusters then)
    uint32_t by_bar;                                       // few columns: the pairs by a bar, not one by one
    uint32_t tries;                                        // of the wait for a claim's answer
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
// k rounds of a maximum over the lane's values and over the warp, and of the least key that has it; or, for more than a few pairs of
// more than a few columns, by a bar: the k-th largest of the lanes' maxima is a lower bound of the k-th largest value, and what
// reaches it, 1.1 to 1.4 k values if they are unlike, is listed in the order of its keys and placed by counting what is larger.  (More than 32
// candidates: one by one.)  Bound by instructions, 66 % of the issue slots.  Top 8 of 65536 x 256 fp32 with lse: 42.6 us, 1.6 TB/s (one by one: 61).
constexpr int kTopRowsThreads = 256;
constexpr uint32_t kTopRowsMaxCols = 1024u, kTopRowsMaxPairs = 32u;

template <class T, int PER>
__global__ void __launch_bounds__(kTopRowsThreads) k_top_rows(TopArgs a) {
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t row = (uint64_t)blockIdx.x * (kTopRowsThreads / 32) + (threadIdx.x >> 5);
    wait_for_previous_kernels();
    if (row >= a.rows) return;
    const T* z = static_cast<const T*>(a.z) + row * a.z_stride;
    __shared__ uint2 lists[kTopRowsThreads / 32][32];
    uint32_t r[PER];                                       // rank + 1; 0: taken, or no column
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t j = lane + 32u * i;
        r[i] = j < a.cols ? rank_of<float>(to_float(z[j])) + 1u : 0u;
    }
    uint32_t mine = 0u, my_key = 0u, place = lane;         // a pair, and where it stands among the row's
    uint32_t most = 0u;
    bool all_found = false;
    if (PER > 2 && a.by_bar) {
        uint32_t top = r[0];
#pragma unroll
        for (int i = 1; i < PER; ++i) top = max(top, r[i]);
        most = __reduce_max_sync(kFullMask, top);
        uint32_t bar = most, left = top;
        for (uint32_t n = 0;; bar = __reduce_max_sync(kFullMask, left)) {
            n += __popc(__ballot_sync(kFullMask, left == bar));
            if (n >= a.k) break;
            if (left == bar) left = 0u;
        }
        uint32_t found = 0u;
        uint2* list = lists[threadIdx.x >> 5];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const unsigned hits = __ballot_sync(kFullMask, r[i] >= bar);
            const uint32_t at = found + __popc(hits & ((1u << lane) - 1u));
            if (r[i] >= bar && at < 32u) list[at] = make_uint2(r[i], lane + 32u * i);
            found += __popc(hits);
        }
        all_found = found <= 32u;
        if (all_found) {
            __syncwarp();
            if (lane < found) { const uint2 c = list[lane]; mine = c.x; my_key = c.y; }
            place = lane < found ? 0u : 32u;
            for (uint32_t o = 0; o < found; ++o) {         // (the list is in the order of the keys)
                const uint32_t other = __shfl_sync(kFullMask, mine, o);
                place += other > mine || (other == mine && o < lane);
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) if (r[i] >= bar) r[i] = 0u;
        }
    }
    if (!all_found) {
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
        most = __shfl_sync(kFullMask, mine, 0);
    }
    if (a.lse || a.tail) {
        const float m = value_of_rank<float>(most - 1u);
        const float e = mine ? exp2_fast((value_of_rank<float>(mine - 1u) - m) * a.c) : 0.f;
        float in = place < a.k ? e : 0.f, rest = place < a.k ? 0.f : e;
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
    if (place < a.k) {
        a.keys[row * a.k + place] = (int32_t)my_key;
        static_cast<T*>(a.values)[row * a.k + place] = from_float<T>(value_of_rank<float>(mine - 1u));
    }
}

// ---- very few columns and many rows: a lane per row ---------------------------------------------------
// The same rounds within a lane: nothing is exchanged.  Top 2 of 65536 x 8 fp32 with lse: 2.6 us (a warp per row: 14.5), of 65536 x 32: 7.0 (14.5).
constexpr int kTopLanesThreads = 64;

template <class T, int PER>
__global__ void __launch_bounds__(kTopLanesThreads) k_top_lanes(TopArgs a) {
    const uint64_t row = (uint64_t)blockIdx.x * kTopLanesThreads + threadIdx.x;
    const T* z = static_cast<const T*>(a.z);
    const uint32_t unit = row_unit(z, a.z_stride);
    wait_for_previous_kernels();
    if (row >= a.rows) return;
    z += row * a.z_stride;
    uint32_t r[PER];                                       // rank + 1; 0: taken, or no column
#pragma unroll
    for (int j = 0; j < PER; j += 8) {
        const uint32_t there = (uint32_t)j < a.cols ? min(a.cols - j, 8u) : 0u;
        float x[8];
        unpack_eight(load_eight(z + j, there, unit), x);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[j + i] = (uint32_t)i < there ? rank_of<float>(x[i]) + 1u : 0u;
    }
    float m = 0.f, in = 0.f, rest[4] = {};
    int32_t* keys = a.keys + row * a.k;
    T* values = static_cast<T*>(a.values) + row * a.k;
    const bool sums = a.lse || a.tail;
#pragma unroll 1
    for (uint32_t n = 0; n < a.k; ++n) {
        uint32_t best = 0u;
        int key = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) best = max(best, r[i]);
#pragma unroll
        for (int i = PER - 1; i >= 0; --i) if (r[i] == best) key = i;
#pragma unroll
        for (int i = 0; i < PER; ++i) if (i == key) r[i] = 0u;
        const float x = value_of_rank<float>(best - 1u);
        keys[n] = key;
        values[n] = from_float<T>(x);
        if (n == 0u) m = x;
        if (sums) in += exp2_fast((x - m) * a.c);
    }
    if (!sums) return;
#pragma unroll
    for (int i = 0; i < PER; ++i) if (r[i]) rest[i % 4] += exp2_fast((value_of_rank<float>(r[i] - 1u) - m) * a.c);
    const float out = (rest[0] + rest[1]) + (rest[2] + rest[3]);
    const bool none = m == -INFINITY;
    if (a.lse) a.lse[row] = none ? m : m / a.temperature + logf(out + in);
    if (a.tail) a.tail[row] = none ? 0.f : out / (out + in);
}

// ---- many columns: a block or a cluster of blocks per row -----------------------------------------
// One pass over the row in tiles.  A vector of 16 bytes whose maximum is below the bar cannot hold one of the k pairs: its
// exponentials are summed and it is forgotten.  The others are listed, warp by warp, and at the end their elements above the bar
// become candidates, while the others join the sum; the k-th largest candidate is found by histograms of eight bits.  The order in which
// candidates are found changes no sum: those that turn out to be no pairs are added as integers.
// Top 64 of 2048 x 128000 bf16 with lse and tail: 165 to 173 us by the GPU, 3.0 to 3.2 TB/s (525 MB; a copy's time 80).  Neither DRAM (33 %) nor the issue slots
// (47 %, 13 instructions an element and lane) are full: 24 warps an SM wait for their tiles, and for one another in the selection at a row's
// end, of which the other blocks of the SM hide a part.  Every value against a list: 2655; a bar that rises from nothing in place of the sample: 284; all candidates kept
// in one place, a barrier a tile: 245.  One row of 128000 over a cluster of eight blocks: 10.3 us (one block: 91, one barrier fewer a step
// of the selection than before: 16).
//
// The first tile is a sample of the row (its 512-byte pieces lie apart as many pieces as there are tiles), and the bar is the
// maximum of one of its vectors: the one whose place from above the k-th of the row has among them (n in the mean), 5 sqrt(n) + 5 places lower.
// With a bar that turns out too high (fewer than k candidates) or too low (no room for them: values in an order that the sample
// does not meet, or many equal ones) the row is gone through again step by step: from a bar that is a lower bound for sure, the
// k-th largest maximum of the first tile, which rises to the k-th candidate whenever there are many.
constexpr int kTopTile = 4;                                // vectors a thread takes per tile
constexpr uint32_t kTopTileVecs = kTopTile * kTopThreads;
constexpr uint32_t kTopList = 1024u;                       // vectors a warp lists
constexpr uint32_t kTopHead = 0xFFFEu, kTopTail = 0xFFFFu;
constexpr uint32_t kTopMaxCols = 1u << 20;                 // (a listed vector is its number among the warp's, in 16 bits: at most 511 tiles)
static_assert(kTopMaxCols / 4u / kTopTileVecs < 511u, "fp32, four to a vector");
constexpr uint32_t kTopBurst = 8u * kTopThreads + 16u;     // candidates that a step of the careful way can add
constexpr uint32_t kTopByCount = 256u;                     // candidates that are sorted by counting the larger ones
constexpr uint32_t kTopFewPairs = 128u;                    // k up to here: less shared memory

// MOST: the largest k
template <uint32_t MOST> struct TopShared {
    static constexpr uint32_t kRoom = MOST <= kTopFewPairs ? MOST + kTopBurst : 4u * MOST;
    static_assert(kRoom >= MOST + kTopBurst, "a step of the careful way finds room");
    unsigned long long cand[kRoom];
    unsigned long long some[MOST < kTopByCount ? kTopByCount : MOST];
    uint4    ring[2][kTopTile][kTopThreads];               // the tile at hand and the next one
    uint16_t list[kTopWarps][kTopList];                    // vectors as 32 (4 tile + u) + lane; kTopHead, kTopTail: the elements around them
    uint32_t hist[3][256];                                 // of three steps in turn; zero when their turn comes
    uint32_t cands, taken;                                 // (cands may count more than there is room for)
    uint32_t most[kTopWarps];
    uint32_t dropped_most;                                 // the candidates that are no pairs: their largest rank, the sum relative to it
    unsigned long long dropped;
    float2   join[kTopWarps];
    float4   cluster[8];                                   // in the first block: m, rest and in of every block
    uint32_t count;                                        // for the neighbours: entries of `sorted`
    Claim    claim;                                        // the block's next row
};

// One step of a selection: the histogram of the eight bits at `shift` of the words whose `fixed` bits are those of `word` (they may
// overlap those eight).  Afterwards the need-th largest word begins with `word`, and `equal` words do.  One barrier: every warp looks
// the bin up for itself, and the histogram of the step before is cleared for the step after the next.
template <class S, class W, class EACH>
__device__ __forceinline__ void select_step(S& s, uint32_t& step, W& word, uint32_t& need, uint32_t& equal, int shift, W fixed, EACH each) {
    static_assert(kTopThreads == 256, "a bin a thread");
    uint32_t* hist = s.hist[step % 3u];
    each([&](W w) { if ((w & fixed) == word) atomicAdd(&hist[(uint32_t)(w >> shift) & 255u], 1u); });
    __syncthreads();
    const int lane = threadIdx.x & 31;
    uint32_t h[8], sum = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += h[i] = hist[255 - (8 * lane + i)];
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(kFullMask, upto, o); if (lane >= o) upto += y; }
    uint32_t at = upto - sum, bin = 0u, above = 0u, in = 0u;
    const bool here = at < need && need <= upto;           // one lane
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (at < need && need <= at + h[i]) { bin = 255u - (uint32_t)(8 * lane + i); above = at; in = h[i]; }
        at += h[i];
    }
    const int who = __ffs((int)__ballot_sync(kFullMask, here)) - 1;
    word |= (W)__shfl_sync(kFullMask, bin, who) << shift;
    need -= __shfl_sync(kFullMask, above, who);
    equal = __shfl_sync(kFullMask, in, who);
    s.hist[(step + 2u) % 3u][threadIdx.x] = 0u;
    ++step;
}

// A lower bound of at least k and at most `enough` of the n candidates (more than k, none below `floor`): k of them if enough = k.  The
// histograms begin with the highest bit in which the candidates' distances from `floor` differ.
template <class S>
__device__ __forceinline__ unsigned long long cut_of(S& s, uint32_t& step, uint32_t n, uint32_t k, uint32_t enough, unsigned long long floor) {
    const uint32_t tid = threadIdx.x, base = (uint32_t)(floor >> 32);
    const unsigned long long low = (unsigned long long)base << 32;
    uint32_t most = 0u;
    for (uint32_t i = tid; i < n; i += kTopThreads) most = max(most, (uint32_t)(s.cand[i] >> 32) - base);
    most = __reduce_max_sync(kFullMask, most);
    if ((tid & 31u) == 0u) s.most[tid >> 5] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTopWarps; ++w) most = max(most, s.most[w]);
    unsigned long long word = 0ull, fixed = 0ull;
    uint32_t need = k, equal = 0u;
    int shift = 64 - __clz((int)most) - 8;                 // (0 or more: without a difference in rank, the keys' upper bits)
    shift = shift < 24 ? 24 : shift;
    for (;;) {
        select_step(s, step, word, need, equal, shift, fixed, [&](auto put) { for (uint32_t i = tid; i < n; i += kTopThreads) put(s.cand[i] - low); });
        if (k - need + equal <= enough || !shift) break;
        fixed = ~0ull << shift;
        shift = shift > 8 ? shift - 8 : 0;
    }
    return word + low;
}

// The k largest of the n candidates (more than k of them, none below `floor`) stay.  Returns a lower bound of them all: the bar.
template <class S>
__device__ __noinline__ unsigned long long cut_candidates(S& s, uint32_t step, uint32_t n, uint32_t k, unsigned long long floor) {
    const uint32_t tid = threadIdx.x;
    const unsigned long long word = cut_of(s, step, n, k, k, floor);
    if (tid == 0) s.taken = 0u;
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kTopThreads) {
        const unsigned long long w = s.cand[i];
        if (w >= word) s.some[atomicAdd(&s.taken, 1u)] = w;
    }
    __syncthreads();
    for (uint32_t i = tid; i < k; i += kTopThreads) s.cand[i] = s.some[i];
    if (tid == 0) s.cands = k;
    for (int h = 0; h < 3; ++h) s.hist[h][tid] = 0u;       // (the caller's count of steps goes on from anywhere)
    __syncthreads();
    return word;
}

// The slice of a row as vectors: in pieces of 32, piece p in tile p % tiles.  A thread's vector u of tile t is number first + 32 t + step u.
struct TopSlice { uint32_t head, tail, vecs, tiles, first, step; };
template <class T> __device__ __forceinline__ TopSlice top_slice(const T* z, uint32_t n) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const Span sp = span_of(z, n);
    TopSlice q;
    q.head = sp.head; q.tail = sp.tail; q.vecs = sp.vecs;
    q.tiles = sp.vecs ? (sp.vecs + kTopTileVecs - 1u) / kTopTileVecs : 1u;
    q.first = warp * q.tiles * 32u + lane; q.step = kTopWarps * q.tiles * 32u;
    return q;
}
// vectors in the first tile: of its pieces all but the row's last are whole
__device__ __forceinline__ uint32_t first_tile_of(const TopSlice& q) {
    const uint32_t pieces = (q.vecs + 31u) / 32u;
    return pieces ? (pieces + q.tiles - 1u) / q.tiles * 32u - ((pieces - 1u) % q.tiles ? 0u : pieces * 32u - q.vecs) : 0u;
}
// of the four vectors of tile t, those that there are
__device__ __forceinline__ uint32_t vectors_of(const TopSlice& q, uint32_t t) {
    const uint32_t v = q.first + 32u * t;
    return v + (kTopTile - 1u) * q.step < q.vecs ? kTopTile : v < q.vecs ? (q.vecs - 1u - v) / q.step + 1u : 0u;
}

// f(rank << 32 | ~key, value) for the elements of a warp's listed vectors, in the list's order.
template <class T, uint32_t MOST, class F>
__device__ __forceinline__ void each_listed(const TopShared<MOST>& s, const T* z, const TopSlice& q, uint32_t listed, uint32_t begin, uint32_t end, F f) {
    constexpr int N = Vec<T>::N, U = 2;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, first_key = begin + q.head;
    const uint4* body = reinterpret_cast<const uint4*>(z + first_key);
    __syncwarp();
    for (uint32_t h = lane; h < listed; h += 32u * U) {
        uint32_t base[U];
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (h + 32u * u >= listed) continue;
            const uint32_t id = s.list[warp][h + 32u * u];
            if (id < kTopHead) {
                const uint32_t v = q.first - lane + (id & 31u) + 32u * (id >> 7) + q.step * (id >> 5 & 3u);
                base[u] = first_key + v * N;
                raw[u] = load16(body + v);
            } else {
                base[u] = id == kTopHead ? first_key - N : end - q.tail;
                alignas(16) T x[N];
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = base[u] + i - begin < end - begin ? z[base[u] + i] : from_float<T>(0.f);
                raw[u] = *reinterpret_cast<const uint4*>(x);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (h + 32u * u >= listed) continue;
            float x[N];
            Vec<T>::unpack(raw[u], x);
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (base[u] + i - begin < end - begin) f(candidate(rank_of<T>(x[i]), base[u] + i), x[i]);
        }
    }
    __syncwarp();
}
// Those above the bar become candidates, as far as there is room; the others join the sum.
template <class T, uint32_t MOST>
__device__ __noinline__ ExpSum collect(TopShared<MOST>& s, const T* z, uint32_t listed, unsigned long long cut, uint32_t begin, uint32_t end, ExpSum e, float c, float slack) {
    each_listed<T>(s, z, top_slice(z + begin, end - begin), listed, begin, end, [&](unsigned long long w, float x) {
        if (w < cut) { e.add(x, c, slack); return; }
        const uint32_t n = atomicAdd(&s.cands, 1u);
        if (n < TopShared<MOST>::kRoom) s.cand[n] = w;
    });
    return e;
}

// The k largest of n candidates (all, if there are no more) in descending order to cand[0 ...).  Returns this thread's part of the others'
// sum, which does not depend on their order.
template <class T, class S>
__device__ __noinline__ ExpSum sort_candidates(S& s, uint32_t step, uint32_t n, uint32_t k, unsigned long long floor, float c, float slack) {
    const uint32_t tid = threadIdx.x;
    ExpSum e;
    uint32_t some = n;                                     // those that are sorted
    if (tid == 0) { s.taken = 0u; s.dropped_most = 0u; s.dropped = 0ull; }
    if (n > k && (n > kTopByCount || n > k + k / 2u + 32u)) {
        // (up to 256 are sorted by counting: a few more than k do no harm)
        const unsigned long long word = cut_of(s, step, n, k, k <= kTopByCount - 32u ? k + 32u : k, floor);
        uint32_t most = 0u;
        for (uint32_t i = tid; i < n; i += kTopThreads) {
            const unsigned long long w = s.cand[i];
            if (w >= word) s.some[atomicAdd(&s.taken, 1u)] = w; else most = max(most, (uint32_t)(w >> 32));
        }
        most = __reduce_max_sync(kFullMask, most);
        if ((tid & 31u) == 0u) atomicMax(&s.dropped_most, most);
        __syncthreads();
        some = s.taken;
        // relative to the largest of them, in units of 2^-40
        const float m = value_of_rank<T>(s.dropped_most);
        unsigned long long sum = 0ull;
        for (uint32_t i = tid; i < n; i += kTopThreads) {
            const unsigned long long w = s.cand[i];
            if (w < word) sum += (unsigned long long)(exp2_fast((value_of_rank<T>((uint32_t)(w >> 32)) - m) * c) * 1099511627776.f);
        }
        sum = warp_sum(sum);
        if ((tid & 31u) == 0u) atomicAdd(&s.dropped, sum);
        __syncthreads();
        if (tid == 0) { e.m = fmaxf(m, kLowest); e.s = (float)s.dropped * (1.f / 1099511627776.f); }
    } else {
        for (uint32_t i = tid; i < n; i += kTopThreads) s.some[i] = s.cand[i];
        __syncthreads();
    }
    if (some <= kTopByCount) {                             // a candidate's place is the number of larger ones
        constexpr uint32_t kParts = 8u;                    // threads of a candidate, next to each other
        for (uint32_t i0 = 0; i0 < some; i0 += kTopThreads / kParts) {
            const uint32_t i = i0 + tid / kParts, part = tid % kParts;
            const unsigned long long x = i < some ? s.some[i] : 0ull;
            uint32_t before = 0u;
            for (uint32_t j = part; j < some; j += kParts) before += s.some[j] > x;
#pragma unroll
            for (uint32_t o = 1u; o < kParts; o <<= 1) before += __shfl_xor_sync(kFullMask, before, o);
            if (i < some && part == 0u) s.cand[before] = x;
        }
        __syncthreads();
        for (uint32_t i = k + tid; i < some; i += kTopThreads) e.add(value_of_rank<T>((uint32_t)(s.cand[i] >> 32)), c, slack);
    } else {                                               // k of them: a bitonic network
        uint32_t size2 = 2u * kTopByCount;
        while (size2 < some) size2 <<= 1;
        for (uint32_t i = some + tid; i < size2; i += kTopThreads) s.some[i] = 0ull;
        for (uint32_t size = 2u; size <= size2; size <<= 1)
            for (uint32_t step2 = size >> 1; step2; step2 >>= 1) {
                __syncthreads();
                for (uint32_t i = tid; i < size2 / 2u; i += kTopThreads) {
                    const uint32_t p = 2u * i - (i & (step2 - 1u)), q = p + step2;
                    const unsigned long long x = s.some[p], y = s.some[q];
                    if ((x < y) == ((p & size) == 0u)) { s.some[p] = y; s.some[q] = x; }
                }
            }
        __syncthreads();
        for (uint32_t i = tid; i < some; i += kTopThreads) s.cand[i] = s.some[i];
        __syncthreads();
    }
    for (int h = 0; h < 3; ++h) s.hist[h][tid] = 0u;       // (the caller's count of steps goes on from anywhere)
    return e;
}

// a lower bound of the need-th largest rank among the maxima of the first tile's vectors (16 of its bits)
template <class T, class S>
__device__ __forceinline__ unsigned long long first_bar(S& s, uint32_t& step, uint32_t need, uint32_t mine, const float (&top)[kTopTile]) {
    constexpr int kTopBit = Rank<T>::kBits - 8;
    uint32_t word = 0u, equal = 0u;
    auto each = [&](auto put) {
#pragma unroll
        for (int u = 0; u < kTopTile; ++u) if ((uint32_t)u < mine) put(rank_of<T>(top[u]));
    };
    select_step(s, step, word, need, equal, kTopBit, 0u, each);
    select_step(s, step, word, need, equal, kTopBit - 8, ~0u << kTopBit, each);
    return (unsigned long long)word << 32;
}

// The bar as a value, for whole vectors: nothing above it may be missed.
template <class T> __device__ __forceinline__ float bar_value(unsigned long long cut) {
    const uint32_t lo = (uint32_t)(cut >> 32);
    return lo > rank_of<T>(INFINITY) ? INFINITY : value_of_rank<T>(lo);      // (nothing is below NaN, the value of 0)
}

// The careful way through a slice: its candidates.  Returns the bar.
template <class T, uint32_t MOST>
__device__ __noinline__ unsigned long long collect_carefully(TopShared<MOST>& s, uint32_t step, const T* z, uint32_t k, uint32_t begin, uint32_t end) {
    constexpr int N = Vec<T>::N;
    const TopSlice q = top_slice(z + begin, end - begin);
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5, first_key = begin + q.head;
    const uint4* body = reinterpret_cast<const uint4*>(z + first_key);
    unsigned long long cut = 0ull;
    if (tid == 0) s.cands = 0u;
    for (uint32_t t = 0; t < q.tiles; ++t) {
        const uint32_t v = q.first + 32u * t, mine = vectors_of(q, t);
        if (t == 0u) {
            float top[kTopTile];
#pragma unroll
            for (int u = 0; u < kTopTile; ++u) top[u] = (uint32_t)u < mine ? Vec<T>::max_nan(load16(body + v + u * q.step)) : 0.f;
            if (k <= first_tile_of(q)) cut = first_bar<T>(s, step, k, mine, top);
        }
        __syncthreads();
        for (uint32_t u = 0; u < (uint32_t)kTopTile; ++u) {
            const float bar = bar_value<T>(cut);
            uint32_t listed = 0u;
            if (t == 0u && u == 0u && warp == 0u) {
                if (q.head) { if (lane == 0) s.list[0][listed] = kTopHead; ++listed; }
                if (q.tail) { if (lane == 0) s.list[0][listed] = kTopTail; ++listed; }
            }
            bool hit = false;
            if (u < mine) {
                const float top = Vec<T>::max_nan(load16(body + v + u * q.step));
                hit = !(top < bar) && !(top == bar && first_key + (v + u * q.step) * N > ~(uint32_t)cut);
            }
            const unsigned hits = __ballot_sync(kFullMask, hit);
            if (hit) s.list[warp][listed + __popc(hits & ((1u << lane) - 1u))] = (uint16_t)(128u * t + 32u * u + lane);
            collect<T>(s, z, listed + __popc(hits), cut, begin, end, ExpSum(), 0.f, 0.f);
            __syncthreads();
            const uint32_t n = s.cands;
            __syncthreads();
            if (n > MOST) cut = cut_candidates(s, step, n, k, cut);
        }
    }
    for (int h = 0; h < 3; ++h) s.hist[h][tid] = 0u;       // (the bar's steps have left some; the caller's count of steps goes on from anywhere)
    __syncthreads();
    return cut;
}
// ... and the sum of what lies below its last pair, whatever the logits.
template <class T>
__device__ __noinline__ ExpSum sum_carefully(const T* z, unsigned long long last, uint32_t begin, uint32_t end, float c, float slack) {
    ExpSum e;
    for (uint32_t j = begin + threadIdx.x; j < end; j += kTopThreads) {
        const float x = to_float(z[j]);
        if (candidate(rank_of<T>(x), j) < last) e.add(x, c, slack);
    }
    return e;
}

// A row that was never gone through.
template <class T>
__device__ __noinline__ void give_up_pairs(int32_t* keys, T* values, uint32_t k, float* lse, float* tail) {
    for (uint32_t i = threadIdx.x; i < k; i += kTopThreads) { keys[i] = -1; values[i] = from_float<T>(NAN); }
    if (threadIdx.x == 0 && lse) *lse = NAN;
    if (threadIdx.x == 0 && tail) *tail = NAN;
}

template <class T, uint32_t MOST>
__global__ void __launch_bounds__(kTopThreads, MOST <= kTopFewPairs ? 3 : 2) k_top(TopArgs a) {
    extern __shared__ __align__(16) unsigned char top_smem[];
    TopShared<MOST>& s = *reinterpret_cast<TopShared<MOST>*>(top_smem);
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    constexpr int N = Vec<T>::N;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5, k = a.k, blocks = cluster.num_blocks(), rank = cluster.block_rank();
    const bool sums = a.lse || a.tail;
    const uint32_t begin = rank * a.slice < a.cols ? rank * a.slice : a.cols, end = begin + a.slice < a.cols ? begin + a.slice : a.cols;
    auto fetch = [&](const T* z, const TopSlice& q, uint32_t t, uint32_t slot) {
        const uint4* body = reinterpret_cast<const uint4*>(z + begin + q.head);
        uint32_t v = q.first + 32u * t;
#pragma unroll
        for (int u = 0; u < kTopTile; ++u, v += q.step) if (v < q.vecs) copy16_async(&s.ring[slot][u][tid], body + v);
        copies_end_group();
    };
    if (tid == 0) claim_init(s.claim);
    for (int h = 0; h < 3; ++h) s.hist[h][tid] = 0u;
    uint32_t step = 0u;
    wait_for_previous_kernels();
    uint32_t slot = 0u;
    uint64_t row = blockIdx.x / blocks;
    {
        const T* z = static_cast<const T*>(a.z) + row * a.z_stride;
        fetch(z, top_slice(z + begin, end - begin), 0u, slot);
    }
    if (tid == 0 && a.claims) claim_ask(s.claim);
    for (uint32_t turn = 0u;; ++turn) {
        const T* z = static_cast<const T*>(a.z) + row * a.z_stride;
        int next_row = -1;
        const TopSlice q = top_slice(z + begin, end - begin);
        const uint32_t there = first_tile_of(q);
        const float expect = (float)k * (float)there / (float)max(q.vecs, 1u);
        const uint32_t guess = min(k, (uint32_t)(expect + 5.f * sqrtf(expect) + 5.f));
        FusedExpSums es;
        unsigned long long cut = 0ull;
        float bar = 0.f;
        uint32_t listed = 0u;
        __syncthreads();
        if (tid == 0) s.cands = 0u;
        for (uint32_t t = 0; t < q.tiles; ++t) {
            if (t + 1u < q.tiles) fetch(z, q, t + 1u, slot ^ 1u);
            else {
                if (a.claims) next_row = claim_answer(s.claim, turn, a.tries);
                if (next_row >= 0) { const T* next = static_cast<const T*>(a.z) + (uint64_t)next_row * a.z_stride; fetch(next, top_slice(next + begin, end - begin), 0u, slot ^ 1u); }
                else copies_end_group();
            }
            wait_copies<1>();
            uint4 raw[kTopTile];
            float top[kTopTile];
#pragma unroll
            for (int u = 0; u < kTopTile; ++u) raw[u] = s.ring[slot][u][tid];
            slot ^= 1u;
            const uint32_t mine = vectors_of(q, t);
            if (mine < kTopTile) {                         // (the last tiles may be short)
#pragma unroll
                for (int u = 0; u < kTopTile; ++u)
                    if ((uint32_t)u >= mine) raw[u] = make_uint4(Vec<T>::kMinusInf, Vec<T>::kMinusInf, Vec<T>::kMinusInf, Vec<T>::kMinusInf);
            }
#pragma unroll
            for (int u = 0; u < kTopTile; ++u) top[u] = Vec<T>::max_nan(raw[u]);
            if (t == 0u) {
                if (guess <= there) cut = first_bar<T>(s, step, guess, mine, top);
                else __syncthreads();
                bar = bar_value<T>(cut);
                if (warp == 0u && q.head) { if (lane == 0) s.list[0][listed] = kTopHead; ++listed; }
                if (warp == 0u && q.tail) { if (lane == 0) s.list[0][listed] = kTopTail; ++listed; }
            }
#pragma unroll
            for (int u = 0; u < kTopTile; ++u) {
                const bool hit = (uint32_t)u < mine && !(top[u] < bar);
                const unsigned hits = __ballot_sync(kFullMask, hit);
                if (hits) {
                    if (hit) {
                        s.list[warp][listed + __popc(hits & ((1u << lane) - 1u))] = (uint16_t)(128u * t + 32u * u + lane);
                        raw[u] = make_uint4(Vec<T>::kMinusInf, Vec<T>::kMinusInf, Vec<T>::kMinusInf, Vec<T>::kMinusInf);      // (summed later)
                        top[u] = -INFINITY;
                    }
                    listed += __popc(hits);
                }
            }
            if (sums) {
                es.raise(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), a.c, a.slack);
#pragma unroll
                for (int u = 0; u < kTopTile; ++u) {
                    float x[N];
                    Vec<T>::unpack(raw[u], x);
                    es.add(x, a.c);
                }
            }
            if (listed > kTopList - 32u * kTopTile && t + 1u < q.tiles) {      // no room for another tile's: the careful way
                if (lane == 0) atomicAdd(&s.cands, TopShared<MOST>::kRoom + 1u);
                listed = 0u;
            }
        }
        ExpSum e = collect<T>(s, z, listed, cut, begin, end, es.whole(a.c), a.c, a.slack);
        // (all have read the last answer; where one's wait for it has run out, it comes too late for all)
        if (__syncthreads_or(next_row == kNoAnswer)) next_row = kNoAnswer;
        if (tid == 0 && next_row >= 0) claim_ask(s.claim);
        uint32_t n = s.cands;
        const bool careful = n > TopShared<MOST>::kRoom || (n < k && cut);
        if (careful) {
            __syncthreads();
            cut = collect_carefully<T>(s, step, z, k, begin, end);
            n = s.cands;
        }
        const ExpSum dropped = sort_candidates<T>(s, step, n, k, cut, a.c, a.slack);
        const uint32_t have = min(n, k);
        // (of all that this block has seen, the first is the largest)
        const float m = have ? fmaxf(value_of_rank<T>((uint32_t)(s.cand[0] >> 32)), kLowest) : kLowest;
        if (sums) {
            if (careful || may_miss_far(m, a.c)) e = sum_carefully<T>(z, have == k ? s.cand[k - 1u] : 0ull, begin, end, a.c, a.slack);
            else e.join(dropped.m, dropped.s, a.c);
        }

        // ---- the pairs: a candidate's place is how many of the whole row's are larger -----------------
        uint32_t* places = reinterpret_cast<uint32_t*>(s.list);
        if (blocks > 1u) {
            if (tid == 0) s.count = have;
            for (uint32_t i = tid; i < have; i += kTopThreads) places[i] = i;
            cluster.sync();
            for (uint32_t j = tid; j < have * (blocks - 1u); j += kTopThreads) {
                const uint32_t i = j / (blocks - 1u), b = j % (blocks - 1u);
                const TopShared<MOST>& o = *cluster.map_shared_rank(&s, b + (b >= rank));
                const unsigned long long w = s.cand[i];
                uint32_t l = 0u, h = o.count;
                while (l < h) { const uint32_t mid = (l + h) >> 1; if (o.cand[mid] > w) l = mid + 1u; else h = mid; }
                atomicAdd(&places[i], l);
            }
            __syncthreads();
        }
        float in = 0.f;
        for (uint32_t i = tid; i < have; i += kTopThreads) {
            const unsigned long long w = s.cand[i];
            const uint32_t place = blocks > 1u ? places[i] : i;
            const float x = value_of_rank<T>((uint32_t)(w >> 32));
            if (place < k) {
                a.keys[row * k + place] = (int32_t)~(uint32_t)w;
                static_cast<T*>(a.values)[row * k + place] = from_float<T>(x);
                in += exp2_fast((x - m) * a.c);
            } else e.add(x, a.c, a.slack);
        }
        if (sums) {
            float rest = warp_sum(e.s * exp2_fast((e.m - m) * a.c));
            in = warp_sum(in);
            if (lane == 0) s.join[warp] = make_float2(rest, in);
            __syncthreads();
            if (warp == 0u) {
                const float2 p = lane < (uint32_t)kTopWarps ? s.join[lane] : make_float2(0.f, 0.f);
                rest = warp_sum(p.x); in = warp_sum(p.y);
                if (lane == 0) cluster.map_shared_rank(&s, 0)->cluster[rank] = make_float4(m, rest, in, 0.f);
            }
        }
        if (blocks > 1u) cluster.sync(); else __syncthreads();
        if (sums && rank == 0u && tid == 0) {
            float top = kLowest, rest = 0.f, inside = 0.f;
            for (uint32_t b = 0; b < blocks; ++b) top = fmaxf(top, s.cluster[b].x);
            for (uint32_t b = 0; b < blocks; ++b) {
                const float f = exp2_fast((s.cluster[b].x - top) * a.c);
                rest += s.cluster[b].y * f; inside += s.cluster[b].z * f;
            }
            const bool none = rest + inside == 0.f;        // every logit is -inf
            if (a.lse) a.lse[row] = none ? -INFINITY : top / a.temperature + logf(rest + inside);
            if (a.tail) a.tail[row] = none ? 0.f : rest / (rest + inside);
        }
        if (next_row == kNoAnswer) {                       // a row that this block was granted has no pairs
            wait_copies<0>();
            const int lost = claim_answer(s.claim, turn);
            if (lost >= 0) give_up_pairs(a.keys + (uint64_t)lost * k, static_cast<T*>(a.values) + (uint64_t)lost * k, k, a.lse ? a.lse + lost : nullptr, a.tail ? a.tail + lost : nullptr);
        }
        if (next_row < 0) break;
        row = (uint64_t)next_row;
    }
}

}  // namespace fsg
