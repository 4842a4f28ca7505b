// Distillation from a teacher's top logits: loss and gradient of a row of student logits z against the teacher's pairs
// (key_i, t_i), i < k, and the share `tail` of the teacher's probability outside of them.  With q = softmax(z / T),
//   p_i  = (1 - tail) softmax(t / T)_i over the pairs whose key lies in [0, V),      rest = sum of q_j over j that are no key,
//   loss = w T^2 ( sum_i p_i (log p_i - log q_key_i) + tail (log tail - log rest) ),
//   d loss / d z_j = w T ( q_j - sum of p_i with key_i = j )       for a key j,
//                  = w T q_j (1 - tail / rest)                     for the others.
// With a tail, the sum of exponentials runs over the others alone: rest then has no cancellation (1 - sum of the keys' q would
// lose it where the student is sure), and the gradient of the others is their share of that sum times w T (rest - tail).
#pragma once

#include <cooperative_groups.h>

#include "async.cuh"
#include "rows.cuh"

namespace fsg {

constexpr int kDistillThreads = 256;                       // that go through the row
constexpr int kDistillWarps   = kDistillThreads / 32;
constexpr int kDistillBlock   = kDistillThreads + 32;      // and a warp for the pairs
constexpr uint32_t kDistillMaxPairs = 1024u;
constexpr uint32_t kDistillMaxCols  = 1u << 20;
constexpr uint32_t kDistillMaxBlocks = 8u;                 // of a cluster

// what a launch computes
constexpr int kLossOnly = 0, kLossAndGrad = 1, kGradOnly = 2;      // kGradOnly: from the sums that a forward launch kept

struct DistillArgs {
    const void* z; void* grad;
    const int32_t* keys; const void* values; const float* tail;
    const float* weight; const float* grad_loss; const float* stats_in;
    float* loss; float* stats_out;
    uint64_t rows, z_stride, grad_stride;
    uint32_t cols, k, values_type;
    uint32_t per, slots, kept;                             // vectors of a row that a block takes; of them a thread; in shared memory
    uint32_t claims;                                       // there are more rows than blocks or clusters at a time
    uint32_t tries;                                        // of every wait
    float temperature, inv_t, c, slack;                    // c = log2(e) / T
};

// What the pairs' warp finds out about a row ...
struct DistillRow {
    float zm, tsum, cross, ksum;                           // largest of the keys' logits; sums over the pairs, relative to the largest of their kind
    float tail, scale, weight;                             // scale: of the gradient
    float m, s;                                            // kGradOnly: what the forward launch kept
    uint32_t flags, row;
    // where the block's share of this row and of the next one is: its first vector, how many
    const uint4* at; const uint4* next_at;
    uint32_t count, next_count, head, tail_count;
};
constexpr uint32_t kRowCounts = 1u, kRowRepeats = 2u, kRowNone = 4u;      // there is a pair with a probability; a key of this block appears again; there are no more rows
// ... and the others: the sum of exponentials, and that of the keys of all blocks.
struct DistillSums { float m, s, ksum; };

struct DistillShared {
    DistillRow  row[2];                                    // for even and odd rows, as everything below that two rows are at work on
    DistillSums sums[2];
    float2 join[2][kDistillWarps];
    float4 peer[2][kDistillMaxBlocks];                     // m, sum and keys' sum of every block of the cluster
    unsigned long long ready[2], done[2], met[2];          // the row's pairs are known; its gradient is written; every block's sums are there
    unsigned long long level;                              // the warps that go through the row have all come so far
    Claim  claim;                                          // of the first block: the cluster's next row
    int    next[2];                                        // the others': what the first has been given
    unsigned long long told[2];                            // (one would not do: the first block may be a turn ahead of another's pairs' warp)
};
// dynamic: uint4 ring[kept][threads], then for each of two rows key, t (later e), z of every pair, then for each of two rows a byte per
// vector of the slice, one for the elements before and one for those behind the vectors: which of the elements are keys of the row
// (a thread's vectors i = 4 n .. 4 n + 3 in one word: vector i of thread t has byte (i / 4) 4 threads + 4 t + i % 4)
__host__ __device__ inline uint32_t distill_map_vectors(uint32_t per) { return (per + 4u * kDistillThreads - 1u) / (4u * kDistillThreads) * (4u * kDistillThreads); }
__host__ __device__ inline uint32_t distill_map_bytes(uint32_t per) { return distill_map_vectors(per) + 4u; }
__device__ __forceinline__ uint32_t map_byte(uint32_t v) {
    const uint32_t i = v / kDistillThreads, t = v % kDistillThreads;
    return i / 4u * (4u * kDistillThreads) + 4u * t + i % 4u;
}
__host__ __device__ inline size_t distill_smem(uint32_t kept, uint32_t k, uint32_t per) {
    kept = (kept + 3u) & ~3u;                              // (four chunks)
    return (size_t)kept * kDistillThreads * 16u + 24u * (size_t)k + 2u * distill_map_bytes(per);
}

// The warps that go through the row wait for one another, for the n-th time; false where that has run out.  (Not bar.sync, which waits
// without a limit for a warp whose own wait has run out.)
__device__ __forceinline__ bool readers_level(DistillShared& s, uint32_t& n, uint32_t tries) {
    __syncwarp();
    if ((threadIdx.x & 31u) == 0u) mbar_arrive(&s.level);
    return __all_sync(kFullMask, mbar_wait(&s.level, n++ & 1u, tries));
}
__device__ __forceinline__ void cluster_arrive() { __syncwarp(); asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { __syncwarp(); asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// A block's share of a row: vectors [first, first + count) behind the row's head; the first block has the head, too, the last one the tail.
struct DistillSlice {
    uint32_t head, tail, vecs, first, count;
};
template <class T> __device__ __forceinline__ DistillSlice distill_slice(const T* z, uint32_t cols, uint32_t per, uint32_t rank) {
    const Span sp = span_of(z, cols);
    DistillSlice q;
    q.head = sp.head; q.tail = sp.tail; q.vecs = sp.vecs;
    q.first = min(rank * per, sp.vecs);
    q.count = min(per, sp.vecs - q.first);
    return q;
}

// The sum of exponentials of a block's share, without the keys of `map` where there is one: from global memory and with any
// logits; thread tid's part of `threads`.
template <class T>
__device__ __noinline__ ExpSum scan_far(const T* z, const uint8_t* map, uint32_t cols, uint32_t per, uint32_t rank, uint32_t blocks, float c, float slack, uint32_t tid, uint32_t threads) {
    constexpr int N = Vec<T>::N;
    const DistillSlice q = distill_slice(z, cols, per, rank);
    ExpSum e;
    for (uint32_t i = tid; i < q.count; i += threads) {
        float x[N];
        Vec<T>::unpack(load16(z + q.head + (uint64_t)(q.first + i) * N), x);
        const uint32_t keys = map ? map[map_byte(i)] : 0u;
#pragma unroll
        for (int j = 0; j < N; ++j) if (!(keys >> j & 1u)) e.add(x[j], c, slack);
    }
    if (rank == 0u && tid < q.head && !(map && map[distill_map_vectors(per)] >> tid & 1u)) e.add(to_float(z[tid]), c, slack);
    if (rank == blocks - 1u && tid < q.tail && !(map && map[distill_map_vectors(per) + 1u] >> tid & 1u)) e.add(to_float(z[cols - q.tail + tid]), c, slack);
    return e;
}

// The warps' sums in one, the same in every lane.
__device__ __forceinline__ ExpSum join_warps(const float2* join, float c) {
    const float2 p = join[(threadIdx.x & 31u) % kDistillWarps];
    ExpSum e;
    e.m = warp_max(p.x);
    e.s = p.y * exp2_fast((p.x - e.m) * c);
#pragma unroll
    for (int o = kDistillWarps / 2; o; o >>= 1) e.s += __shfl_xor_sync(kFullMask, e.s, o);
    return e;
}

// grad = by 2^((z - m) c) of a block's share, from global memory and with any logits (by = 0: zero).
template <class TZ, class TG>
__device__ __noinline__ void write_far(const TZ* z, TG* g, uint32_t cols, uint32_t per, uint32_t rank, uint32_t blocks, float by, float m, float c) {
    constexpr int N = Vec<TZ>::N;
    const DistillSlice q = distill_slice(z, cols, per, rank);
    const bool wide = (reinterpret_cast<uintptr_t>(g + q.head) & 15u) == 0u;
    for (uint32_t i = threadIdx.x; i < q.count; i += kDistillThreads) {
        const uint64_t j = q.head + (uint64_t)(q.first + i) * N;
        float x[N];
        if (by != 0.f) Vec<TZ>::unpack(load16(z + j), x);
#pragma unroll
        for (int n = 0; n < N; ++n) x[n] = by != 0.f ? exp2_fast((x[n] - m) * c) * by : 0.f;
        store_values(g + j, x, wide);
    }
    auto single = [&](uint32_t j) { g[j] = from_float<TG>(by != 0.f ? exp2_fast((to_float(z[j]) - m) * c) * by : 0.f); };
    if (rank == 0u && threadIdx.x < q.head) single(threadIdx.x);
    if (rank == blocks - 1u && threadIdx.x < q.tail) single(cols - q.tail + threadIdx.x);
}

// The place of key j in the map of a block's share, in bits, or -1 if another block has it.
template <class T>
__device__ __forceinline__ int key_bit(const DistillSlice& q, uint32_t j, uint32_t per, uint32_t rank, uint32_t blocks) {
    constexpr uint32_t N = Vec<T>::N;
    const uint32_t edges = distill_map_vectors(per);
    if (j < q.head) return rank == 0u ? (int)(edges * 8u + j) : -1;
    const uint32_t v = (j - q.head) / N;
    if (v >= q.vecs) return rank == blocks - 1u ? (int)((edges + 1u) * 8u + j - q.head - q.vecs * N) : -1;
    return v - q.first < q.count ? (int)(map_byte(v - q.first) * 8u + (j - q.head) % N) : -1;
}

// The pairs' warp: what it finds out about a row, one row ahead of the others.
template <class TZ, int MODE>
__device__ __forceinline__ void prepare_pairs(const DistillArgs& a, uint64_t row, uint32_t rank, uint32_t blocks, DistillRow& out, int* s_key, float* s_t, float* s_z, uint8_t* map) {
    constexpr uint32_t U = 4u;
    const uint32_t lane = threadIdx.x & 31u, k = a.k;
    const bool mapped = MODE != kLossOnly || a.tail;
    const TZ* z = static_cast<const TZ*>(a.z) + row * a.z_stride;
    const DistillSlice q = distill_slice(z, a.cols, a.per, rank);
    DistillRow r;
    r.weight = a.weight ? a.weight[row] : 1.f;
    r.tail = a.tail ? a.tail[row] : 0.f;
    r.scale = a.temperature * (MODE != kLossOnly && a.grad_loss ? a.grad_loss[row] : 1.f);
    r.m = MODE == kGradOnly ? a.stats_in[2 * row] : 0.f;
    r.s = MODE == kGradOnly ? a.stats_in[2 * row + 1] : 0.f;
    float tm = -INFINITY, zm = kLowest;
    bool again = false, no_number = false;
    if (r.weight != 0.f) {
        for (uint32_t i0 = lane; i0 < k; i0 += 32u * U) {
            int key[U];
            float t[U], zk[U];
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                const uint32_t i = i0 + 32u * u;
                key[u] = -1; t[u] = -INFINITY;
                if (i < k) { key[u] = a.keys[row * k + i]; t[u] = load_typed(a.values, row * k + i, a.values_type); }
            }
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                if (key[u] < 0 || (uint32_t)key[u] >= a.cols) { key[u] = -1; t[u] = -INFINITY; }
                zk[u] = key[u] >= 0 ? to_float(z[key[u]]) : -INFINITY;
            }
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                const uint32_t i = i0 + 32u * u;
                if (i >= k) continue;
                s_key[i] = key[u]; s_t[i] = t[u]; s_z[i] = zk[u];
                tm = fmaxf(tm, t[u]); zm = fmaxf(zm, zk[u]); no_number |= t[u] != t[u];
                if (mapped && key[u] >= 0) {
                    const int b = key_bit<TZ>(q, (uint32_t)key[u], a.per, rank, blocks);
                    if (b >= 0) again |= atomicOr(reinterpret_cast<uint32_t*>(map) + (b >> 5), 1u << (b & 31)) >> (b & 31) & 1u;
                }
            }
        }
    }
    tm = warp_max(tm); zm = warp_max(zm);
    again = __any_sync(kFullMask, again);
    // weight 0, or no pair with any probability: the row counts for nothing (the largest does not show a NaN, which makes the row's sums NaN)
    const bool counts = tm > -INFINITY || __any_sync(kFullMask, no_number);
    __syncwarp();
    float tsum = 0.f, cross = 0.f, ksum = 0.f;
    if (counts) {
        for (uint32_t i = lane; i < k; i += 32u) {
            const float d = s_t[i] - tm, e = exp2_fast(d * a.c), y = s_z[i] - zm;
            tsum += e;
            if (e != 0.f) cross += e * (d - y);
            s_t[i] = e;
            // a key that appears several times counts once for the student
            bool first = mapped && s_key[i] >= 0 && key_bit<TZ>(q, (uint32_t)s_key[i], a.per, rank, blocks) >= 0;
            if (again) for (uint32_t j = 0; j < i; ++j) first &= s_key[j] != s_key[i];
            if (first) ksum += exp2_fast(y * a.c);
        }
    }
    r.tsum = warp_sum(tsum); r.cross = warp_sum(cross); r.ksum = warp_sum(ksum); r.zm = zm;
    r.scale *= r.weight;
    r.flags = (counts ? kRowCounts : 0u) | (again ? kRowRepeats : 0u);
    r.at = reinterpret_cast<const uint4*>(z + q.head) + q.first; r.count = q.count; r.head = q.head; r.tail_count = q.tail;
    r.row = (uint32_t)row; r.next_at = nullptr; r.next_count = 0u;
    if (lane == 0) out = r;
}

// What both kinds of warps conclude from the sums.
struct DistillTotals { float top, rest, total; bool none; };
__device__ __forceinline__ DistillTotals totals_of(const DistillRow& r, const DistillSums& e, float c) {
    DistillTotals t;
    const bool tailed = r.tail != 0.f;
    t.top = tailed ? fmaxf(e.m, r.zm) : e.m;
    t.rest = e.s * exp2_fast((e.m - t.top) * c);
    t.total = tailed ? t.rest + e.ksum * exp2_fast((r.zm - t.top) * c) : e.s;
    t.none = !(r.flags & kRowCounts) || t.total == 0.f;    // (every logit of the row is -inf: it counts for nothing, too)
    return t;
}

// The pairs' warp: the loss, and the gradient of the keys, once the others have written theirs; the row's part of the map is clear again.
template <class TZ, class TG, int MODE>
__device__ __forceinline__ void finish_pairs(const DistillArgs& a, uint64_t row, uint32_t rank, uint32_t blocks, const DistillRow& r, const DistillSums& e,
                                             const int* s_key, const float* s_t, const float* s_z, uint8_t* map) {
    const uint32_t lane = threadIdx.x & 31u, k = a.k;
    const TZ* z = static_cast<const TZ*>(a.z) + row * a.z_stride;
    const DistillSlice q = distill_slice(z, a.cols, a.per, rank);
    const DistillTotals t = totals_of(r, e, a.c);
    if (MODE != kGradOnly && rank == 0u && lane == 0) {
        float loss = 0.f;
        if (!t.none) {
            // sum p_i (log p_i - log q_i): both logarithms relative to the largest of their kind
            const float log_total = logf(t.total), share = 1.f - r.tail;
            if (share != 0.f || r.tsum != r.tsum) loss = share * (r.cross / r.tsum * a.inv_t + logf(share / r.tsum) + ((t.top - r.zm) * a.inv_t + log_total));
            if (r.tail != 0.f) loss += r.tail * (logf(r.tail / e.s) - (e.m - t.top) * a.inv_t + log_total);
            loss *= r.weight * a.temperature * a.temperature;
        }
        if (a.loss) a.loss[row] = loss;
        if (a.stats_out) { a.stats_out[2 * row] = t.none ? 0.f : e.m; a.stats_out[2 * row + 1] = t.none ? 0.f : e.s; }
    }
    if (!(MODE != kLossOnly || a.tail) || r.weight == 0.f) return;
    const float share = (1.f - r.tail) / r.tsum;
    TG* g = MODE == kLossOnly ? nullptr : static_cast<TG*>(a.grad) + row * a.grad_stride;
    for (uint32_t i = lane; i < k; i += 32u) {
        const int key = s_key[i];
        const int b = key >= 0 ? key_bit<TZ>(q, (uint32_t)key, a.per, rank, blocks) : -1;
        if (b < 0) continue;
        map[b >> 3] = 0u;
        if (MODE == kLossOnly || t.none) continue;
        // all probability of a key that appears several times goes to its first pair
        float p = s_t[i];
        bool first = true;
        if (r.flags & kRowRepeats) {
            p = 0.f;
            for (uint32_t j = 0; j < k; ++j) if (s_key[j] == key) { p += s_t[j]; first &= j >= i; }
        }
        if (first) g[key] = from_float<TG>(r.scale * (exp2_fast((s_z[i] - t.top) * a.c) / t.total - p * share));
    }
}

// A row that has been given up: nothing of it is a number.  One warp.
template <class TG>
__device__ __noinline__ void give_up_row(TG* g, uint32_t cols, float* loss, float* stats) {
    const uint32_t lane = threadIdx.x & 31u;
    if (g) for (uint32_t j = lane; j < cols; j += 32u) g[j] = from_float<TG>(NAN);
    if (lane == 0 && loss) *loss = NAN;
    if (lane < 2u && stats) stats[lane] = NAN;
}

// A block or a cluster of blocks per row.  A block's share of the row stays in shared memory between the two passes, each thread's
// vectors in places of its own: the thread that has used a vector for the last time asks for the next row's vector in its place, so that
// reads go on while gradients are written, and no barrier stands between a copy and its use.  (Vectors beyond the shared memory, of
// rows above half a megabyte, are read twice.)  The ninth warp has the pairs: those of the next row while the others go through this
// one, and the keys' gradients of the row before.
// 4096 x 128000 bf16 with a bf16 gradient: 432 to 492 us by the GPU, 4.3 to 4.9 TB/s (2.1 GB; a copy's time 320).  A row in one block that
// reads it twice: 597; in the shared memory of a cluster, block-wide barriers: 488; several vectors between two looks at the largest: 467;
// mbarriers in place of the block-wide barriers: 438; in place of the readers' own as well: 461 -> 444 on one GPU.  Neither DRAM nor the instructions' issue (53 %) is full: a cluster of four waits for its
// slowest block twice a row, and what it waits with is 3 x 64 KB an SM.
// 1023 x 50257 fp32, loss alone: 47 us, 4.4 TB/s (a copy's time 31.5); one pass has 32 KB of copies ahead in place of the row: 55 -> 47.
// The backward pass of 2048 x 32000 fp16: 47.5 to 53 us by the GPU, 5.0 to 5.5 TB/s (40).
// Every wait has a limit.  What a warp may overwrite is what others have told it that they are done with, and what it reads is what it has
// been told is there: a warp whose wait runs out goes to the kernel's end, and then those that wait for it do.  There, once the whole cluster
// has come, the pairs' warp of a block that has not finished its rows, or has been granted one that it never began, makes all of them NaN.
template <class TZ, class TG, int MODE>
__global__ void __launch_bounds__(kDistillBlock, 3) k_distill(DistillArgs a) {
    extern __shared__ __align__(16) unsigned char distill_smem_bytes[];
    __shared__ DistillShared s;
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    constexpr int N = Vec<TZ>::N;
    constexpr int G = MODE != kLossAndGrad ? 2 : 4;        // groups of copies of a row
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5, k = a.k, blocks = cluster.num_blocks(), rank = cluster.block_rank();
    int* s_key = reinterpret_cast<int*>(distill_smem_bytes + (size_t)((a.kept + 3u) & ~3u) * kDistillThreads * 16u);      // two rows' each
    float* s_t = reinterpret_cast<float*>(s_key + 2u * k);
    float* s_z = s_t + 2u * k;
    uint8_t* maps = reinterpret_cast<uint8_t*>(s_z + 2u * k);
    const uint32_t map_bytes = distill_map_bytes(a.per);
    wait_for_previous_kernels();
    const uint32_t first = blockIdx.x / blocks;

    if (warp == (uint32_t)kDistillWarps) {
        for (uint32_t i = lane; i < map_bytes / 2u; i += 32u) reinterpret_cast<uint32_t*>(maps)[i] = 0u;
        if (lane == 0) {
            for (int b = 0; b < 2; ++b) { mbar_init(&s.ready[b], 1u); mbar_init(&s.done[b], kDistillWarps); mbar_init(&s.met[b], blocks); mbar_init(&s.told[b], 1u); }
            mbar_init(&s.level, kDistillWarps);
            claim_init(s.claim);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncthreads();
        if (blocks > 1u) { cluster_arrive(); cluster_wait(); }      // (every block of the cluster has begun)
        if (a.claims && rank == 0u && lane == 0) claim_ask(s.claim);
        // turn i: the i-th row's pairs; then, once its gradient is written, the row before is finished
        int row = (int)first, last = -1, next = -1, question = -1;      // (question: one without an answer when a wait ran out)
        bool lost = false;
        for (uint32_t i = 0;; ++i) {
            const uint32_t b = i & 1u, o = b ^ 1u;
            next = -1;
            if (row >= 0) {
                prepare_pairs<TZ, MODE>(a, (uint64_t)row, rank, blocks, s.row[b], s_key + b * k, s_t + b * k, s_z + b * k, maps + b * map_bytes);
                // the cluster's next row: the first block has asked for it a turn ago, and tells the others
                if (a.claims && lane == 0) {
                    if (rank == 0u) {
                        next = claim_answer(s.claim, i, a.tries);
                        if (next >= 0) { next /= (int)blocks; claim_ask(s.claim); }
                        // (it is here once row i - 2's gradient is written, to which every block has contributed after it had read
                        // what it was told then: that place and its barrier are free)
                        if (next != kNoAnswer) for (uint32_t to = 1u; to < blocks; ++to) { *cluster.map_shared_rank(&s.next[b], to) = next; mbar_arrive_at(&s.told[b], to); }
                    } else next = mbar_wait_cluster(&s.told[b], i >> 1 & 1u, a.tries) ? s.next[b] : kNoAnswer;
                }
                next = __shfl_sync(kFullMask, next, 0);
                if (next == kNoAnswer) { lost = true; question = (int)i; break; }
                if (next >= 0 && lane == 0) {
                    const TZ* z = static_cast<const TZ*>(a.z) + (uint64_t)next * a.z_stride;
                    const DistillSlice n = distill_slice(z, a.cols, a.per, rank);
                    s.row[b].next_at = reinterpret_cast<const uint4*>(z + n.head) + n.first; s.row[b].next_count = n.count;
                }
            } else if (lane == 0) s.row[b].flags = kRowNone;
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.ready[b]);
            if (last >= 0) {
                if (!__all_sync(kFullMask, mbar_wait(&s.done[o], ((i - 1u) >> 1) & 1u, a.tries))) {
                    lost = true;
                    if (next >= 0) question = (int)i + 1;
                    break;
                }
                if (MODE == kLossOnly && blocks == 1u) {
                    const TZ* z = static_cast<const TZ*>(a.z) + (uint64_t)last * a.z_stride;
                    ExpSum e = join_warps(s.join[o], a.c);
                    if ((s.row[o].flags & kRowCounts) && (e.s == 0.f || may_miss_far(e.m, a.c)))
                        e = warp_join(scan_far(z, s.row[o].tail != 0.f ? maps + o * map_bytes : nullptr, a.cols, a.per, rank, blocks, a.c, a.slack, lane, 32u), a.c);
                    if (lane == 0) s.sums[o] = DistillSums{e.m, e.s, s.row[o].ksum};
                    __syncwarp();
                }
                finish_pairs<TZ, TG, MODE>(a, (uint64_t)last, rank, blocks, s.row[o], s.sums[o], s_key + o * k, s_t + o * k, s_z + o * k, maps + o * map_bytes);
                __syncwarp();
            }
            if (row < 0) break;
            last = row; row = next;
        }
        cluster_arrive(); cluster_wait();                  // (no block leaves while another may write to its shared memory)
        if (lost) {
            int granted = -1;
            if (rank == 0u && lane == 0 && a.claims && question >= 0) granted = claim_answer(s.claim, (uint32_t)question);
            granted = __shfl_sync(kFullMask, granted, 0);
            for (int n = 0; n < 4; ++n) {
                const int r = n == 0 ? last : n == 1 ? row : n == 2 ? next : granted < 0 ? -1 : granted / (int)blocks;
                if (r >= 0) give_up_row(MODE == kLossOnly ? nullptr : static_cast<TG*>(a.grad) + (uint64_t)r * a.grad_stride, a.cols, a.loss ? a.loss + r : nullptr, a.stats_out ? a.stats_out + 2 * (uint64_t)r : nullptr);
            }
        }
        return;
    }

    uint4* ring = reinterpret_cast<uint4*>(distill_smem_bytes) + tid;
    // One pass (the loss or the gradient alone): a row in chunks of `group` vectors a thread, two chunks ahead, whatever the row's length.  Two
    // passes: four chunks that stay, and the rest of the row without.
    constexpr bool kOnePass = MODE != kLossAndGrad;
    constexpr uint32_t U = 4u;                             // vectors between two looks at keys and largest
    const uint32_t group = ((a.kept + G - 1u) / G + U - 1u) / U * U, chunks = kOnePass ? max((a.slots + group - 1u) / group, (uint32_t)G) : (uint32_t)G;
    auto mine_of = [&](uint32_t count) { return (count + kDistillThreads - 1u - tid) / kDistillThreads; };      // (this thread's of so many vectors)
    // chunk n of a row to the chunk's place `to` in the shared memory
    auto fetch = [&](const uint4* at, uint32_t mine, uint32_t n, uint32_t to) {
        const uint32_t from = n * group, end = min(min(from + group, kOnePass ? a.slots : a.kept), mine);
        at += tid;
        uint4* place = ring + to * group * kDistillThreads;
#pragma unroll 4
        for (uint32_t i = from; i < end; ++i, place += kDistillThreads) copy16_async(place, at + i * kDistillThreads);
        copies_end_group();
    };
    uint32_t turn = 0u;                                    // one pass: the place of the chunk at hand
    auto fetch_ahead = [&](const DistillRow& r, uint32_t mine, uint32_t next_mine, uint32_t n) {
        if (n + G < chunks) fetch(r.at, mine, n + G, turn); else fetch(r.next_at, next_mine, n + G - chunks, turn);
        turn = (turn + 1u) % G;
    };
    {
        const TZ* z = static_cast<const TZ*>(a.z) + (uint64_t)first * a.z_stride;
        const DistillSlice q = distill_slice(z, a.cols, a.per, rank);
#pragma unroll 1
        for (uint32_t n = 0; n < (uint32_t)G; ++n) fetch(reinterpret_cast<const uint4*>(z + q.head) + q.first, mine_of(q.count), n, n);
    }
    __syncthreads();
    if (blocks > 1u) { cluster_arrive(); cluster_wait(); }
    uint32_t meetings = 0u;
    for (uint32_t i = 0u;; ++i) {
        const uint32_t b = i & 1u, parity = i >> 1 & 1u;
        if (!__all_sync(kFullMask, mbar_wait(&s.ready[b], parity, a.tries))) break;
        const DistillRow& r = s.row[b];
        if (r.flags & kRowNone) break;
        const uint64_t row = r.row;
        const TZ* z = static_cast<const TZ*>(a.z) + row * a.z_stride;
        const uint32_t mine = mine_of(r.count), next_mine = mine_of(r.next_count);
        const bool counts = r.flags & kRowCounts, tailed = r.tail != 0.f;

        // ---- the sum of exponentials, of all classes or (with a tail) of those that are no key ----
        ExpSum e;
        const uint8_t* skip = tailed ? maps + b * map_bytes : nullptr;
        if (MODE != kGradOnly) {
            FusedExpSums es;
            // a vector without the elements that are keys
            auto without = [](uint4 raw, uint32_t keys) {
                if (keys) {
                    TZ* x = reinterpret_cast<TZ*>(&raw);
#pragma unroll
                    for (int j = 0; j < N; ++j) if (keys >> j & 1u) x[j] = from_float<TZ>(-INFINITY);
                }
                return raw;
            };
#pragma unroll 1
            for (uint32_t n = 0; n < chunks + (kOnePass ? 0u : 1u); ++n) {
                if (kOnePass) wait_copies<G - 1>();
                else if (n == 0u) wait_copies<3>();
                else if (n == 1u) wait_copies<2>();
                else if (n == 2u) wait_copies<1>();
                else wait_copies<0>();
                // (two passes, the last round: what does not fit into the shared memory)
                const bool rest = !kOnePass && n == chunks;
                const uint32_t from = rest ? a.kept : n * group, to = counts ? rest ? mine : min(min(from + group, kOnePass ? a.slots : a.kept), mine) : 0u;
                const uint4* place = ring + (kOnePass ? turn : n) * group * kDistillThreads;
                uint32_t i = from;
                // U vectors at a time: one look at their keys, one at their largest
                if (!rest) {
#pragma unroll 1
                    for (; i + U <= to; i += U, place += U * kDistillThreads) {
                        uint4 raw[U];
                        float top[U];
#pragma unroll
                        for (int u = 0; u < (int)U; ++u) raw[u] = place[u * kDistillThreads];
#pragma unroll
                        for (int u = 0; u < (int)U; ++u) top[u] = Vec<TZ>::max(raw[u]);
                        if (skip) {
                            const uint32_t keys = reinterpret_cast<const uint32_t*>(skip)[i / 4u * kDistillThreads + tid];      // (i is a multiple of four)
                            if (keys) {
#pragma unroll
                                for (int u = 0; u < (int)U; ++u)
                                    if (keys >> (8 * u) & 255u) { raw[u] = without(raw[u], keys >> (8 * u) & 255u); top[u] = Vec<TZ>::max(raw[u]); }
                            }
                        }
                        float most = top[0];
#pragma unroll
                        for (int u = 1; u < (int)U; ++u) most = fmaxf(most, top[u]);
                        es.raise(most, a.c, a.slack);
#pragma unroll
                        for (int u = 0; u < (int)U; ++u) {
                            float x[N];
                            Vec<TZ>::unpack(raw[u], x);
                            es.add(x, a.c);
                        }
                    }
                }
#pragma unroll 1
                for (; i < to; ++i, place += kDistillThreads) {
                    const uint4 raw = without(rest ? load16(r.at + i * kDistillThreads + tid) : *place, skip ? skip[map_byte(i * kDistillThreads + tid)] : 0u);
                    float x[N];
                    Vec<TZ>::unpack(raw, x);
                    es.raise(Vec<TZ>::max(raw), a.c, a.slack);
                    es.add(x, a.c);
                }
                if (kOnePass) fetch_ahead(r, mine, next_mine, n);
            }
            if (counts) {
                e = es.whole(a.c);
                if (rank == 0u && tid < r.head && !(skip && skip[distill_map_vectors(a.per)] >> tid & 1u)) e.add(to_float(z[tid]), a.c, a.slack);
                if (rank == blocks - 1u && tid < r.tail_count && !(skip && skip[distill_map_vectors(a.per) + 1u] >> tid & 1u)) e.add(to_float(z[a.cols - r.tail_count + tid]), a.c, a.slack);
            }
            e = warp_join(e, a.c);
            if (lane == 0) s.join[b][warp] = make_float2(e.m, e.s);
            if (MODE == kLossOnly && blocks == 1u) {       // (the pairs' warp joins them: nobody waits for anybody here)
                __syncwarp();
                if (lane == 0) mbar_arrive(&s.done[b]);
                continue;
            }
            if (!readers_level(s, meetings, a.tries)) break;
            e = join_warps(s.join[b], a.c);
            if (counts && (e.s == 0.f || may_miss_far(e.m, a.c))) {
                if (!readers_level(s, meetings, a.tries)) break;
                e = warp_join(scan_far(z, skip, a.cols, a.per, rank, blocks, a.c, a.slack, tid, kDistillThreads), a.c);
                if (lane == 0) s.join[b][warp] = make_float2(e.m, e.s);
                if (!readers_level(s, meetings, a.tries)) break;
                e = join_warps(s.join[b], a.c);
            }
        }
        DistillSums sums{e.m, e.s, r.ksum};
        if (blocks > 1u) {
            if (MODE == kGradOnly && !readers_level(s, meetings, a.tries)) break;      // (all have met for the row before: the barrier is free)
            if (tid < blocks) {
                cluster.map_shared_rank(&s, tid)->peer[b][rank] = make_float4(e.m, e.s, r.ksum, 0.f);
                mbar_arrive_at(&s.met[b], tid);
            }
            if (!__all_sync(kFullMask, mbar_wait_cluster(&s.met[b], parity, a.tries))) break;
            // (eight places, of which the cluster has one, two, four or all)
            const float4 p = s.peer[b][lane % blocks];
            sums.m = warp_max(p.x);
            sums.s = p.y * exp2_fast((p.x - sums.m) * a.c);
            sums.ksum = p.z;
            for (uint32_t o = blocks / 2u; o; o >>= 1) {
                sums.s += __shfl_xor_sync(kFullMask, sums.s, o);
                sums.ksum += __shfl_xor_sync(kFullMask, sums.ksum, o);
            }
        }
        if (MODE == kGradOnly) { sums.m = r.m; sums.s = r.s; }
        if (tid == 0) s.sums[b] = sums;

        // ---- the gradient of the classes that are no key (the pairs' warp overwrites the keys') -----------
        if (MODE != kLossOnly) {
            const DistillTotals t = totals_of(r, sums, a.c);
            TG* g = static_cast<TG*>(a.grad) + row * a.grad_stride;
            const float ref = sums.m * a.c;
            float by = t.none || sums.s == 0.f ? 0.f : r.scale * (tailed ? t.rest / t.total - r.tail : 1.f) / sums.s;
            const bool near = by != 0.f && !is_far(sums.m, a.c);
            if (!near) write_far(z, g, a.cols, a.per, rank, blocks, by, sums.m, a.c);
            by *= exp2_fast(-__fmaf_rn(sums.m, a.c, -ref));
            const unsigned long long cc = pair_of(a.c, a.c), bb = pair_of(by, by), minus_r = pair_of(-ref, -ref);
            const bool wide = (reinterpret_cast<uintptr_t>(g + r.head) & 15u) == 0u;
            TG* out = g + (reinterpret_cast<const TZ*>(r.at + tid) - z);
            auto put = [&](const uint4& raw, uint32_t i) {
                float x[N];
                Vec<TZ>::unpack(raw, x);
#pragma unroll
                for (int j = 0; j < N; j += 2) {
                    float2 y = halves(fma_pairs(pair_of(x[j], x[j + 1]), cc, minus_r));
                    y = halves(mul_pairs(pair_of(exp2_fast(y.x), exp2_fast(y.y)), bb));
                    x[j] = y.x; x[j + 1] = y.y;
                }
                store_values(out + (uint64_t)(i * kDistillThreads) * N, x, wide);
            };
            if (near) {
                auto put_one = [&](uint32_t j) { g[j] = from_float<TG>(exp2_fast(__fmaf_rn(to_float(z[j]), a.c, -ref)) * by); };
                if (rank == 0u && tid < r.head) put_one(tid);
                if (rank == blocks - 1u && tid < r.tail_count) put_one(a.cols - r.tail_count + tid);
            }
#pragma unroll 1
            for (uint32_t n = 0; n < chunks + (kOnePass ? 0u : 1u); ++n) {
                if (kOnePass) wait_copies<G - 1>();
                const bool rest = !kOnePass && n == chunks;
                const uint32_t from = rest ? a.kept : n * group, to = near ? rest ? mine : min(min(from + group, kOnePass ? a.slots : a.kept), mine) : 0u;
                const uint4* place = ring + (kOnePass ? turn : n) * group * kDistillThreads;
                uint32_t i = from;
                if (!rest) {
#pragma unroll 1
                    for (; i + U <= to; i += U, place += U * kDistillThreads) {
                        uint4 raw[U];
#pragma unroll
                        for (int u = 0; u < (int)U; ++u) raw[u] = place[u * kDistillThreads];
#pragma unroll
                        for (int u = 0; u < (int)U; ++u) put(raw[u], i + u);
                    }
                }
#pragma unroll 1
                for (; i < to; ++i, place += kDistillThreads) put(rest ? load16(r.at + i * kDistillThreads + tid) : *place, i);
                if (kOnePass) fetch_ahead(r, mine, next_mine, n);
                else if (!rest) fetch(r.next_at, next_mine, n, n);
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.done[b]);
    }
    wait_copies<0>();
    cluster_arrive(); cluster_wait();
}

}  // namespace fsg
