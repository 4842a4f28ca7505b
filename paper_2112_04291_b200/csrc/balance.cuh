// Per-expert counts of the experts that a router selected, and the balance loss with its gradient.  Per segment s of tokens
// (x: the router's logits, p = softmax(x), E experts, n_s tokens that count):
//   f_e = counts_se / sum_e counts_se,      L_s = coef E sum_e f_e (1/n_s) sum_t p_te,
//   dL_s / dx_te = (coef E / n_s) p_te (f_e - sum_e' f_e' p_te').
// The gradient depends on the counts alone and not on the mean of p: with the counts known first, one pass over x gives the
// gradient and, as the sum over the tokens of sum_e f_e p_te, the loss.
#pragma once

#include <cooperative_groups.h>

#include "rows.cuh"

namespace fsg {

constexpr int kBalanceThreads = 256;
constexpr int kBalanceWarps   = kBalanceThreads / 32;
constexpr int kCountThreads   = 512;
constexpr uint32_t kBalanceMaxExperts = 1024u;
constexpr uint32_t kBalanceMaxBlocks  = 2048u;

struct CountArgs {
    const int32_t* selected; const uint8_t* mask; const uint64_t* offsets;
    uint32_t* counts; uint32_t* counted;
    uint64_t tokens; uint32_t k, experts, segments, rows_per_block;
};

struct BalanceArgs {
    const void* x; void* grad; const uint8_t* mask; const uint64_t* offsets;
    const uint32_t* counts; const uint32_t* counted; const float* grad_loss;
    float* loss; double* partials; unsigned int* done;
    uint64_t tokens, x_stride, grad_stride; uint32_t experts, segments, rows_per_block;
    float coef;
};

// The segments of tokens: [offsets[s], offsets[s + 1]), within [0, tokens); one of all tokens without offsets.
struct Segments {
    const uint64_t* offsets; uint64_t tokens; uint32_t count;
    __device__ __forceinline__ uint64_t edge(uint32_t s) const {
        const uint64_t v = offsets ? offsets[s] : (s ? tokens : 0ull);
        return v < tokens ? v : tokens;
    }
    // The first segment that ends behind token t.  A warp looks at 32 ends at a time (a search of two ends a step waits for memory
    // three times as often).
    __device__ __forceinline__ uint32_t find(uint64_t t) const {
        if (!offsets) return 0u;
        const uint32_t lane = threadIdx.x & 31u;
        uint32_t lo = 0u, hi = count;                      // it is among [lo, hi]
        while (lo < hi) {
            const uint32_t step = (hi - lo + 31u) / 32u, at = lo + step * lane;      // ends lo, lo + step, ...
            const unsigned behind = __ballot_sync(kFullMask, at < hi && edge(at + 1u) > t);
            const uint32_t first = behind ? (uint32_t)__ffs((int)behind) - 1u : 32u;
            const uint32_t end = lo + step * first;        // the first of them behind t, or none
            if (!first) return lo;
            const uint32_t past = (hi - lo - 1u) / step;   // the last that was looked at
            hi = behind ? end : hi;
            lo = (behind ? end - step : lo + step * past) + 1u;
        }
        return lo;
    }
};

// The selections of `n` tokens into a histogram in shared memory.
__device__ __forceinline__ void count_tokens(const CountArgs& a, uint64_t from, uint32_t n, uint32_t* hist, uint32_t* tokens_in) {
    const uint32_t tid = threadIdx.x;
    if (a.mask) {
        uint32_t mine = 0u;
        for (uint32_t t = tid; t < n; t += kCountThreads) mine += a.mask[from + t] != 0;
        mine = __reduce_add_sync(kFullMask, mine);
        if ((tid & 31u) == 0u && mine) atomicAdd(tokens_in, mine);
    } else if (tid == 0) *tokens_in = n;
    const int32_t* sel = a.selected + from * a.k;
    const uint32_t all = n * a.k;
    auto put = [&](int e, uint32_t i) {
        if (e >= 0 && (uint32_t)e < a.experts && (!a.mask || a.mask[from + i / a.k])) atomicAdd(&hist[e], 1u);
    };
    constexpr uint32_t U = 4u;
    for (uint32_t i = tid; i < all; i += U * kCountThreads) {
        int e[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) e[u] = i + u * kCountThreads < all ? sel[i + u * kCountThreads] : -1;
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) put(e[u], i + u * kCountThreads);
    }
}

// A cluster of blocks per segment: a histogram each, added up over the cluster's shared memory.  Writes every count, so that nothing is
// cleared before.
__global__ void __launch_bounds__(kCountThreads) k_expert_counts(CountArgs a) {
    namespace cg = cooperative_groups;
    __shared__ uint32_t hist[kBalanceMaxExperts], tokens_in;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t tid = threadIdx.x, blocks = cluster.num_blocks(), rank = cluster.block_rank();
    wait_for_previous_kernels();
    const Segments seg{a.offsets, a.tokens, a.segments};
    for (uint32_t s = blockIdx.x / blocks; s < a.segments; s += gridDim.x / blocks) {
        const uint64_t from = seg.edge(s), to = seg.edge(s + 1u);
        const uint64_t n = from < to ? to - from : 0ull, b = from + n * rank / blocks, e = from + n * (rank + 1u) / blocks;
        for (uint32_t i = tid; i < a.experts; i += kCountThreads) hist[i] = 0u;
        if (tid == 0) tokens_in = 0u;
        __syncthreads();
        count_tokens(a, b, (uint32_t)(e - b), hist, &tokens_in);
        cluster.sync();
        for (uint32_t i = rank * kCountThreads + tid; i < a.experts; i += blocks * kCountThreads) {
            uint32_t sum = 0u;
            for (uint32_t o = 0; o < blocks; ++o) sum += *cluster.map_shared_rank(&hist[i], o);
            a.counts[(uint64_t)s * a.experts + i] = sum;
        }
        if (rank == 0u && tid == 0) {
            uint32_t sum = 0u;
            for (uint32_t o = 0; o < blocks; ++o) sum += *cluster.map_shared_rank(&tokens_in, o);
            a.counted[s] = sum;
        }
        cluster.sync();
    }
}

// Many tokens: a block per run of them, a histogram per segment, added to the counts (cleared before) with integer atomics, whose order
// changes nothing.
__global__ void __launch_bounds__(kCountThreads) k_clear_counts(CountArgs a) {
    wait_for_previous_kernels();
    allow_next_kernel();
    const uint64_t n = (uint64_t)a.segments * a.experts, step = (uint64_t)gridDim.x * kCountThreads;
    for (uint64_t i = (uint64_t)blockIdx.x * kCountThreads + threadIdx.x; i < n; i += step) a.counts[i] = 0u;
    for (uint64_t i = (uint64_t)blockIdx.x * kCountThreads + threadIdx.x; i < a.segments; i += step) a.counted[i] = 0u;
}
__global__ void __launch_bounds__(kCountThreads) k_add_expert_counts(CountArgs a) {
    __shared__ uint32_t hist[kBalanceMaxExperts], tokens_in;
    const uint32_t tid = threadIdx.x;
    wait_for_previous_kernels();
    const uint64_t r0 = (uint64_t)blockIdx.x * a.rows_per_block, r1 = r0 + a.rows_per_block < a.tokens ? r0 + a.rows_per_block : a.tokens;
    const Segments seg{a.offsets, a.tokens, a.segments};
    for (uint32_t s = seg.find(r0); s < a.segments; ++s) {
        uint64_t from = seg.edge(s), to = seg.edge(s + 1u);
        if (from >= r1) break;
        if (from < r0) from = r0;
        if (to > r1) to = r1;
        if (from >= to) continue;
        __syncthreads();
        for (uint32_t e = tid; e < a.experts; e += kCountThreads) hist[e] = 0u;
        if (tid == 0) tokens_in = 0u;
        __syncthreads();
        count_tokens(a, from, (uint32_t)(to - from), hist, &tokens_in);
        __syncthreads();
        for (uint32_t e = tid; e < a.experts; e += kCountThreads) if (hist[e]) atomicAdd(&a.counts[(uint64_t)s * a.experts + e], hist[e]);
        if (tid == 0 && tokens_in) atomicAdd(&a.counted[s], tokens_in);
    }
}

// 65536 x 256 bf16 with its gradient: 16 us, 4.2 TB/s (67 MB; a copy's time 10.2), with the counts of 8 experts a token 23 us in three launches.
// Bound by issue slots (57 %) and latency: 16 warps an SM.  A warp per token whatever the width: 81 with the counts; the next tokens' logits not
// ahead: 34; eight experts a lane: 26 (the reductions over lanes, and all that a token costs once, are then spread over half as many values).
// A block per run of tokens; LANES lanes share a token, each with CHUNKS times eight neighbouring experts, whose f it keeps in
// registers.  The logits of the next token (of the next few, with eight experts a lane: two in fp32, four in 16 bits) are on their way while those
// at hand are worked on.  With sixteen 16-bit experts a lane that is 16 KB an SM, half of what the memory's latency takes.
// The sum of a block's part of segment s goes to partials[block + s]: of two
// neighbours in the sequence of (block, segment) meetings one index grows, so that no two share a place.  The block that ends last
// adds the parts of each segment in their order.
template <class T, int CHUNKS> constexpr int kBalanceAhead = CHUNKS > 1 ? 1 : sizeof(T) == 2 ? 4 : 2;      // tokens that a group of lanes has in flight
template <class T, class TG, int LANES, int CHUNKS>
__global__ void __launch_bounds__(kBalanceThreads, CHUNKS > 1 ? 2 : 3) k_balance(BalanceArgs a) {
    __shared__ double part[kBalanceWarps];
    __shared__ uint32_t last;
    constexpr uint32_t PER_WARP = 32 / LANES;              // tokens
    constexpr int AHEAD = kBalanceAhead<T, CHUNKS>;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5, E = a.experts, group = lane / LANES, place = lane % LANES;
    constexpr float kLog2e = 1.4426950408889634f;
    constexpr uint32_t kStep = kBalanceWarps * PER_WARP;
    const uint64_t x_step = kStep * a.x_stride, g_step = kStep * a.grad_stride;
    const T* xs = static_cast<const T*>(a.x);
    TG* gs = static_cast<TG*>(a.grad);
    auto width_of = [&](int c) { const uint32_t e = (c * LANES + place) * 8u; return e < E ? min(E - e, 8u) : 0u; };
    const uint32_t x_unit = row_unit(xs, a.x_stride), g_unit = row_unit(gs, a.grad_stride);
    wait_for_previous_kernels();
    const uint64_t r0 = (uint64_t)blockIdx.x * a.rows_per_block, r1 = r0 + a.rows_per_block < a.tokens ? r0 + a.rows_per_block : a.tokens;
    const Segments seg{a.offsets, a.tokens, a.segments};
    for (uint32_t s = seg.find(r0); s < a.segments; ++s) {
        uint64_t from = seg.edge(s), to = seg.edge(s + 1u);
        if (from >= r1) break;
        if (from < r0) from = r0;
        if (to > r1) to = r1;
        if (from >= to) continue;
        // (32-bit numbers of the tokens behind `from`, pointers that walk)
        const uint32_t n_tokens = (uint32_t)(to - from), mine = warp * PER_WARP + group;
        Eight<T> next[AHEAD][CHUNKS];
        bool next_counts[AHEAD];
        uint32_t ahead = mine;
        const T* x_at = xs + (from + mine) * a.x_stride + place * 8u;
        const uint8_t* mask_at = a.mask ? a.mask + from + mine : nullptr;
        auto fetch = [&](int d) {
            next_counts[d] = ahead < n_tokens && (!mask_at || *mask_at);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) next[d][c] = load_eight(x_at + c * (LANES * 8), next_counts[d] ? width_of(c) : 0u, x_unit);
            ahead += kStep; x_at += x_step;
            if (mask_at) mask_at += kStep;
        };
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) fetch(d);
        float f[CHUNKS][8];
        {
            uint32_t n[CHUNKS][8];
            unsigned long long all = 0ull;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    n[c][i] = (uint32_t)i < width_of(c) ? a.counts[(uint64_t)s * E + (c * LANES + place) * 8u + i] : 0u;
                    all += n[c][i];
                }
#pragma unroll
            for (int o = LANES / 2; o; o >>= 1) all += __shfl_xor_sync(kFullMask, all, o);
            const float share = all ? 1.f / (float)all : 0.f;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) f[c][i] = (float)n[c][i] * share;
        }
        const uint32_t counted = a.counted[s];
        float scale = counted ? a.coef * (float)E / (float)counted : 0.f;
        if (a.grad_loss) scale *= a.grad_loss[s];
        double sum = 0.0;
        TG* g_at = gs + (from + mine) * a.grad_stride + place * 8u;
        for (uint32_t i0 = warp * PER_WARP; i0 < n_tokens;) {
            float dots_of_steps = 0.f;
#pragma unroll
            for (int d = 0; d < AHEAD; ++d, i0 += kStep, g_at += g_step) {
                if (i0 >= n_tokens) break;
                float v[CHUNKS][8];
                const bool counts = next_counts[d];
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) unpack_eight(next[d][c], v[c]);
                fetch(d);
                float m = kLowest;                         // (a token whose logits are all -inf: every p is 0)
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) m = fmaxf(m, v[c][i]);
                if (LANES == 32) m = warp_max(m);
                else {
#pragma unroll
                    for (int o = LANES / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kFullMask, m, o));
                }
                const unsigned long long minus_m = pair_of(-m, -m), cc = pair_of(kLog2e, kLog2e);
                unsigned long long totals = 0ull, dots = 0ull;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const float2 y = halves(mul_pairs(add_pairs(pair_of(v[c][i], v[c][i + 1]), minus_m), cc));
                        v[c][i] = exp2_fast(y.x); v[c][i + 1] = exp2_fast(y.y);
                        const unsigned long long p = pair_of(v[c][i], v[c][i + 1]);
                        totals = add_pairs(totals, p);
                        dots = fma_pairs(p, pair_of(f[c][i], f[c][i + 1]), dots);
                    }
                const float2 tt = halves(totals), dd = halves(dots);
                float total = tt.x + tt.y, dot = dd.x + dd.y;
#pragma unroll
                for (int o = LANES / 2; o; o >>= 1) { total += __shfl_xor_sync(kFullMask, total, o); dot += __shfl_xor_sync(kFullMask, dot, o); }
                const float inv = total == 0.f ? 0.f : 1.f / total;
                dot *= inv;
                dots_of_steps += dot;
                if (gs && i0 + group < n_tokens) {
                    const unsigned long long minus_dot = pair_of(-dot, -dot);
                    const float by = counts ? scale * inv : 0.f;
                    const unsigned long long bb = pair_of(by, by);
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c) {
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            const float2 y = halves(mul_pairs(mul_pairs(pair_of(v[c][i], v[c][i + 1]), bb), add_pairs(pair_of(f[c][i], f[c][i + 1]), minus_dot)));
                            v[c][i] = y.x; v[c][i + 1] = y.y;
                        }
                        store_eight(g_at + c * (LANES * 8), width_of(c), g_unit, v[c]);
                    }
                }
            }
            sum += (double)dots_of_steps;
        }
        if (a.loss) {
            // every lane of a group has its tokens' sum: one lane of each
            if (place) sum = 0.0;
            sum = warp_sum(sum);
            __syncthreads();
            if (lane == 0) part[warp] = sum;
            __syncthreads();
            if (tid == 0) {
                double p = 0.0;
                for (int w = 0; w < kBalanceWarps; ++w) p += part[w];
                a.partials[(uint64_t)blockIdx.x + s] = p;
            }
        }
    }
    if (!a.loss) return;
    if (tid == 0) {
        __threadfence();                                   // (this thread wrote the block's parts)
        last = atomicAdd(a.done, 1u) == gridDim.x - 1u;
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    // Few segments: all threads for each; many: eight lanes for each.
    auto parts_of = [&](uint32_t s, uint32_t first, uint32_t step) {
        const uint64_t from = seg.edge(s), to = seg.edge(s + 1u);
        double sum = 0.0;
        if (from < to) {
            const uint64_t b0 = from / a.rows_per_block, b1 = (to - 1u) / a.rows_per_block;
            for (uint64_t b = b0 + first; b <= b1; b += step) sum += __ldcg(a.partials + b + s);
        }
        return sum;
    };
    auto finish = [&](uint32_t s, uint32_t n, double sum) { a.loss[s] = n ? (float)((double)a.coef * (double)E * sum / (double)n) : 0.f; };
    if (a.segments < 8u) {
        for (uint32_t s = 0; s < a.segments; ++s) {
            const uint32_t n = a.counted[s];
            const double sum = block_sum<kBalanceWarps>(parts_of(s, tid, kBalanceThreads), part);
            if (tid == 0) finish(s, n, sum);
        }
    } else {
        for (uint32_t s0 = 0; s0 < a.segments; s0 += kBalanceThreads / 8) {
            const uint32_t s = s0 + tid / 8u;
            const uint32_t n = s < a.segments ? a.counted[s] : 0u;
            double sum = s < a.segments ? parts_of(s, tid % 8u, 8u) : 0.0;
#pragma unroll
            for (int o = 4; o; o >>= 1) sum += __shfl_xor_sync(kFullMask, sum, o);
            if (s < a.segments && tid % 8u == 0u) finish(s, n, sum);
        }
    }
    if (tid == 0) *a.done = 0u;
}

}  // namespace fsg
