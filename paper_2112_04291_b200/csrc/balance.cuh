// Per-expert counts of the experts that a router selected, and the balance loss with its gradient.  Per segment s of tokens
// (x: the router's logits, p = softmax(x), E experts, n_s tokens that count):
//   f_e = counts_se / sum_e counts_se,      L_s = coef E sum_e f_e (1/n_s) sum_t p_te,
//   dL_s / dx_te = (coef E / n_s) p_te (f_e - sum_e' f_e' p_te').
// The gradient depends on the counts alone and not on the mean of p: with the counts known first, one pass over x gives the
// gradient and, as the sum over the tokens of sum_e f_e p_te, the loss.
#pragma once

#include "rows.cuh"

namespace fsg {

constexpr int kBalanceThreads = 256;
constexpr int kBalanceWarps   = kBalanceThreads / 32;
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
    // the first segment that ends behind token t
    __device__ __forceinline__ uint32_t find(uint64_t t) const {
        uint32_t lo = 0u, hi = count;
        while (lo < hi) { const uint32_t mid = (lo + hi) >> 1; if (edge(mid + 1u) > t) hi = mid; else lo = mid + 1u; }
        return lo;
    }
};

// A block per run of tokens: a histogram per segment in shared memory, added to the counts (cleared before) with integer atomics,
// whose order changes nothing.
__global__ void __launch_bounds__(kBalanceThreads) k_expert_counts(CountArgs a) {
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
        for (uint32_t e = tid; e < a.experts; e += kBalanceThreads) hist[e] = 0u;
        if (tid == 0) tokens_in = 0u;
        __syncthreads();
        const uint32_t n = (uint32_t)(to - from);
        if (a.mask) {
            uint32_t mine = 0u;
            for (uint32_t t = tid; t < n; t += kBalanceThreads) mine += a.mask[from + t] != 0;
            if (mine) atomicAdd(&tokens_in, mine);
        } else if (tid == 0) tokens_in = n;
        const int32_t* sel = a.selected + from * a.k;
        for (uint32_t i = tid; i < n * a.k; i += kBalanceThreads) {
            const int e = sel[i];
            if (e >= 0 && (uint32_t)e < a.experts && (!a.mask || a.mask[from + i / a.k])) atomicAdd(&hist[e], 1u);
        }
        __syncthreads();
        for (uint32_t e = tid; e < a.experts; e += kBalanceThreads) if (hist[e]) atomicAdd(&a.counts[(uint64_t)s * a.experts + e], hist[e]);
        if (tid == 0 && tokens_in) atomicAdd(&a.counted[s], tokens_in);
    }
}

// A block per run of tokens, a warp per token.  The sum of a block's part of segment s goes to partials[block + s]: of two
// neighbours in the sequence of (block, segment) meetings one index grows, so that no two share a place.  The block that ends last
// adds the parts of each segment in their order.
template <class T, class TG>
__global__ void __launch_bounds__(kBalanceThreads) k_balance(BalanceArgs a) {
    __shared__ float f[kBalanceMaxExperts];
    __shared__ unsigned long long whole[kBalanceWarps];
    __shared__ double part[kBalanceWarps];
    __shared__ uint32_t last;
    constexpr int PER = kBalanceMaxExperts / 32;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5, E = a.experts;
    constexpr float kLog2e = 1.4426950408889634f;
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
        unsigned long long mine = 0ull;
        for (uint32_t e = tid; e < E; e += kBalanceThreads) mine += a.counts[(uint64_t)s * E + e];
        const unsigned long long all = block_sum<kBalanceWarps>(mine, whole);
        for (uint32_t e = tid; e < E; e += kBalanceThreads) f[e] = all ? (float)a.counts[(uint64_t)s * E + e] / (float)all : 0.f;
        __syncthreads();
        const uint32_t n = a.counted[s];
        float scale = n ? a.coef * (float)E / (float)n : 0.f;
        if (a.grad_loss) scale *= a.grad_loss[s];
        double sum = 0.0;
        for (uint64_t t = from + warp; t < to; t += kBalanceWarps) {
            const T* x = static_cast<const T*>(a.x) + t * a.x_stride;
            TG* g = a.grad ? static_cast<TG*>(a.grad) + t * a.grad_stride : nullptr;
            float v[PER], m = -INFINITY;
            const bool counts = !a.mask || a.mask[t];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint32_t e = lane + 32u * i;
                v[i] = counts && e < E ? to_float(x[e]) : -INFINITY;
                m = fmaxf(m, v[i]);
            }
            m = fmaxf(warp_max(m), kLowest);               // (a token whose logits are all -inf: every p is 0)
            float total = 0.f, dot = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint32_t e = lane + 32u * i;
                v[i] = exp2_fast((v[i] - m) * kLog2e);
                total += v[i];
                if (e < E) dot += v[i] * f[e];
            }
            total = warp_sum(total);
            const float inv = total == 0.f ? 0.f : 1.f / total;
            dot = warp_sum(dot) * inv;
            if (g) {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const uint32_t e = lane + 32u * i;
                    if (e < E) g[e] = from_float<TG>(scale * (v[i] * inv) * (f[e] - dot));
                }
            }
            sum += (double)dot;
        }
        if (a.loss) {
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
    __syncthreads();
    if (tid == 0) {
        __threadfence();                                   // (this thread wrote the block's parts)
        last = atomicAdd(a.done, 1u) == gridDim.x - 1u;
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    for (uint32_t s = warp; s < a.segments; s += kBalanceWarps) {
        const uint64_t from = seg.edge(s), to = seg.edge(s + 1u);
        double sum = 0.0;
        if (from < to) {
            const uint64_t b0 = from / a.rows_per_block, b1 = (to - 1u) / a.rows_per_block;
            for (uint64_t b = b0 + lane; b <= b1; b += 32u) sum += __ldcg(a.partials + b + s);
        }
        sum = warp_sum(sum);
        if (lane == 0) { const uint32_t n = a.counted[s]; a.loss[s] = n ? (float)((double)a.coef * (double)E * sum / (double)n) : 0.f; }
    }
    if (tid == 0) *a.done = 0u;
}

}  // namespace fsg
