// The k largest of a row of logits as (key, value) pairs, in descending order and, among equals, in ascending order of their keys;
// with them log sum_j exp(z_j / T) and the share of that sum outside of the pairs.
//
// Values are compared as 32-bit words that ascend with them (NaN above all, -0 equal to +0); a candidate is that word and the
// complement of its key in 64 bits, so that no two are equal and the order in which they are found does not matter.
#pragma once

#include "rows.cuh"

namespace fsg {

constexpr int kTopThreads = 512;
constexpr int kTopWarps   = kTopThreads / 32;
constexpr uint32_t kTopMaxPairs = 1024u;

struct TopArgs {
    const void* z; int32_t* keys; void* values; float* lse; float* tail;
    uint64_t rows, z_stride;
    uint32_t cols, k;
    float temperature, c;                                  // c = log2(e) / T
};

__device__ __forceinline__ uint32_t rank_of(float x) {
    const uint32_t b = __float_as_uint(__fadd_rn(x, 0.f));
    return x != x ? 0xFFFFFFFFu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of_rank(uint32_t r) {
    return __uint_as_float(r & 0x80000000u ? r ^ 0x80000000u : ~r);      // (of NaN's word: a NaN)
}
__device__ __forceinline__ unsigned long long candidate(uint32_t rank, uint32_t key) { return (unsigned long long)rank << 32 | (uint32_t)~key; }

// f(j, z_j) for the elements [0, n) of a row, in no particular order.
template <class T, class F>
__device__ __forceinline__ void for_each_element(const T* z, uint32_t n, F f) {
    constexpr int N = Vec<T>::N, U = 4;
    const uint32_t tid = threadIdx.x;
    const Span sp = span_of(z, n);
    if (tid < sp.head) f(tid, to_float(z[tid]));
    if (tid < sp.tail) { const uint32_t j = n - sp.tail + tid; f(j, to_float(z[j])); }
    const T* body = z + sp.head;
    for (uint32_t v0 = tid; v0 < sp.vecs; v0 += U * kTopThreads) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v0 + u * kTopThreads < sp.vecs) raw[u] = load16(body + (uint64_t)(v0 + u * kTopThreads) * N);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t v = v0 + u * kTopThreads;
            if (v >= sp.vecs) break;
            float x[N];
            Vec<T>::unpack(raw[u], x);
#pragma unroll
            for (int i = 0; i < N; ++i) f(sp.head + v * N + i, x[i]);
        }
    }
}

struct TopShared {
    unsigned long long cand[kTopMaxPairs];
    uint32_t hist[256];
    uint32_t bin, above, equal, taken;
    float  one[kTopWarps];
    uint32_t count[kTopWarps];
};

// The bin that holds the `need`-th entry counted from the last bin down, and how many lie in later bins.  One warp.
__device__ __forceinline__ void find_bin(const uint32_t* hist, uint32_t need, uint32_t& bin, uint32_t& above, uint32_t& in_bin) {
    const int lane = threadIdx.x & 31;
    uint32_t h[8], sum = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += h[i] = hist[255 - (8 * lane + i)];
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(kFullMask, upto, o); if (lane >= o) upto += y; }
    const uint32_t before = upto - sum;
    if (before < need && need <= upto) {                   // exactly one lane
        uint32_t at = before;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (at < need && need <= at + h[i]) { bin = 255u - (uint32_t)(8 * lane + i); above = at; in_bin = h[i]; }
            at += h[i];
        }
    }
}

// Descending order of the first `count` (a power of two) candidates.
__device__ __forceinline__ void sort_candidates(unsigned long long* cand, uint32_t count) {
    for (uint32_t size = 2u; size <= count; size <<= 1)
        for (uint32_t step = size >> 1; step; step >>= 1) {
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < count / 2u; i += kTopThreads) {
                const uint32_t a = 2u * i - (i & (step - 1u)), b = a + step;
                const unsigned long long x = cand[a], y = cand[b];
                if ((x < y) == ((a & size) == 0u)) { cand[a] = y; cand[b] = x; }
            }
        }
    __syncthreads();
}

// A block per row: the k-th largest word by four histograms of eight bits, then the pairs, then the sums.
template <class T>
__global__ void __launch_bounds__(kTopThreads) k_top(TopArgs a) {
    __shared__ TopShared s;
    const uint32_t tid = threadIdx.x, k = a.k;
    uint32_t pow2 = 1u;
    while (pow2 < k) pow2 <<= 1;
    wait_for_previous_kernels();
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* z = static_cast<const T*>(a.z) + row * a.z_stride;
        uint32_t prefix = 0u, need = k, equal = 0u;
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            if (tid < 256u) s.hist[tid] = 0u;
            __syncthreads();
            const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
            for_each_element(z, a.cols, [&](uint32_t, float x) {
                const uint32_t r = rank_of(x);
                if ((r & mask) == prefix) atomicAdd(&s.hist[r >> shift & 255u], 1u);
            });
            __syncthreads();
            if (tid < 32u) find_bin(s.hist, need, s.bin, s.above, s.equal);
            __syncthreads();
            prefix |= s.bin << shift; need -= s.above; equal = s.equal;
        }
        // `need` of the `equal` values with the word `prefix`, and all above it
        if (tid == 0) s.taken = 0u;
        for (uint32_t i = tid; i < pow2; i += kTopThreads) s.cand[i] = 0ull;
        __syncthreads();
        for_each_element(z, a.cols, [&](uint32_t j, float x) {
            const uint32_t r = rank_of(x);
            if (r > prefix || (r == prefix && need == equal)) s.cand[atomicAdd(&s.taken, 1u)] = candidate(r, j);
        });
        __syncthreads();
        if (need < equal) {                                // the first of them by key
            uint32_t got = 0u;
            for (uint32_t j0 = 0; j0 < a.cols && got < need; j0 += kTopThreads) {
                const bool hit = j0 + tid < a.cols && rank_of(to_float(z[j0 + tid])) == prefix;
                const unsigned ballot = __ballot_sync(kFullMask, hit);
                if ((tid & 31u) == 0u) s.count[tid >> 5] = __popc(ballot);
                __syncthreads();
                uint32_t before = got, all = 0u;
                for (uint32_t w = 0; w < (uint32_t)kTopWarps; ++w) { if (w < tid >> 5) before += s.count[w]; all += s.count[w]; }
                before += __popc(ballot & ((1u << (tid & 31u)) - 1u));
                if (hit && before < need) s.cand[k - need + before] = candidate(prefix, j0 + tid);
                got += all;
                __syncthreads();
            }
        }
        sort_candidates(s.cand, pow2);
        if (a.lse || a.tail) {
            const float m = value_of_rank((uint32_t)(s.cand[0] >> 32)), last = value_of_rank(prefix);
            float rest = 0.f, in = 0.f;
            for_each_element(z, a.cols, [&](uint32_t, float x) { if (rank_of(x) < prefix) rest += exp2_fast((x - m) * a.c); });
            for (uint32_t i = tid; i < k; i += kTopThreads) in += exp2_fast((value_of_rank((uint32_t)(s.cand[i] >> 32)) - m) * a.c);
            rest = block_sum<kTopWarps>(rest, s.one);
            in = block_sum<kTopWarps>(in, s.one);
            if (tid == 0) {
                if (need < equal) rest += (float)(equal - need) * exp2_fast((last - m) * a.c);
                const bool none = m == -INFINITY;
                if (a.lse) a.lse[row] = none ? m : m / a.temperature + logf(rest + in);
                if (a.tail) a.tail[row] = none ? 0.f : rest / (rest + in);
            }
        }
        for (uint32_t i = tid; i < k; i += kTopThreads) {
            const uint32_t key = ~(uint32_t)s.cand[i];
            a.keys[row * k + i] = (int32_t)key;
            static_cast<T*>(a.values)[row * k + i] = z[key];
        }
        __syncthreads();
    }
}

}  // namespace fsg
