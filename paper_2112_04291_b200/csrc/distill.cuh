// Distillation from a teacher's top logits: loss and gradient of a row of student logits z against the teacher's pairs
// (key_i, t_i), i < k, and the share `tail` of the teacher's probability outside of them.  With q = softmax(z / T),
//   p_i  = (1 - tail) softmax(t / T)_i over the pairs whose key lies in [0, V),      rest = sum of q_j over j that are no key,
//   loss = w T^2 ( sum_i p_i (log p_i - log q_key_i) + tail (log tail - log rest) ),
//   d loss / d z_j = w T ( q_j - sum of p_i with key_i = j )       for a key j,
//                  = w T q_j (1 - tail / rest)                     for the others.
// With a tail, the sum of exponentials runs over the others alone: rest then has no cancellation (1 - sum of the keys' q would
// lose it where the student is sure), and the gradient of the others is their share of that sum times w T (rest - tail).
#pragma once

#include "rows.cuh"

namespace fsg {

constexpr int kDistillThreads = 512;
constexpr int kDistillWarps   = kDistillThreads / 32;
constexpr uint32_t kDistillMaxPairs = 1024u;
constexpr uint32_t kDistillMaxCols  = 1u << 20;            // a bit per class in shared memory

// what a launch computes
constexpr int kLossOnly = 0, kLossAndGrad = 1, kGradOnly = 2;      // kGradOnly: from the sums that a forward launch kept

struct DistillArgs {
    const void* z; void* grad;
    const int32_t* keys; const void* values; const float* tail;
    const float* weight; const float* grad_loss; const float* stats_in;
    float* loss; float* stats_out;
    uint64_t rows, z_stride, grad_stride;
    uint32_t cols, k, values_type;
    float temperature, inv_t, c, slack;                    // c = log2(e) / T
};

struct DistillShared {
    int   key[kDistillMaxPairs];                           // -1: absent
    float z[kDistillMaxPairs], p[kDistillMaxPairs], lp[kDistillMaxPairs];
    float2 join[kDistillWarps];
    float  one[kDistillWarps];
    double two[kDistillWarps];
};

// bits j .. j + N - 1 of the map of keys (which has a word more than it needs)
template <int N> __device__ __forceinline__ uint32_t key_bits(const uint32_t* map, uint32_t j) {
    return __funnelshift_r(map[j >> 5], map[(j >> 5) + 1u], j & 31u) & ((1u << N) - 1u);
}

// The sum of exponentials of a row's elements [0, n), without the keys of `map` where there is one.
template <class T>
__device__ __forceinline__ ExpSum scan_row(const T* z, uint32_t n, const uint32_t* map, float c, float slack) {
    constexpr int N = Vec<T>::N, U = 4;
    const uint32_t tid = threadIdx.x;
    const Span sp = span_of(z, n);
    ExpSum e;
    auto single = [&](uint32_t j) { if (!map || !(map[j >> 5] >> (j & 31u) & 1u)) e.add(to_float(z[j]), c, slack); };
    if (tid < sp.head) single(tid);
    if (tid < sp.tail) single(n - sp.tail + tid);
    const T* body = z + sp.head;
    for (uint32_t v0 = tid; v0 < sp.vecs; v0 += U * kDistillThreads) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v0 + u * kDistillThreads < sp.vecs) raw[u] = load16(body + (uint64_t)(v0 + u * kDistillThreads) * N);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t v = v0 + u * kDistillThreads;
            if (v >= sp.vecs) break;
            float f[N];
            Vec<T>::unpack(raw[u], f);
            float top = Vec<T>::max(raw[u]);
            if (map) {
                const uint32_t b = key_bits<N>(map, sp.head + v * N);
                if (b) {
                    top = kLowest;
#pragma unroll
                    for (int i = 0; i < N; ++i) { if (b >> i & 1u) f[i] = -INFINITY; top = fmaxf(top, f[i]); }
                }
            }
            e.raise(top, c, slack);
#pragma unroll
            for (int i = 0; i < N; ++i) e.s += exp2_fast((f[i] - e.m) * c);
        }
    }
    return e;
}

// grad[j] = a 2^((z_j - m) c) for the elements [0, n) of a row (a = 0: zero).
template <class TZ, class TG>
__device__ __forceinline__ void write_row(const TZ* z, TG* g, uint32_t n, float a, float m, float c) {
    constexpr int N = Vec<TZ>::N, U = 4;
    const uint32_t tid = threadIdx.x;
    const Span sp = span_of(z, n);
    const bool wide = (reinterpret_cast<uintptr_t>(g + sp.head) & 15u) == 0u;
    auto single = [&](uint32_t j) { g[j] = from_float<TG>(exp2_fast((to_float(z[j]) - m) * c) * a); };
    if (tid < sp.head) single(tid);
    if (tid < sp.tail) single(n - sp.tail + tid);
    const TZ* body = z + sp.head;
    TG* out = g + sp.head;
    for (uint32_t v0 = tid; v0 < sp.vecs; v0 += U * kDistillThreads) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v0 + u * kDistillThreads < sp.vecs) raw[u] = load16(body + (uint64_t)(v0 + u * kDistillThreads) * N);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t v = v0 + u * kDistillThreads;
            if (v >= sp.vecs) break;
            float f[N];
            Vec<TZ>::unpack(raw[u], f);
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = exp2_fast((f[i] - m) * c) * a;
            store_values(out + (uint64_t)v * N, f, wide);
        }
    }
}
template <class TG>
__device__ __forceinline__ void zero_row(TG* g, uint32_t n) {
    constexpr int N = Vec<TG>::N;
    const Span sp = span_of(g, n);
    if (threadIdx.x < sp.head) g[threadIdx.x] = from_float<TG>(0.f);
    if (threadIdx.x < sp.tail) g[n - sp.tail + threadIdx.x] = from_float<TG>(0.f);
    for (uint32_t v = threadIdx.x; v < sp.vecs; v += kDistillThreads) store16(g + sp.head + (uint64_t)v * N, make_uint4(0u, 0u, 0u, 0u));
}

// A block per row: the pairs, one pass over the row for the sum of exponentials, one more for the gradient (from the L2).
template <class TZ, class TG, int MODE>
__global__ void __launch_bounds__(kDistillThreads) k_distill(DistillArgs a) {
    extern __shared__ uint32_t map[];                      // a bit per class: it is a key of this row
    __shared__ DistillShared s;
    const uint32_t tid = threadIdx.x, k = a.k;
    const uint32_t words = (a.cols + 31u) / 32u + 1u;
    const bool mapped = MODE != kLossOnly || a.tail;
    wait_for_previous_kernels();
    if (mapped) for (uint32_t i = tid; i < words; i += kDistillThreads) map[i] = 0u;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const TZ* z = static_cast<const TZ*>(a.z) + row * a.z_stride;
        TG* g = MODE == kLossOnly ? nullptr : static_cast<TG*>(a.grad) + row * a.grad_stride;
        const float w = a.weight ? a.weight[row] : 1.f;
        __syncthreads();                                   // (the last row's pairs are no longer in use)

        // ---- the pairs -----------------------------------------------------------------------
        float tm = -INFINITY, zm = kLowest;
        bool again = false;
        if (w != 0.f) {
            for (uint32_t i = tid; i < k; i += kDistillThreads) {
                const int key = a.keys[row * k + i];
                const bool here = key >= 0 && (uint32_t)key < a.cols;
                const float t = here ? load_typed(a.values, row * k + i, a.values_type) : -INFINITY;
                const float zk = here ? to_float(z[key]) : -INFINITY;
                s.key[i] = here ? key : -1; s.lp[i] = t; s.z[i] = zk;
                tm = fmaxf(tm, t); zm = fmaxf(zm, zk);
                if (here && mapped) again |= atomicOr(&map[key >> 5], 1u << (key & 31)) >> (key & 31) & 1u;
            }
        }
        tm = block_max<kDistillWarps>(tm, s.one);
        if (!(tm > -INFINITY)) {                           // weight 0, or no pair with any probability: the row counts for nothing
            if (mapped && w != 0.f) for (uint32_t i = tid; i < k; i += kDistillThreads) if (s.key[i] >= 0) map[s.key[i] >> 5] = 0u;
            if (MODE != kLossOnly) zero_row(g, a.cols);
            if (tid == 0) {
                if (MODE != kGradOnly && a.loss) a.loss[row] = 0.f;
                if (MODE != kGradOnly && a.stats_out) { a.stats_out[2 * row] = 0.f; a.stats_out[2 * row + 1] = 0.f; }
            }
            continue;
        }
        zm = block_max<kDistillWarps>(zm, s.one);
        again = __syncthreads_or(again);
        float tsum = 0.f;
        for (uint32_t i = tid; i < k; i += kDistillThreads) tsum += s.p[i] = exp2_fast((s.lp[i] - tm) * a.c);
        tsum = block_sum<kDistillWarps>(tsum, s.one);
        const float tail = a.tail ? a.tail[row] : 0.f;
        const bool tailed = tail != 0.f;
        const float share = (1.f - tail) / tsum, log_share = logf(1.f - tail) - logf(tsum);
        for (uint32_t i = tid; i < k; i += kDistillThreads) { s.p[i] *= share; s.lp[i] = (s.lp[i] - tm) * a.inv_t + log_share; }

        // ---- the sum of exponentials, of all classes or (with a tail) of those that are no key ----
        ExpSum e;
        if (MODE == kGradOnly) { e.m = a.stats_in[2 * row]; e.s = a.stats_in[2 * row + 1]; }
        else e = block_join<kDistillWarps>(scan_row(z, a.cols, tailed ? map : nullptr, a.c, a.slack), s.join, a.c);
        __syncthreads();
        // A key that appears several times counts once for the student, and all its pairs' probability goes to its first pair.
        float ksum = 0.f, top = e.m, total = e.s, lead[(kDistillMaxPairs + kDistillThreads - 1) / kDistillThreads];
        if (tailed) top = fmaxf(e.m, zm);
#pragma unroll
        for (int n = 0; n < (int)(sizeof(lead) / sizeof(float)); ++n) {
            const uint32_t i = tid + n * kDistillThreads;
            lead[n] = -1.f;                                // no gradient of its own
            if (i >= k || s.key[i] < 0) continue;
            float p = s.p[i];
            bool first = true;
            if (again) {
                p = 0.f;
                for (uint32_t j = 0; j < k; ++j) if (s.key[j] == s.key[i]) { p += s.p[j]; first &= j >= i; }
            }
            if (first) { lead[n] = p; if (tailed) ksum += exp2_fast((s.z[i] - top) * a.c); }
        }
        const float rest = e.s * exp2_fast((e.m - top) * a.c);
        if (tailed) total = block_sum<kDistillWarps>(ksum, s.one) + rest;
        const bool none = total == 0.f;                    // every logit of the row is -inf: it counts for nothing, too
        if (MODE != kGradOnly) {
            double sum = 0.0;
            const float log_total = logf(total);
            for (uint32_t i = tid; i < k; i += kDistillThreads)
                if (s.key[i] >= 0 && s.p[i] != 0.f) sum += (double)(s.p[i] * (s.lp[i] - (s.z[i] - top) * a.inv_t + log_total));
            sum = block_sum<kDistillWarps>(sum, s.two);
            if (tid == 0) {
                if (tailed) sum += (double)(tail * (logf(tail) - (e.m - top) * a.inv_t - logf(e.s) + log_total));
                if (a.loss) a.loss[row] = none ? 0.f : w * a.temperature * a.temperature * (float)sum;
                if (a.stats_out) { a.stats_out[2 * row] = e.m; a.stats_out[2 * row + 1] = e.s; }
            }
        }
        // ---- the gradient ----------------------------------------------------------------------
        if (MODE != kLossOnly) {
            const float scale = none ? 0.f : w * a.temperature * (a.grad_loss ? a.grad_loss[row] : 1.f);
            if (none) zero_row(g, a.cols);
            else write_row(z, g, a.cols, e.s == 0.f ? 0.f : scale * (tailed ? rest / total - tail : 1.f) / e.s, e.m, a.c);
            __syncthreads();
#pragma unroll
            for (int n = 0; n < (int)(sizeof(lead) / sizeof(float)); ++n) {
                const uint32_t i = tid + n * kDistillThreads;
                if (i < k && s.key[i] >= 0 && !none && !(lead[n] < 0.f)) g[s.key[i]] = from_float<TG>(scale * (exp2_fast((s.z[i] - top) * a.c) / total - lead[n]));
            }
        }
        if (mapped) for (uint32_t i = tid; i < k; i += kDistillThreads) if (s.key[i] >= 0) map[s.key[i] >> 5] = 0u;
    }
}

}  // namespace fsg
