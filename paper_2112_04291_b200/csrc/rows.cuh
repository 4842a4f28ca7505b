// Rows of logits: element types, 16-byte loads and stores at any row alignment, sums of exponentials relative to a running
// maximum, and block-wide reductions.  Shared by the kernels on top logits, the distillation loss and the balance loss.
//
// exp(x / T) is taken as 2^(x c), c = log2(e) / T, always of a difference (x - m): a difference of two logits is exact where it
// matters, whereas x c - m c would carry the rounding of m c (and overflow for a row of the type's lowest value).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace fsg {

constexpr uint32_t kTypeF32 = 0u, kTypeBf16 = 1u, kTypeF16 = 2u;
constexpr float    kLowest  = -3.402823466e+38f;

__device__ __forceinline__ float exp2_fast(float x) {       // relative error 2^-22; results below 2^-126 are zero
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <class T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// element i of an array whose type is known at run time only
__device__ __forceinline__ float load_typed(const void* p, uint64_t i, uint32_t type) {
    return type == kTypeF32 ? static_cast<const float*>(p)[i]
         : type == kTypeBf16 ? to_float(static_cast<const __nv_bfloat16*>(p)[i]) : to_float(static_cast<const __half*>(p)[i]);
}

// 16 bytes that are read once by one thread
__device__ __forceinline__ uint4 load16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
// 16 bytes from global to shared memory without a register in between.  Each thread waits for, and reads, what it has copied itself.
__device__ __forceinline__ void copy16_async(void* smem, const void* p) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(__cvta_generic_to_global(p)) : "memory");
}
__device__ __forceinline__ void copies_end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }
__device__ __forceinline__ void store16(void* p, uint4 v) {
    asm volatile("st.global.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

__device__ __forceinline__ float nan_or_max(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// The elements of a 16-byte vector of T, and their maximum (without NaN, or NaN if there is one).
template <class T> struct Vec;
template <> struct Vec<float> {
    static constexpr int N = 4;
    static constexpr uint32_t kMinusInf = 0xFF800000u;      // a word of -inf
    static __device__ __forceinline__ void unpack(uint4 v, float (&f)[4]) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ float max(uint4 v) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    static __device__ __forceinline__ float max_nan(uint4 v) {
        return nan_or_max(nan_or_max(__uint_as_float(v.x), __uint_as_float(v.y)), nan_or_max(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    static constexpr uint32_t kMinusInf = 0xFF80FF80u;
    static __device__ __forceinline__ void unpack(uint4 v, float (&f)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
    static __device__ __forceinline__ float max(uint4 v) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
        const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__bfloat162float(m.x), __bfloat162float(m.y));
    }
    static __device__ __forceinline__ float max_nan(uint4 v) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
        const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
        return nan_or_max(__bfloat162float(m.x), __bfloat162float(m.y));
    }
};
template <> struct Vec<__half> {
    static constexpr int N = 8;
    static constexpr uint32_t kMinusInf = 0xFC00FC00u;
    static __device__ __forceinline__ void unpack(uint4 v, float (&f)[8]) {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 x = __half22float2(h[i]); f[2 * i] = x.x; f[2 * i + 1] = x.y; }
    }
    static __device__ __forceinline__ float max(uint4 v) {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
        const __half2 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__half2float(m.x), __half2float(m.y));
    }
    static __device__ __forceinline__ float max_nan(uint4 v) {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
        const __half2 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
        return nan_or_max(__half2float(m.x), __half2float(m.y));
    }
};

// N consecutive values to an array of T, in 16-byte stores (wide) or one by one.
template <int N> __device__ __forceinline__ void store_values(float* p, const float (&f)[N], bool wide) {
    if (wide) {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            store16(p + i, make_uint4(__float_as_uint(f[i]), __float_as_uint(f[i + 1]), __float_as_uint(f[i + 2]), __float_as_uint(f[i + 3])));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = f[i];
    }
}
template <class T> __device__ __forceinline__ uint32_t pack_two(float a, float b);
template <> __device__ __forceinline__ uint32_t pack_two<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack_two<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <class T, int N> __device__ __forceinline__ void store_values(T* p, const float (&f)[N], bool wide) {
    static_assert(N == 8, "a vector of 16-bit values");
    if (wide) store16(p, make_uint4(pack_two<T>(f[0], f[1]), pack_two<T>(f[2], f[3]), pack_two<T>(f[4], f[5]), pack_two<T>(f[6], f[7])));
    else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = from_float<T>(f[i]);
    }
}

// Eight consecutive elements from p on as they are, those behind the first n as -inf.  unit: 16 or 8 where p lies on a boundary of so
// many bytes, otherwise less.
template <class T> struct Eight { uint4 raw[8 / Vec<T>::N]; };
template <class T> __device__ __forceinline__ Eight<T> load_eight(const T* p, uint32_t n, uint32_t unit) {
    constexpr int N = Vec<T>::N, H = N / 2;                // elements of 16 and of 8 bytes
    Eight<T> r;
    if (unit == 16u && n >= 8u) {
#pragma unroll
        for (int h = 0; h < 8 / N; ++h) r.raw[h] = load16(p + h * N);
    } else {
        alignas(16) T x[8];
#pragma unroll
        for (int h = 0; h < 8; h += H) {
            if (unit >= 8u && n >= (uint32_t)(h + H)) *reinterpret_cast<uint2*>(x + h) = *reinterpret_cast<const uint2*>(p + h);
            else {
#pragma unroll
                for (int i = h; i < h + H; ++i) x[i] = (uint32_t)i < n ? p[i] : from_float<T>(-INFINITY);
            }
        }
#pragma unroll
        for (int h = 0; h < 8 / N; ++h) r.raw[h] = *reinterpret_cast<const uint4*>(x + h * N);
    }
    return r;
}
template <class T> __device__ __forceinline__ void unpack_eight(const Eight<T>& r, float (&f)[8]) {
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int h = 0; h < 8 / N; ++h) {
        float x[N];
        Vec<T>::unpack(r.raw[h], x);
#pragma unroll
        for (int i = 0; i < N; ++i) f[h * N + i] = x[i];
    }
}
template <class T> __device__ __forceinline__ void store_eight(T* p, uint32_t n, uint32_t unit, const float (&f)[8]) {
    constexpr int H = Vec<T>::N / 2;
    if (unit == 16u && n >= 8u) store_values(p, f, true);
    else {
        alignas(16) T x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = from_float<T>(f[i]);
#pragma unroll
        for (int h = 0; h < 8; h += H) {
            if (unit >= 8u && n >= (uint32_t)(h + H)) *reinterpret_cast<uint2*>(p + h) = *reinterpret_cast<const uint2*>(x + h);
            else {
#pragma unroll
                for (int i = h; i < h + H; ++i) if ((uint32_t)i < n) p[i] = x[i];
            }
        }
    }
}
// 16, 8 or 0: the boundary on which every row of so many elements apart begins
template <class T> __device__ __forceinline__ uint32_t row_unit(const T* p, uint64_t stride) {
    const uint64_t at = reinterpret_cast<uintptr_t>(p) | stride * sizeof(T);
    return at & 7u ? 0u : at & 15u ? 8u : 16u;
}

// A run of n elements from p on: `head` single elements up to a 16-byte boundary, `vecs` vectors, `tail` single elements.
struct Span {
    uint32_t head, vecs, tail;
};
template <class T> __device__ __forceinline__ Span span_of(const T* p, uint32_t n) {
    Span s;
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u) / (uint32_t)sizeof(T);
    s.head = off ? (uint32_t)Vec<T>::N - off : 0u;
    if (s.head > n) s.head = n;
    s.vecs = (n - s.head) / (uint32_t)Vec<T>::N;
    s.tail = n - s.head - s.vecs * (uint32_t)Vec<T>::N;
    return s;
}

// sum of 2^((x - m) c) over the values added so far.  m is one of them, or the lowest value; it follows the largest only once that
// is 2^40 times what m gives, so that the sum is hardly ever rescaled and stays far from overflow.  Infinite values of -inf add
// nothing; NaN and +inf make the sum NaN.
struct ExpSum {
    float m, s;
    __device__ __forceinline__ ExpSum() : m(kLowest), s(0.f) {}
    __device__ __forceinline__ void raise(float top, float c, float slack) {
        if (top > m + slack) { s *= exp2_fast((m - top) * c); m = top; }
    }
    __device__ __forceinline__ void add(float x, float c, float slack) {
        raise(x, c, slack);
        s += exp2_fast((x - m) * c);
    }
    __device__ __forceinline__ void join(float m2, float s2, float c) {
        const float top = fmaxf(m, m2);
        s = s * exp2_fast((m - top) * c) + s2 * exp2_fast((m2 - top) * c);
        m = top;
    }
};
// Two fp32 operations in one instruction.
__device__ __forceinline__ unsigned long long pair_of(float a, float b) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 halves(unsigned long long p) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
    return r;
}
__device__ __forceinline__ unsigned long long add_pairs(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long mul_pairs(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ unsigned long long fma_pairs(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// |m| c of 2^26 and more: m c rounded to fp32 would be off by 2 and more.
__device__ __forceinline__ bool is_far(float m, float c) { return !(fabsf(m) * c < 67108864.f); }
// ... of 2^25 and more: there may be something left next to m of a sum whose own largest value is far (neighbours of fp32 are 2^4 to 2^8 apart
// there, and the value that a sum is relative to may be 2^40 below its largest).
__device__ __forceinline__ bool may_miss_far(float m, float c) { return !(fabsf(m) * c < 33554432.f); }

// The same sum, of vectors: four partial sums, two operations at a time; raise() before add(), with the maximum of what is added.  The
// argument takes one fused operation: 2^(x c - r), r = m c rounded, which whole() makes up for.  Where m is far the
// sum is 0 instead: next to a largest value well below that border, what it would hold is 0 indeed; where the row's largest value may miss
// something, or its sum is 0, the caller takes the sum the other way.  A NaN that was added stays: r is finite, so that no other value gives one.
struct FusedExpSums {
    float m, r;
    unsigned long long s[2];
    __device__ __forceinline__ FusedExpSums() : m(kLowest), r(kLowest), s{0ull, 0ull} {}
    static __device__ __forceinline__ float nan_or_zero(float x) { return x != x ? x : 0.f; }
    __device__ __forceinline__ void raise(float top, float c, float slack) {
        if (top > m + slack) {
            const float now = fminf(fmaxf(top * c, kLowest), -kLowest), f = exp2_fast(r - now);
            const bool far = is_far(m, c);                 // (the sum may be anything)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float2 p = halves(s[i]);
                s[i] = far ? pair_of(nan_or_zero(p.x), nan_or_zero(p.y)) : mul_pairs(s[i], pair_of(f, f));
            }
            m = top; r = now;
        }
    }
    template <int N> __device__ __forceinline__ void add(const float (&x)[N], float c) {
        const unsigned long long minus_r = pair_of(-r, -r), cc = pair_of(c, c);
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float2 y = halves(fma_pairs(pair_of(x[i], x[i + 1]), cc, minus_r));
            s[i / 2 & 1] = add_pairs(s[i / 2 & 1], pair_of(exp2_fast(y.x), exp2_fast(y.y)));
        }
    }
    __device__ __forceinline__ ExpSum whole(float c) const {
        const float2 p = halves(add_pairs(s[0], s[1]));
        ExpSum e;
        e.m = m;
        e.s = is_far(m, c) ? nan_or_zero(p.x + p.y) : (p.x + p.y) * exp2_fast(-__fmaf_rn(m, c, -r));
        return e;
    }
};

// 40 powers of two, in logits (bounded: m + slack has to stay below any value when m is the lowest)
__host__ __device__ __forceinline__ float exp_slack(float c) { return fminf(40.f / c, 1e30f); }

// (as integers that ascend with the values; NaN must not be among them)
__device__ __forceinline__ float warp_max(float v) {
    int b = __float_as_int(v);
    b = __reduce_max_sync(kFullMask, b ^ (b >> 31 & 0x7FFFFFFF));
    return __int_as_float(b ^ (b >> 31 & 0x7FFFFFFF));
}
template <class F> __device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFullMask, v, o);
    return v;
}
__device__ __forceinline__ ExpSum warp_join(ExpSum e, float c) {
    const float top = warp_max(e.m);
    e.s = warp_sum(e.s * exp2_fast((e.m - top) * c));
    e.m = top;
    return e;
}

// Block-wide, the result in every thread; `s` holds a value per warp and is free again once the next barrier has passed.
template <int WARPS, class F> __device__ __forceinline__ F block_sum(F v, F* s) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_sum(lane < WARPS ? s[lane] : (F)0);
}

}  // namespace fsg
