// Device helpers of the token-cache kernels: types, e4m3 codes, masks, and one row of
// attention by the definition.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "tokens.cuh"

namespace mure {

template <class T> struct TokType;
template <> struct TokType<float> {
    static __device__ __forceinline__ float up(float x) { return x; }
    static __device__ __forceinline__ float down(float x) { return x; }
};
template <> struct TokType<__half> {
    static __device__ __forceinline__ float up(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half down(float x) { return __float2half_rn(x); }
};
template <> struct TokType<__nv_bfloat16> {
    static __device__ __forceinline__ float up(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 down(float x) { return __float2bfloat16_rn(x); }
};

// 2^(byte - 127); byte 255 stands for NaN.  (Byte 0 is 2^-127, a subnormal.)
__device__ __forceinline__ float scale_of(uint32_t byte)
{
    return __uint_as_float(byte == 255u ? 0x7FFFFFFFu : byte == 0u ? 0x00400000u : byte << 23);
}

// The scale byte of a row whose largest magnitude has the bits `amax` (non-negative):
// a = m 2^k with m in [1, 2); 448 = 1.75 * 2^8, so the least e with a 2^-e <= 448 is k - 8, or
// k - 7 where m > 1.75.  Subnormals and zero fall under the least byte.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax)
{
    if (amax >= 0x7F800000u) return 255u;
    const int e = (int)(amax >> 23) - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, 0);
}

// x / scale, exact unless it leaves the normal numbers far below the codes: x * 2^(127 - byte), byte <= 247.
__device__ __forceinline__ float unscale(float x, uint32_t byte) { return x * __uint_as_float((254u - byte) << 23); }

// 2^x by the hardware's approximation (2 units in the last place; results below 2^-126 are 0).
__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ float2 e4m3_values(uint16_t two)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
    return __half22float2(*reinterpret_cast<__half2 *>(&h));
}

// Eight values of a row of T, as fp32, and back.
template <class T>
__device__ __forceinline__ void load8(const T *p, int vec, float *x)
{
    if (vec) {
        alignas(16) T t[8];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(t)[i] = reinterpret_cast<const uint4 *>(p)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = TokType<T>::up(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = TokType<T>::up(p[i]);
    }
}

template <class T>
__device__ __forceinline__ void store8(T *p, int vec, const float *x)
{
    if (vec) {
        alignas(16) T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = TokType<T>::down(x[i]);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(t)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = TokType<T>::down(x[i]);
    }
}

// Eight values of a cell's row at element offset `off` of a pool.
template <class T, bool E4M3>
__device__ __forceinline__ void cell8(const void *pool, const uint8_t *scales, int64_t row, int d, int c, float *x)
{
    if (E4M3) {
        const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(pool) + row * d + c);
        const float s = scale_of(scales[row]);
        const uint32_t u[2] = {w.x, w.y};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = e4m3_values((uint16_t)(u[i >> 1] >> (16 * (i & 1))));
            x[2 * i] = f.x * s;
            x[2 * i + 1] = f.y * s;
        }
    } else {
        load8(static_cast<const T *>(pool) + row * d + c, 1, x);
    }
}

// Row index of cell j of sequence b for cached head h.
__device__ __forceinline__ int64_t cell_row(const TokPool &p, const int32_t *table, int h, int j)
{
    const int64_t page = __ldg(table + (j >> p.page_log2));
    return ((page * p.hk + h) << p.page_log2) | (j & ((1 << p.page_log2) - 1));
}

// The entry k of an ascending prefix array with prefix[k] <= x < prefix[k + 1], by a whole warp
// (32 probes a step: two dependent loads for up to 1,024 entries).
__device__ __forceinline__ int find_prefix(const int32_t *prefix, int n, int x)
{
    int lo = 0, len = n;                         // the answer lies in [lo, lo + len)
    const int lane = threadIdx.x & 31;
    while (len > 1) {
        const int step = (len + 31) / 32;
        const int at = lo + lane * step;
        const bool le = at < lo + len && __ldg(prefix + at) <= x;
        const int k = 31 - __clz(__ballot_sync(0xffffffffu, le));
        len = min(step, lo + len - (lo + k * step));
        lo += k * step;
    }
    return lo;
}

// Whether the cell j may be attended to from position p (j < the cells held is the caller's).
__device__ __forceinline__ bool tok_seen(int j, int p, int window, int sinks)
{
    return j <= p && (window == 0 || j > p - window || j < sinks);
}

// One row of attention by the definition, by a whole warp, over the cells j0 .. j1 - 1: only cells
// that the row may attend to are read.  q: the row's D values (any memory); the warp's lanes
// below D / 8 hold eight output sums each in o (not divided), all lanes the maximum m of
// scale_log2 q k (-inf: no cell) and the sum l of 2^(. - m).
template <class T, bool E4M3>
__device__ __forceinline__ void attend_row(const TokPool &pool, const int32_t *table, int h, const T *q, int qvec, int p,
                                           int j0, int j1, int window, int sinks, float scale_log2, float *o, float &m,
                                           float &l)
{
    const int lane = threadIdx.x & 31, D = pool.d;
    // half of a small scale's power of two goes to q (exactly), so that a sum of products cannot overflow where
    // the score does not
    const int half = min((int)(__float_as_uint(scale_log2) >> 23) - 127, 0) / 2;
    const float before = __uint_as_float((uint32_t)(127 + half) << 23), after = scale_log2 * __uint_as_float((uint32_t)(127 - half) << 23);
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = 0.f;
    j1 = min(j1, p + 1);
    for (int base = j0; base < j1; base += 32) {
        if (window && base + 31 <= p - window && base >= sinks) {      // wholly before the window
            const int first = p - window + 1;
            base += (first - base) / 32 * 32 - 32;
            if (base + 32 >= j1) break;
            continue;
        }
        const int j = base + lane;
        const bool see = j < j1 && tok_seen(j, p, window, sinks);
        float s = 0.f;
        if (see) {
            const int64_t row = cell_row(pool, table, h, j);
            for (int c = 0; c < D; c += 8) {
                float a[8], b[8];
                cell8<T, E4M3>(pool.k, pool.ks, row, D, c, a);
                load8(q + c, qvec, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(a[i], b[i] * before, s);
            }
            s *= after;
        }
        float top = see ? s : -INFINITY;
        bool bad = see && isnan(s);
#pragma unroll
        for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        bad = __any_sync(0xffffffffu, bad);
        const float mn = bad ? NAN : (isnan(m) ? m : fmaxf(m, top));
        const float ref = mn == -INFINITY ? 0.f : mn;
        const float keep = exp2f(m - ref);                              // m = -inf: 0
        const float pr = see ? exp2f(s - ref) : 0.f;
        float sum = pr;
#pragma unroll
        for (int x = 16; x; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
        l = l * keep + sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] *= keep;
        m = mn;
        uint32_t seen = __ballot_sync(0xffffffffu, see);
        while (seen) {
            const int k = __ffs(seen) - 1;
            seen &= seen - 1;
            const float pk = __shfl_sync(0xffffffffu, pr, k);
            const int64_t row = cell_row(pool, table, h, base + k);
            if (lane * 8 < D) {
                float a[8];
                cell8<T, E4M3>(pool.v, pool.vs, row, D, lane * 8, a);
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = fmaf(pk, a[i], o[i]);
            }
        }
    }
}

}  // namespace mure
