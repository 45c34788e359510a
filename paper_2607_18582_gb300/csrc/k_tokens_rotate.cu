// Token caches: each head's query and key normed and rotated by its token's position, in one pass, which in its
// second form also writes the keys (and the values) into their cells.
//
//   y = x w / sqrt(mean(x^2) + eps);  a pair (a, b) of y's first values -> (a cos u - b sin u, b cos u + a sin u)
//
// with u the position along the pair's axis times the pair's frequency.  The angle is held as a part of a turn in
// 64-bit fixed point: the position times (frequency / 2 pi) 2^64, modulo 2^64, is exact to position 2^-64 turns, so
// a token at position 2^30 is rotated as well as one at 5, and only the remainder goes to sine and cosine in fp32.
// A block takes a tile of up to 16 tokens of one sequence, computes its sines and cosines once into shared memory
// and all heads' rows from them.  A row lies with a power-of-two group of a warp, eight values a thread: with pairs
// of halves four from either half, so that a pair never leaves its thread, the row's sum of squares is a few shuffles
// away, and an e4m3 row is quantised in the pass that rotated it.  Everything is fp32 up to one rounding to the
// activations' type; codes are made from that rounding, so that both ways to a cell store the same bits.
#include "tokens_util.cuh"

namespace mure {

namespace {

constexpr int kThreads = 128;
constexpr int kRows = 4;         // rows that a thread has on their way

struct RotateParams {
    TokPool pool;
    TokBatch b;
    TokRotary r;
    TokRows q, k, v, q_out, k_out;
    int q_heads, k_heads, rows;  // of a token: its query, key and (into cells) value rows
    int lanes;                   // threads per row
};

enum { kToRows = 0, kToCells = 1, kToCodes = 2 };

// Four values as they lie in memory, and in fp32.
template <class T> struct Quad;
template <> struct Quad<float> {
    uint4 w;
    __device__ __forceinline__ void up(float *x) const
    {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
    __device__ __forceinline__ void down(const float *x)
    {
        w = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __device__ __forceinline__ void load(const float *p, int vec)
    {
        if (vec) w = *reinterpret_cast<const uint4 *>(p);
        else down(p);
    }
    __device__ __forceinline__ void store(float *p, int vec) const
    {
        if (vec) *reinterpret_cast<uint4 *>(p) = w;
        else up(p);
    }
};
template <class T> struct Quad {
    uint2 w;
    __device__ __forceinline__ void up(float *x) const
    {
        const T *t = reinterpret_cast<const T *>(&w);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = TokType<T>::up(t[i]);
    }
    __device__ __forceinline__ void down(const float *x)
    {
        T *t = reinterpret_cast<T *>(&w);
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = TokType<T>::down(x[i]);
    }
    __device__ __forceinline__ void load(const T *p, int vec)
    {
        if (vec) w = *reinterpret_cast<const uint2 *>(p);
        else {
            T *t = reinterpret_cast<T *>(&w);
#pragma unroll
            for (int i = 0; i < 4; ++i) t[i] = p[i];
        }
    }
    __device__ __forceinline__ void store(T *p, int vec) const
    {
        if (vec) *reinterpret_cast<uint2 *>(p) = w;
        else {
            const T *t = reinterpret_cast<const T *>(&w);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = t[i];
        }
    }
};

template <class T, int TO, bool ADJ>
__global__ void __launch_bounds__(kThreads) k_tokens_rotate(RotateParams p)
{
    extern __shared__ __align__(16) float shared[];
    TokSeq sq;
    const Tile t = tile_of(p.b, false, sq);
    const int D = p.pool.d, half = p.r.rot / 2;
    float *cosine = shared, *sine = shared + kTokTile * half, *weight = shared + 2 * kTokTile * half;
    for (int u = threadIdx.x; u < t.n * half; u += kThreads) {
        const int i = u / half, k = u - i * half;
        const int64_t token = sq.row0 + t.i0 + i;
        const int at = p.r.positions ? __ldg(p.r.positions + __ldg(p.r.axis + k) * p.r.position_stride + token)
                                     : sq.pos + (p.b.node ? __ldg(&p.b.node[token].depth) : t.i0 + i);
        const uint64_t turn = (uint64_t)(int64_t)at * __ldg(p.r.turn + k);
        // to the nearest 2^-32 of a turn, in -1/2 .. 1/2
        const float part = (float)(int32_t)(uint32_t)((turn + 0x80000000ull) >> 32) * 0x1p-31f;
        sincospif(part, sine + u, cosine + u);
    }
    for (int u = threadIdx.x; u < 2 * D; u += kThreads) weight[u] = __ldg(p.r.weight + u);
    __syncthreads();

    const int slot = threadIdx.x & (p.lanes - 1), per = kThreads / p.lanes;
    const bool in = slot * 8 < D, turned = slot * 8 < p.r.rot;
    // this thread's values of a row: two runs of four; with pairs of halves the rotated ones lie half a rotation apart
    const int ia = !ADJ && turned ? slot * 4 : slot * 8, ib = !ADJ && turned ? half + slot * 4 : slot * 8 + 4;
    const int all = t.n * p.rows, step = per * gridDim.y, step_i = step / p.rows, step_h = step - step_i * p.rows;
    const int32_t *table = p.b.table + sq.table0;
    int r = blockIdx.y * per + threadIdx.x / p.lanes;
    int i = r / p.rows, h = r - i * p.rows;
    const float over = 1.f / D;
    for (int base = blockIdx.y * per; base < all; base += step * kRows) {
        Quad<T> a[kRows], b[kRows];
        int ri[kRows], rh[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            ri[u] = r < all && in ? i : -1;
            rh[u] = h;
            a[u] = b[u] = Quad<T>{};
            if (ri[u] >= 0) {
                const TokRows &from = h < p.q_heads ? p.q : h < p.q_heads + p.k_heads ? p.k : p.v;
                const int head = h < p.q_heads ? h : h < p.q_heads + p.k_heads ? h - p.q_heads : h - p.q_heads - p.k_heads;
                const T *x = reinterpret_cast<const T *>(from.p) + (int64_t)(sq.row0 + t.i0 + i) * from.ts + head * from.hs;
                a[u].load(x + ia, from.vec);
                b[u].load(x + ib, from.vec);
            }
            r += step;
            i += step_i;
            h += step_h;
            if (h >= p.rows) { h -= p.rows; ++i; }
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            if (base + u * step >= all) break;                       // (for all threads alike)
            const bool on = ri[u] >= 0, is_q = rh[u] < p.q_heads, is_v = TO != kToRows && rh[u] >= p.q_heads + p.k_heads;
            float y[8];
            a[u].up(y);
            b[u].up(y + 4);
            if (p.r.norm_q || p.r.norm_k) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(y[e], y[e], sum);
                for (int x = p.lanes >> 1; x; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
                float f = rsqrtf(fmaf(sum, over, p.r.eps));
                // squares that leave fp32's range: once more, of the values times a power of two
                const bool lost = !(sum >= 0x1p-80f && sum < INFINITY);
                if (__any_sync(0xffffffffu, lost)) {
                    const float g = sum < 1.f ? 0x1p60f : 0x1p-70f;
                    float again = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) again = fmaf(y[e] * g, y[e] * g, again);
                    for (int x = p.lanes >> 1; x; x >>= 1) again += __shfl_xor_sync(0xffffffffu, again, x);
                    if (lost) f = rsqrtf(fmaf(again, over, p.r.eps * g * g)) * g;
                }
                if (is_q ? p.r.norm_q : !is_v && p.r.norm_k) {
                    const float4 wa = *reinterpret_cast<const float4 *>(weight + (is_q ? 0 : D) + (in ? ia : 0));
                    const float4 wb = *reinterpret_cast<const float4 *>(weight + (is_q ? 0 : D) + (in ? ib : 0));
                    y[0] *= f * wa.x; y[1] *= f * wa.y; y[2] *= f * wa.z; y[3] *= f * wa.w;
                    y[4] *= f * wb.x; y[5] *= f * wb.y; y[6] *= f * wb.z; y[7] *= f * wb.w;
                }
            }
            if (turned && !is_v && on) {
                const float4 c = *reinterpret_cast<const float4 *>(cosine + ri[u] * half + slot * 4);
                const float4 s = *reinterpret_cast<const float4 *>(sine + ri[u] * half + slot * 4);
                auto pair = [&](float &x0, float &x1, float cu, float su) {
                    const float t0 = fmaf(x0, cu, -x1 * su), t1 = fmaf(x1, cu, x0 * su);
                    x0 = t0;
                    x1 = t1;
                };
                if (ADJ) {
                    pair(y[0], y[1], c.x, s.x); pair(y[2], y[3], c.y, s.y);
                    pair(y[4], y[5], c.z, s.z); pair(y[6], y[7], c.w, s.w);
                } else {
                    pair(y[0], y[4], c.x, s.x); pair(y[1], y[5], c.y, s.y);
                    pair(y[2], y[6], c.z, s.z); pair(y[3], y[7], c.w, s.w);
                }
            }
            if (!is_v) {                                             // the one rounding to the activations' type
                a[u].down(y);
                b[u].down(y + 4);
            }
            const int token = sq.row0 + t.i0 + ri[u];
            if (TO == kToRows || is_q) {
                if (on) {
                    const TokRows &to = is_q ? p.q_out : p.k_out;
                    T *o = reinterpret_cast<T *>(to.p) + (int64_t)token * to.ts + (is_q ? rh[u] : rh[u] - p.q_heads) * to.hs;
                    a[u].store(o + ia, to.vec);
                    b[u].store(o + ib, to.vec);
                }
            }
            if (TO == kToRows) continue;
            const int head = rh[u] - p.q_heads - (is_v ? p.k_heads : 0);
            void *pool = is_v ? p.pool.v : p.pool.k;
            if (TO == kToCells) {
                if (on && !is_q) {
                    T *o = static_cast<T *>(pool) + cell_row(p.pool, table, head, sq.pos + t.i0 + ri[u]) * D;
                    a[u].store(o + ia, 1);
                    b[u].store(o + ib, 1);
                }
            } else if (__any_sync(0xffffffffu, on && !is_q)) {
                uint32_t most = 0;
                a[u].up(y);
                b[u].up(y + 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(y[e]) & 0x7FFFFFFFu);
                for (int x = p.lanes >> 1; x; x >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, x));
                const uint32_t byte = scale_byte(most);
                if (on && !is_q) {
                    const int64_t row = cell_row(p.pool, table, head, sq.pos + t.i0 + ri[u]);
                    uint32_t w[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        w[e] = byte == 255u ? 0u
                                            : e4m3_pair(unscale(y[4 * e], byte), unscale(y[4 * e + 1], byte)) |
                                                  e4m3_pair(unscale(y[4 * e + 2], byte), unscale(y[4 * e + 3], byte)) << 16;
                    uint8_t *o = static_cast<uint8_t *>(pool) + row * D;
                    *reinterpret_cast<uint32_t *>(o + ia) = w[0];
                    *reinterpret_cast<uint32_t *>(o + ib) = w[1];
                    if (slot == 0) (is_v ? p.pool.vs : p.pool.ks)[row] = (uint8_t)byte;
                }
            }
        }
    }
}

template <class T, int TO, bool ADJ>
int go(const RotateParams &p, int64_t tiles, cudaStream_t s)
{
    // where tiles are few, several blocks share one: down to one step of rows each
    const int per = kThreads / p.lanes, most = (p.rows + per - 1) / per;
    const int64_t want = (4 * (int64_t)sm_count() + tiles - 1) / tiles;
    const unsigned y = (unsigned)(want < most ? want : most);
    const size_t bytes = ((size_t)kTokTile * p.r.rot + 2 * p.pool.d) * sizeof(float);
    k_tokens_rotate<T, TO, ADJ><<<dim3((unsigned)tiles, y), kThreads, bytes, s>>>(p);
    return 1;
}

template <class T>
int by_target(const RotateParams &p, int to, int64_t tiles, cudaStream_t s)
{
    const bool adj = p.r.adjacent != 0;
    if (to == kToRows) return adj ? go<T, kToRows, true>(p, tiles, s) : go<T, kToRows, false>(p, tiles, s);
    if (to == kToCells) return adj ? go<T, kToCells, true>(p, tiles, s) : go<T, kToCells, false>(p, tiles, s);
    return adj ? go<T, kToCodes, true>(p, tiles, s) : go<T, kToCodes, false>(p, tiles, s);
}

}  // namespace

int launch_tokens_rotate(const TokPool &pool, const TokBatch &b, const TokRotary &r, int dtype, int form, bool cells, int q_heads,
                         int k_heads, TokRows q, TokRows k, TokRows v, TokRows q_out, TokRows k_out, int64_t tiles, cudaStream_t s)
{
    const int rows = q_heads + k_heads * (cells ? 2 : 1);
    if (tiles == 0 || rows == 0) return 0;
    const RotateParams p{pool, b, r, q, k, v, q_out, k_out, q_heads, k_heads, rows, row_lanes(pool.d)};
    const int to = !cells ? kToRows : form == MURE_FORM_E4M3 ? kToCodes : kToCells;
    if (dtype == MURE_F32) return by_target<float>(p, to, tiles, s);
    if (dtype == MURE_F16) return by_target<__half>(p, to, tiles, s);
    return by_target<__nv_bfloat16>(p, to, tiles, s);
}

}  // namespace mure
