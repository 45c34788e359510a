// Token caches: each head's query and key normed and rotated by its token's position, in one pass, which in its
// second form also writes the keys (and the values) into their cells.
//
//   y = x w / sqrt(mean(x^2) + eps);  a pair (a, b) of y's first values -> (a cos u - b sin u, b cos u + a sin u)
//
// with u the position along the pair's axis times the pair's frequency.  The angle is held as a part of a turn in
// 64-bit fixed point: the position times (frequency / 2 pi) 2^64, modulo 2^64, is exact to position 2^-64 turns, so
// a token at position 2^30 is rotated as well as one at 5, and only the remainder goes to sine and cosine in fp32.
// A row lies with a power-of-two group of a warp, eight values a thread: with pairs of halves four from either half, so
// that a pair never leaves its thread, the row's sum of squares is a few shuffles away, and an e4m3 row is quantised in
// the pass that rotated it.  A group takes a token and some or all of its heads: its sines and cosines, times the
// weights, stay in registers from head to head.  A block takes a tile of up to 16 tokens of one sequence.
// Everything is fp32 up to one rounding to the activations' type; codes are made from that rounding, so that both ways to
// a cell store the same bits.
#include <type_traits>

#include "tokens_util.cuh"

namespace mure {

namespace {

constexpr int kThreads = 128;
constexpr int kRows = 4;         // rows that a thread has on their way
constexpr int kBlocks = 16;      // blocks per SM that a launch has at least, where it has the rows

struct RotateParams {
    TokPool pool;
    TokBatch b;
    TokRotary r;
    TokRows q, k, v, q_out, k_out;
    int q_heads, k_heads;
    int lanes;                   // threads per row
};

enum { kToRows = 0, kToCells = 1, kToCodes = 2 };

// A thread's eight values of a row as they lie in memory: two runs of four, or (ONE) one of eight.
template <class T, bool ONE>
struct Eight {
    static constexpr int kWords = sizeof(T) * 2;                     // 32-bit words
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T *p, int second, int vec)
    {
        if (vec) {
            if (ONE) {
#pragma unroll
                for (int i = 0; i < kWords / 4; ++i)
                    reinterpret_cast<uint4 *>(w)[i] = reinterpret_cast<const uint4 *>(p)[i];
            } else if (sizeof(T) == 4) {
                reinterpret_cast<uint4 *>(w)[0] = *reinterpret_cast<const uint4 *>(p);
                reinterpret_cast<uint4 *>(w)[kWords / 4 - 1] = *reinterpret_cast<const uint4 *>(p + second);
            } else {
                reinterpret_cast<uint2 *>(w)[0] = *reinterpret_cast<const uint2 *>(p);
                reinterpret_cast<uint2 *>(w)[1] = *reinterpret_cast<const uint2 *>(p + second);
            }
        } else {
            T *t = reinterpret_cast<T *>(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = p[i < 4 ? i : second + i - 4];
        }
    }
    __device__ __forceinline__ void store(T *p, int second, int vec) const
    {
        if (vec) {
            if (ONE) {
#pragma unroll
                for (int i = 0; i < kWords / 4; ++i)
                    reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(w)[i];
            } else if (sizeof(T) == 4) {
                *reinterpret_cast<uint4 *>(p) = reinterpret_cast<const uint4 *>(w)[0];
                *reinterpret_cast<uint4 *>(p + second) = reinterpret_cast<const uint4 *>(w)[kWords / 4 - 1];
            } else {
                *reinterpret_cast<uint2 *>(p) = reinterpret_cast<const uint2 *>(w)[0];
                *reinterpret_cast<uint2 *>(p + second) = reinterpret_cast<const uint2 *>(w)[1];
            }
        } else {
            const T *t = reinterpret_cast<const T *>(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i < 4 ? i : second + i - 4] = t[i];
        }
    }
    __device__ __forceinline__ void up(float *x) const
    {
        const T *t = reinterpret_cast<const T *>(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = TokType<T>::up(t[i]);
    }
    __device__ __forceinline__ void down(const float *x)
    {
        T *t = reinterpret_cast<T *>(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = TokType<T>::down(x[i]);
    }
    // the bits of the largest magnitude, as fp32
    __device__ __forceinline__ uint32_t most() const
    {
        uint32_t a = 0;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) a = __vmaxu2(a, w[i] & 0x7FFF7FFFu);
            return max(a & 0xFFFFu, a >> 16);
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) a = max(a, w[i] & 0x7FFFFFFFu);
            return a;
        }
    }
    static __device__ __forceinline__ uint32_t bits_up(uint32_t a)
    {
        if constexpr (sizeof(T) == 4) return a;
        const uint16_t h = (uint16_t)a;
        return __float_as_uint(TokType<T>::up(*reinterpret_cast<const T *>(&h)));
    }
};

template <class T, int TO, bool ADJ>
__global__ void __launch_bounds__(kThreads, 5) k_tokens_rotate(RotateParams p)
{
    using X = Eight<T, ADJ>;
    TokSeq sq;
    const Tile t = tile_of(p.b, false, sq);
    const int D = p.pool.d, slot = threadIdx.x & (p.lanes - 1), group = threadIdx.x / p.lanes, groups = kThreads / p.lanes;
    const bool in = slot * 8 < D, turned = slot * 8 < p.r.rot;
    // this thread's values of a row: two runs of four; with pairs of halves the rotated ones lie half a rotation apart
    const int half = p.r.rot / 2, at = !ADJ && turned ? slot * 4 : slot * 8, second = !ADJ && turned ? half : 4;
    const float over = 1.f / D;
    // the block's groups over the tile's tokens: of fewer tokens than groups each has several, which share its heads
    const int share = t.n < groups ? groups / t.n : 1;
    const int parts = share * gridDim.y, part = blockIdx.y * share + group % share;
    const int32_t *table = p.b.table + sq.table0;

    for (int i0 = 0; i0 < t.n; i0 += groups / share) {
        const int i = i0 + group / share;
        const bool here = in && i < t.n;
        const int64_t token = sq.row0 + t.i0 + i;
        float cosine[4] = {1.f, 1.f, 1.f, 1.f}, sine[4] = {0.f, 0.f, 0.f, 0.f};
        if (here && turned) {
            const int own = p.r.positions ? 0 : sq.pos + (p.b.node ? __ldg(&p.b.node[token].depth) : t.i0 + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int k = slot * 4 + e;
                const int pos = p.r.positions ? __ldg(p.r.positions + __ldg(p.r.axis + k) * p.r.position_stride + token) : own;
                const uint64_t turn = (uint64_t)(int64_t)pos * __ldg(p.r.turn + k);
                // to the nearest 2^-32 of a turn, in -1/2 .. 1/2
                const float u = (float)(int32_t)(uint32_t)((turn + 0x80000000ull) >> 32) * 0x1p-31f;
                sincospif(u, sine + e, cosine + e);
            }
        }
        // KIND 0: queries, 1: keys, 2: values
        auto rows = [&](auto kind, const TokRows &from, const TokRows &to, int heads) {
            constexpr int KIND = decltype(kind)::value;
            constexpr bool kCells = KIND > 0 && TO != kToRows, kCodes = KIND > 0 && TO == kToCodes;
            const bool norm = KIND == 0 ? p.r.norm_q : KIND == 1 && p.r.norm_k;
            // x -> (a cw - b sw', b cw' + a sw): each pair's cosine and sine times its weights
            float w[8], ca[4], sb[4], cb[4], sa[4];
            if (KIND < 2) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    w[e] = norm && here ? __ldg(p.r.weight + (KIND == 0 ? 0 : D) + at + (e < 4 ? e : second + e - 4)) : 1.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float wa = w[ADJ ? 2 * e : e], wb = w[ADJ ? 2 * e + 1 : e + 4];
                    ca[e] = cosine[e] * wa; sa[e] = sine[e] * wa;
                    cb[e] = cosine[e] * wb; sb[e] = sine[e] * wb;
                }
            }
            const T *src = reinterpret_cast<const T *>(from.p) + token * from.ts + at;
            T *dst = kCells ? nullptr : reinterpret_cast<T *>(to.p) + token * to.ts + at;
            for (int h0 = part; h0 - part < heads; h0 += parts * kRows) {
                X x[kRows];
#pragma unroll
                for (int u = 0; u < kRows; ++u) {
                    const int h = h0 + u * parts;
#pragma unroll
                    for (int e = 0; e < X::kWords; ++e) x[u].w[e] = 0u;
                    if (here && h < heads) x[u].load(src + h * from.hs, second, from.vec);
                }
#pragma unroll
                for (int u = 0; u < kRows; ++u) {
                    const int h = h0 + u * parts;
                    if (h - part >= heads) break;                    // (for all threads alike)
                    const bool on = here && h < heads;
                    float y[8];
                    if (KIND < 2) {
                        x[u].up(y);
                        float f = 1.f;
                        if (norm) {
                            float sum = 0.f;
#pragma unroll
                            for (int e = 0; e < 8; ++e) sum = fmaf(y[e], y[e], sum);
                            for (int s = p.lanes >> 1; s; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
                            f = rsqrtf(fmaf(sum, over, p.r.eps));
                            // squares that leave fp32's range: once more, of the values times a power of two
                            const bool lost = on && !(sum >= 0x1p-80f && sum < INFINITY);
                            if (__any_sync(0xffffffffu, lost)) {
                                const float g = sum < 1.f ? 0x1p60f : 0x1p-70f;
                                float again = 0.f;
#pragma unroll
                                for (int e = 0; e < 8; ++e) again = fmaf(y[e] * g, y[e] * g, again);
                                for (int s = p.lanes >> 1; s; s >>= 1) again += __shfl_xor_sync(0xffffffffu, again, s);
                                if (lost) f = rsqrtf(fmaf(again, over, p.r.eps * g * g)) * g;
                            }
#pragma unroll
                            for (int e = 0; e < 8; ++e) y[e] *= f;
                        }
                        if (turned) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                float &a = y[ADJ ? 2 * e : e], &b = y[ADJ ? 2 * e + 1 : e + 4];
                                const float t0 = fmaf(a, ca[e], -b * sb[e]), t1 = fmaf(b, cb[e], a * sa[e]);
                                a = t0;
                                b = t1;
                            }
                        } else if (norm) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) y[e] *= w[e];
                        }
                        x[u].down(y);                                // the one rounding to the activations' type
                    }
                    if (!kCells) {
                        if (on) x[u].store(dst + h * to.hs, second, to.vec);
                    } else {
                        void *pool = KIND == 2 ? p.pool.v : p.pool.k;
                        const int64_t row = on ? cell_row(p.pool, table, h, sq.pos + t.i0 + i) : 0;
                        if (!kCodes) {
                            if (on) x[u].store(static_cast<T *>(pool) + row * D + at, second, 1);
                        } else {
                            uint32_t most = x[u].most();
                            for (int s = p.lanes >> 1; s; s >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, s));
                            const uint32_t byte = scale_byte(X::bits_up(most));
                            if (on) {
                                x[u].up(y);
                                uint32_t c[2];
#pragma unroll
                                for (int e = 0; e < 2; ++e)
                                    c[e] = byte == 255u ? 0u
                                                        : e4m3_pair(unscale(y[4 * e], byte), unscale(y[4 * e + 1], byte)) |
                                                              e4m3_pair(unscale(y[4 * e + 2], byte), unscale(y[4 * e + 3], byte)) << 16;
                                uint8_t *o = static_cast<uint8_t *>(pool) + row * D + at;
                                if (ADJ) *reinterpret_cast<uint2 *>(o) = make_uint2(c[0], c[1]);
                                else {
                                    *reinterpret_cast<uint32_t *>(o) = c[0];
                                    *reinterpret_cast<uint32_t *>(o + second) = c[1];
                                }
                                if (slot == 0) (KIND == 2 ? p.pool.vs : p.pool.ks)[row] = (uint8_t)byte;
                            }
                        }
                    }
                }
            }
        };
        rows(std::integral_constant<int, 0>{}, p.q, p.q_out, p.q_heads);
        rows(std::integral_constant<int, 1>{}, p.k, p.k_out, p.k_heads);
        if (TO != kToRows) rows(std::integral_constant<int, 2>{}, p.v, p.v, p.k_heads);
    }
}

template <class T, int TO, bool ADJ>
int go(const RotateParams &p, int64_t tiles, cudaStream_t s)
{
    // several blocks share a tile until there are enough of them, down to one row of queries each
    const int groups = kThreads / p.lanes, heads = p.q_heads > p.k_heads ? p.q_heads : p.k_heads;
    const int64_t want = (kBlocks * (int64_t)sm_count() + tiles - 1) / tiles, most = (heads + groups - 1) / groups;
    k_tokens_rotate<T, TO, ADJ><<<dim3((unsigned)tiles, (unsigned)(want < most ? want : most)), kThreads, 0, s>>>(p);
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
    if (tiles == 0 || q_heads + k_heads == 0) return 0;
    const RotateParams p{pool, b, r, q, k, v, q_out, k_out, q_heads, k_heads, row_lanes(pool.d)};
    const int to = !cells ? kToRows : form == MURE_FORM_E4M3 ? kToCodes : kToCells;
    if (dtype == MURE_F32) return by_target<float>(p, to, tiles, s);
    if (dtype == MURE_F16) return by_target<__half>(p, to, tiles, s);
    return by_target<__nv_bfloat16>(p, to, tiles, s);
}

}  // namespace mure
