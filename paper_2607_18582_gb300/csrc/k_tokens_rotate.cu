// Token caches: each head's query and key normed and rotated by its token's position, in one pass, which in its
// second form also writes the keys (and the values) into their cells.
//
//   y = x w / sqrt(mean(x^2) + eps);  a pair (a, b) of y's first values -> (a cos u - b sin u, b cos u + a sin u)
//
// with u the position along the pair's axis times the pair's frequency.  The angle is held as a part of a turn in
// 64-bit fixed point: the position times (frequency / 2 pi) 2^64, modulo 2^64, is exact to position 2^-64 turns, so
// a token at position 2^30 is rotated as well as one at 5, and only the remainder goes to sine and cosine, in fp32 and what that leaves.
// A row lies with a power-of-two group of a warp, 16 (or eight) values a thread: with pairs of halves half of them from either half, so
// that a pair never leaves its thread, the row's sum of squares is a few shuffles away, and an e4m3 row is quantised in
// the pass that rotated it.  A group takes a token and some or all of its heads: its sines and cosines, times the
// weights, stay in registers from head to head.  A block takes a tile of up to 16 tokens of one sequence.
// A thread's rows are copied ahead through shared memory, where only it reads them, so that no barrier is needed and
// registers hold one row at a time.  Everything is fp32 up to one rounding to the activations' type; codes are made from that rounding, so that both ways to
// a cell store the same bits.
//
// Measured (GB300): 57,000 tokens of 32 and 8 heads of 128 bf16 values, normed and rotated, keys and values into e4m3 cells:
// 216 to 220 us, 5.9 TB/s of what it has to move, issue slots 62 % busy at 3.8 warps per scheduler.
// 28,000 tokens of 16 heads of 80 f16 values, neighbouring pairs, positions along three axes, no norm: 61 us, 4.7 TB/s:
// latency and issue, a group has one token and five of its eight lanes a part of the row.  (Groups of as many lanes as a row
// needs: as fast, but 216 -> 236 us with the sums over five lanes; eight values a thread 364 and 82 us.)  What small
// angles and rows of subnormal numbers cost is in these figures: 218 -> 220 us on one card.
#include <type_traits>

#include "simt_tile.cuh"
#include "tokens_util.cuh"

namespace mure {

namespace {

constexpr int kThreads = 128;
constexpr int kAhead = 3;        // batches of rows on their way
constexpr int kBlocks = 4;        // per SM that run at a time

struct RotateParams {
    TokPool pool;
    TokBatch b;
    TokRotary r;
    TokRows q, k, v, q_out, k_out;
    int q_heads, k_heads;
    int lanes;                   // threads per row
    int64_t tokens;
};

enum { kToRows = 0, kToCells = 1, kToCodes = 2 };

// A thread's N values of a row as they lie in memory, two runs of N / 2.
template <class T, int N>
struct Part {
    static constexpr int kWords = N * (int)sizeof(T) / 4;            // 32-bit words
    static constexpr int kRun = N / 2;
    uint32_t w[kWords];
    // a piece of it that one copy brings: 16 bytes, or a run of 8
    static constexpr int kPiece = kRun * sizeof(T) < 16 ? 8 : 16, kPieces = N * (int)sizeof(T) / kPiece;
    static constexpr int kPer = kPiece / (int)sizeof(T), kRunPieces = kPieces / 2;
    using Piece = typename std::conditional<kPiece == 8, uint2, uint4>::type;
    __device__ __forceinline__ void piece(int i, Piece v) { reinterpret_cast<Piece *>(w)[i] = v; }
    __device__ __forceinline__ void store(T *p, int second, int vec) const
    {
        if (vec) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                T *q = p + (r ? second : 0);
                if constexpr (kRun * sizeof(T) == 8) *reinterpret_cast<uint2 *>(q) = reinterpret_cast<const uint2 *>(w)[r];
                else {
#pragma unroll
                    for (int i = 0; i < kWords / 8; ++i)
                        reinterpret_cast<uint4 *>(q)[i] = reinterpret_cast<const uint4 *>(w)[r * (kWords / 8) + i];
                }
            }
        } else {
            const T *t = reinterpret_cast<const T *>(w);
#pragma unroll
            for (int i = 0; i < N; ++i) p[i < kRun ? i : second + i - kRun] = t[i];
        }
    }
    // in fp32, two values at a time
    __device__ __forceinline__ void up(f32x2 *x) const
    {
        const T *t = reinterpret_cast<const T *>(w);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) x[i] = pack2(TokType<T>::up(t[2 * i]), TokType<T>::up(t[2 * i + 1]));
    }
    __device__ __forceinline__ void down(const f32x2 *x)
    {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float2 v = unpack2(x[i]);
            if constexpr (sizeof(T) == 4) {
                w[2 * i] = __float_as_uint(v.x);
                w[2 * i + 1] = __float_as_uint(v.y);
            } else if constexpr (std::is_same<T, __half>::value) {
                const __half2 h = __floats2half2_rn(v.x, v.y);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
    }
    // the bits of the largest magnitude, in the values' type, and as fp32
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

// Sine and cosine of t 2^-64 turns: quarter turns aside, the eighth of a turn that is left as an fp32 multiple of 2^-32, and what
// that leaves (below 2^-27 of a turn) by the first order.  The low half of t counts where the angle is small: its sine then has
// fp32's relative bits as well.
__device__ __forceinline__ void of_turn(uint64_t t, float &sine, float &cosine)
{
    const uint32_t hi = (uint32_t)((t + 0x80000000ull) >> 32), q = (hi + 0x20000000u) >> 30;
    const int32_t lo = (int32_t)(uint32_t)t, r = (int32_t)(hi - (q << 30));
    const float near = (float)r, rest = fmaf((float)lo, 0x1p-32f, (float)(r - (int32_t)near)) * (3.14159265f * 0x1p-31f);
    float s, c;
    sincospif(near * 0x1p-31f, &s, &c);
    const float s1 = fmaf(c, rest, s), c1 = fmaf(-s, rest, c);
    sine = q & 1 ? c1 : s1;
    cosine = q & 1 ? s1 : c1;
    sine = q & 2 ? -sine : sine;
    cosine = (q + 1) & 2 ? -cosine : cosine;
}

template <class T, int TO, bool ADJ, int N>
__global__ void __launch_bounds__(kThreads, 4) k_tokens_rotate(RotateParams p)
{
    using X = Part<T, N>;
    constexpr int kRows = 64 / (N * (int)sizeof(T));                 // rows of a batch: 64 bytes of a thread
    constexpr int kKinds = TO == kToRows ? 2 : 3;                    // queries, keys, values
    __shared__ typename X::Piece ring[kAhead + 1][kRows * X::kPieces][kThreads];
    __shared__ float sines[N][kThreads];                             // a thread's own: its pairs' cosines, then their sines
    TokSeq sq;
    const Tile t = tile_of(p.b, false, sq);
    const int D = p.pool.d, slot = threadIdx.x & (p.lanes - 1), group = threadIdx.x / p.lanes, groups = kThreads / p.lanes;
    const bool in = slot * N < D, turned = slot * N < p.r.rot;
    // this thread's values of a row: two runs, half of the rotated values apart (or of the others): a pair of halves has one in
    // either, neighbours are in one, and the lanes' copies lie side by side
    const int half = p.r.rot / 2, at = turned ? slot * (N / 2) : p.r.rot + (slot * N - p.r.rot) / 2, second = turned ? half : (D - p.r.rot) / 2;
    const float over = 1.f / D;
    // the block's groups over the tile's tokens: of fewer tokens than groups each has several, which share its heads
    const int share = t.n < groups ? groups / t.n : 1, together = groups / share;
    const int parts = share * gridDim.y, part = blockIdx.y * share + group % share;
    const int32_t *table = p.b.table + sq.table0;

    // A group's rows, batch after batch: of its first token the queries part, part + parts, ..., its keys, its values, then
    // its next token's.  Batches are copied to shared memory kAhead before they are worked on; a thread copies what it
    // works on itself, so that it has none but its own copies to wait for.
    struct At {
        int i, kind, h;                                              // token (group's own part is added), kind, first head less part
    };
    auto heads_of = [&](int kind) { return kind == 0 ? p.q_heads : p.k_heads; };
    auto next = [&](At a) {
        a.h += parts * kRows;
        while (a.h >= heads_of(a.kind)) {                            // (for all threads alike; a kind may have no heads)
            a.h = 0;
            if (++a.kind == kKinds) {
                a.kind = 0;
                a.i += together;
                break;
            }
        }
        if (a.h == 0 && a.kind == 0 && p.q_heads == 0) a.kind = 1;
        return a;
    };
    At now{0, p.q_heads ? 0 : 1, 0}, then = now;                     // the batch that is worked on, and the next to be copied
    // of the next to be copied: its first row, the steps from row to row, and how many heads are left from there on
    const T *src = nullptr;
    int64_t src_step = 0;
    int left = 0, vec = 0;
    auto fetch = [&](int at_slot) {
        if (then.h == 0) {
            const TokRows &from = then.kind == 0 ? p.q : then.kind == 1 ? p.k : p.v;
            const int i = then.i + group / share;
            const bool on = in && i < t.n;
            src = reinterpret_cast<const T *>(from.p) + (on ? (int64_t)(sq.row0 + t.i0 + i) * from.ts + part * from.hs + at : 0);
            src_step = on ? parts * from.hs : 0;
            left = on ? heads_of(then.kind) - part : 0;
            vec = from.vec;
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const bool on = left > 0;
#pragma unroll
            for (int e = 0; e < X::kPieces; ++e) {
                typename X::Piece *to = &ring[at_slot][u * X::kPieces + e][threadIdx.x];
                const T *x = src + (e < X::kRunPieces ? e * X::kPer : second + (e - X::kRunPieces) * X::kPer);
                if (vec) {
                    if (on) {
                        const uint32_t s = (uint32_t)__cvta_generic_to_shared(to);
                        if constexpr (X::kPiece == 16)
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s), "l"(x) : "memory");
                        else
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(s), "l"(x) : "memory");
                    }
                } else if (on) {                                     // rows that start anywhere
                    alignas(16) T v[X::kPer];
#pragma unroll
                    for (int c = 0; c < X::kPer; ++c) v[c] = x[c];
                    *to = *reinterpret_cast<const typename X::Piece *>(v);
                }
            }
            src += src_step;
            left -= parts;
        }
    };
    int slot_now = 0, slot_then = 0;
    auto copy = [&] {
        if (then.i < t.n) {
            fetch(slot_then);
            then = next(then);
        }
        slot_then = slot_then + 1 == kAhead + 1 ? 0 : slot_then + 1;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll 1
    for (int i = 0; i < kAhead; ++i) copy();

    while (now.i < t.n) {
        const int i = now.i + group / share;
        const bool here = in && i < t.n;
        const int64_t token = here ? sq.row0 + t.i0 + i : sq.row0;
        if (here && turned) {
            const int own = p.r.positions ? 0 : sq.pos + (p.b.node ? __ldg(&p.b.node[token].depth) : t.i0 + i);
#pragma unroll
            for (int e = 0; e < N / 2; ++e) {
                const int k = !ADJ ? at + e : e < N / 4 ? at / 2 + e : (half + at) / 2 + e - N / 4;
                const int pos = p.r.positions ? __ldg(p.r.positions + __ldg(p.r.axis + k) * p.r.position_stride + token) : own;
                const uint64_t turn = (uint64_t)(int64_t)pos * __ldg(p.r.turn + k);
                float sine, cosine;
                of_turn(turn, sine, cosine);
                sines[e][threadIdx.x] = cosine;
                sines[N / 2 + e][threadIdx.x] = sine;
            }
        }
        // the token's cell: of head 0, in the pools' rows
        const int64_t cell = TO != kToRows && here ? cell_row(p.pool, table, 0, sq.pos + t.i0 + i) : 0;
        // all of the token's rows of a kind
        auto rows = [&](auto of_kind, const TokRows &to) {
            constexpr int KIND = decltype(of_kind)::value;
            constexpr bool kCells = KIND > 0 && TO != kToRows, kCodes = KIND > 0 && TO == kToCodes;
            const int heads = heads_of(KIND);
            const bool norm = KIND == 0 ? p.r.norm_q : KIND == 1 && p.r.norm_k;
            // two of a thread's values y, next to one another, become y c + y' s: y' the ones that they are paired with, c and s
            // their cosines and sines, times the weights (of values that are not rotated c is the weights)
            f32x2 c[N / 2], s[N / 2];
            if (KIND < 2) {
                alignas(16) float w[N];
#pragma unroll
                for (int e = 0; e < N; ++e) w[e] = 1.f;
                if (norm && here) {
                    const float *weight = p.r.weight + (KIND == 0 ? 0 : D) + at;
#pragma unroll
                    for (int e = 0; e < N; e += 4)
                        *reinterpret_cast<float4 *>(w + e) = __ldg(reinterpret_cast<const float4 *>(weight + (e < N / 2 ? e : second + e - N / 2)));
                }
                auto cosine = [&](int e) { return turned ? sines[e][threadIdx.x] : 1.f; };
                auto sine = [&](int e) { return turned ? sines[N / 2 + e][threadIdx.x] : 0.f; };
#pragma unroll
                for (int e = 0; e < N / 2; ++e) {
                    if (ADJ) {
                        c[e] = pack2(cosine(e) * w[2 * e], cosine(e) * w[2 * e + 1]);
                        s[e] = pack2(-sine(e) * w[2 * e + 1], sine(e) * w[2 * e]);      // (with the other value's weight)
                    } else {
                        const int k = 2 * e % (N / 2), o = (2 * e + N / 2) % N;
                        const float sign = e < N / 4 ? -1.f : 1.f;
                        c[e] = pack2(cosine(k) * w[2 * e], cosine(k + 1) * w[2 * e + 1]);
                        s[e] = pack2(sign * sine(k) * w[o], sign * sine(k + 1) * w[o + 1]);
                    }
                }
            }
            // into rows, or cells (a head's lie a page's rows behind the one's before it)
            const int64_t row0 = cell + ((int64_t)part << p.pool.page_log2), cell_step = (int64_t)parts << p.pool.page_log2;
            T *dst = kCells ? static_cast<T *>(KIND == 2 ? p.pool.v : p.pool.k) + (row0 * D + at)
                            : reinterpret_cast<T *>(to.p) + token * to.ts + part * to.hs + at;
            const int64_t dst_step = kCells ? cell_step * D : parts * to.hs;
            uint8_t *code = reinterpret_cast<uint8_t *>(KIND == 2 ? p.pool.v : p.pool.k) + (row0 * D + at);
            uint8_t *byte_at = (KIND == 2 ? p.pool.vs : p.pool.ks) + row0;
            for (int h0 = 0; h0 < heads; h0 += parts * kRows) {
                copy();
                asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
                X x[kRows];
#pragma unroll
                for (int u = 0; u < kRows; ++u)
#pragma unroll
                    for (int e = 0; e < X::kPieces; ++e)
                        x[u].piece(e, here && h0 + part + u * parts < heads ? ring[slot_now][u * X::kPieces + e][threadIdx.x] : typename X::Piece{});
                slot_now = slot_now + 1 == kAhead + 1 ? 0 : slot_now + 1;
                now = next(now);
#pragma unroll
                for (int u = 0; u < kRows; ++u) {
                    if (h0 + u * parts >= heads) break;              // (for all threads alike)
                    const bool on = here && h0 + part + u * parts < heads;
                    f32x2 y[N / 2];
                    if (KIND < 2) {
                        x[u].up(y);
                        if (norm) {
                            auto over_lanes = [&](f32x2 two) {
                                float sum = unpack2(two).x + unpack2(two).y;
                                for (int l = p.lanes >> 1; l; l >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, l);
                                return sum;
                            };
                            f32x2 two = 0;
#pragma unroll
                            for (int e = 0; e < N / 2; ++e) two = fma2(y[e], y[e], two);
                            const float sum = over_lanes(two);
                            float f = rsqrtf(fmaf(sum, over, p.r.eps));
                            // squares that leave fp32's range: once more, of the values times a power of two.  Small ones (below
                            // an eps of 2^-100 they do not count) are multiplied by it and then by the root, large ones the other
                            // way round: no step then leaves the range where the outcome does not, the least numbers' either
                            if (__any_sync(0xffffffffu, on && !(sum >= 0x1p-80f && sum < INFINITY))) {
                                const bool small = sum < 0x1p-80f, lost = small ? p.r.eps < 0x1p-100f : !(sum < INFINITY);
                                const float g = small ? 0x1p100f : 0x1p-70f;
                                f32x2 again = 0;
#pragma unroll
                                for (int e = 0; e < N / 2; ++e) {
                                    const f32x2 z = mul2(y[e], pack2(g, g));
                                    again = fma2(z, z, again);
                                }
                                const float root = rsqrtf(fmaf(over_lanes(again), over, p.r.eps * g * g));
                                const float before = !lost ? 1.f : small ? g : root;
#pragma unroll
                                for (int e = 0; e < N / 2; ++e) y[e] = mul2(y[e], pack2(before, before));
                                if (lost) f = small ? root : g;
                            }
#pragma unroll
                            for (int e = 0; e < N / 2; ++e) y[e] = mul2(y[e], pack2(f, f));
                        }
                        if (turned) {
                            f32x2 z[N / 2];
#pragma unroll
                            for (int e = 0; e < N / 2; ++e) {
                                const f32x2 o = ADJ ? pack2(unpack2(y[e]).y, unpack2(y[e]).x) : y[(e + N / 4) % (N / 2)];
                                z[e] = fma2(y[e], c[e], mul2(o, s[e]));
                            }
#pragma unroll
                            for (int e = 0; e < N / 2; ++e) y[e] = z[e];
                        } else if (norm) {
#pragma unroll
                            for (int e = 0; e < N / 2; ++e) y[e] = mul2(y[e], c[e]);
                        }
                        x[u].down(y);                                // the one rounding to the activations' type
                    }
                    if (!kCodes) {
                        if (on) x[u].store(dst, second, kCells ? 1 : to.vec);
                        dst += dst_step;
                    } else {
                        uint32_t most = x[u].most();
                        for (int l = p.lanes >> 1; l; l >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, l));
                        const uint32_t byte = scale_byte(X::bits_up(most));
                        if (on) {
                            x[u].up(y);
                            const float unit = unscale(1.f, byte);   // (a row with an infinity or a NaN: zeros, below)
                            uint32_t q[N / 4];
#pragma unroll
                            for (int e = 0; e < N / 4; ++e) {
                                const float2 a = unpack2(mul2(y[2 * e], pack2(unit, unit))), b = unpack2(mul2(y[2 * e + 1], pack2(unit, unit)));
                                q[e] = byte == 255u ? 0u : e4m3_pair(a.x, a.y) | e4m3_pair(b.x, b.y) << 16;
                            }
                            if (N == 16) {
                                *reinterpret_cast<uint2 *>(code) = make_uint2(q[0], q[1]);
                                *reinterpret_cast<uint2 *>(code + second) = make_uint2(q[N / 4 - 2], q[N / 4 - 1]);
                            } else {
                                *reinterpret_cast<uint32_t *>(code) = q[0];
                                *reinterpret_cast<uint32_t *>(code + second) = q[1];
                            }
                            if (slot == 0) *byte_at = (uint8_t)byte;
                        }
                        code += dst_step;
                        byte_at += cell_step;
                    }
                }
            }
        };
        rows(std::integral_constant<int, 0>{}, p.q_out);
        rows(std::integral_constant<int, 1>{}, p.k_out);
        if (TO != kToRows) rows(std::integral_constant<int, 2>{}, p.v);
    }
}

template <class T, int TO, bool ADJ, int N>
int go(RotateParams p, int64_t tiles, cudaStream_t s)
{
    p.lanes = 1;
    while (p.lanes * N < p.pool.d) p.lanes *= 2;
    // several blocks share a tile's heads as long as all run at a time, down to two batches of queries for each group: each
    // has its sines to compute again (3,200 tokens of 32 and 8 heads, in two waves 27 us, in one 19)
    const int groups = kThreads / p.lanes, heads = p.q_heads > p.k_heads ? p.q_heads : p.k_heads;
    const int64_t tokens = (p.tokens + tiles - 1) / tiles, share = tokens < groups ? groups / tokens : 1, each = share * (128 / (N * sizeof(T)));
    const int64_t fit = kBlocks * (int64_t)sm_count() / tiles, want = fit > 1 ? fit : 1, most = (heads + each - 1) / each;
    k_tokens_rotate<T, TO, ADJ, N><<<dim3((unsigned)tiles, (unsigned)(want < most ? want : most)), kThreads, 0, s>>>(p);
    return 1;
}

template <class T, int TO, bool ADJ>
int by_width(const RotateParams &p, int64_t tiles, cudaStream_t s)
{
    return p.pool.d % 16 == 0 && p.r.rot % 16 == 0 ? go<T, TO, ADJ, 16>(p, tiles, s) : go<T, TO, ADJ, 8>(p, tiles, s);
}

template <class T>
int by_target(const RotateParams &p, int to, int64_t tiles, cudaStream_t s)
{
    const bool adj = p.r.adjacent != 0;
    if (to == kToRows) return adj ? by_width<T, kToRows, true>(p, tiles, s) : by_width<T, kToRows, false>(p, tiles, s);
    if (to == kToCells) return adj ? by_width<T, kToCells, true>(p, tiles, s) : by_width<T, kToCells, false>(p, tiles, s);
    return adj ? by_width<T, kToCodes, true>(p, tiles, s) : by_width<T, kToCodes, false>(p, tiles, s);
}

}  // namespace

int launch_tokens_rotate(const TokPool &pool, const TokBatch &b, const TokRotary &r, int dtype, int form, bool cells, int q_heads,
                         int k_heads, TokRows q, TokRows k, TokRows v, TokRows q_out, TokRows k_out, int64_t tokens, int64_t tiles,
                         cudaStream_t s)
{
    if (tiles == 0 || q_heads + k_heads == 0) return 0;
    const RotateParams p{pool, b, r, q, k, v, q_out, k_out, q_heads, k_heads, 1, tokens};
    const int to = !cells ? kToRows : form == MURE_FORM_E4M3 ? kToCodes : kToCells;
    if (dtype == MURE_F32) return by_target<float>(p, to, tiles, s);
    if (dtype == MURE_F16) return by_target<__half>(p, to, tiles, s);
    return by_target<__nv_bfloat16>(p, to, tiles, s);
}

}  // namespace mure
