// Token caches: attention of few rows (a decoding step's single tokens), and of any rows in fp32.
//
// A sequence's cells are read once per cached head, all query heads of the group as the 16 rows of
// one mma tile, so the kernel is bound by device memory: 4 D flops per row and cell against
// 2 D bytes a cell.  What decides is the bytes in flight and an even split:
//   - the (sequence, cached head) pairs are dealt out whole to the resident blocks, the longest first,
//     those that do not fit an even share in parts; a pair that is cut is joined by the block that
//     finishes last, in the order of its parts (equal bits whatever the order of arrival);
//   - each warp of a block takes a quarter of every tile with a running maximum and sum of its
//     own, and a ring of cp.async stages of its own: no barrier in the loop;
//   - e4m3 codes are widened in registers to f16 (one conversion for two, exact), whatever the rows' type:
//     bf16 rows of q become f16 ones with their largest magnitude brought to 8 .. 16 by a power of two,
//     exact down to 2^-18 of it and in units of 2^-27 of it below (f16 products take half the conversions of
//     bf16 ones here, and a score moves by no more than 2^-28 of the largest q times the sum of |k|).  A cell's scale of K goes to its score and that of V, relative to the
//     largest met so far, to its probability, in fp32 (scales far below the largest: in part to the values; a
//     spread beyond what f16 then holds sends the rows to the definition).
// fp32 rows take the same way with TF32 products: every operand is split in two TF32 halves, a = a_hi + a_lo,
// and a product is a_hi b_hi + a_hi b_lo + a_lo b_hi (codes are TF32 values as they are: two products).
// What a row's scores are taken relative to lies 7 below their running maximum and moves only when that
// grows by more than 8 (in powers of two): the sums then need no rescaling in nearly all steps. Powers
// reach 2^15, which f16 holds, and those down to 2^-21 of the largest keep all its bits.
//
// The 16-bit products take P = 2^(s - m) rounded to the cells' type (f16 on codes): that is what the mma takes,
// and the sums of P beside it keep all their bits.  A second product with P's low half would halve the error
// (1.2 to 1.4 times that of an output rounded once) for half of the mma work more.  Powers come from the
// hardware's approximation, 2 units in fp32's last place.
//
// Measured (GB300): two sequences of 100,000 and 131,000 cells, 8 cached heads of 128 bf16 values: 155 us,
// 6.3 TB/s.  64 sequences of 500 to 12,000 e4m3 cells, the same heads: 175 us, 4.9 TB/s: bound by latency there,
// not by issue: three blocks per SM, 2.7 warps per scheduler, issue in 47 % of the cycles and wait most of all for
// results of fixed latency (870 instructions per warp and 32 cells, of which 128 widen codes).  96 sequences of f16
// cells within a window of 1,024: 26 us, 3.8 TB/s, a unit of ten tiles per block.  fp32 chunks (6 sequences,
// 12 heads of 64): 127 us, the mma pipe 43 % busy.
#include <type_traits>

#include "tokens_util.cuh"

namespace mure {

namespace {

constexpr int kWarps = 4;
constexpr int kAlign = 16;

// 16-bit rows on codes: how far apart, in powers of two, the scales of V that a warp meets may lie.  A probability
// p <= 1 of its row's largest is held as an f16 number near 2^7 p, in units of 2^-25 at worst.  A cell's scale
// relative to the largest goes to its value down to 2^-14, exactly, and below that to the probability, which then is
// good to 2^-32 / 2^-6 = 2^-26 of the row's largest at 2^-20.  Past that the rows are done by the definition.
// (Following the scales, K's too, costs 64 sequences on codes 172 -> 175 us.)
constexpr int kSpread = 20;

// The largest scale byte of K on codes: a sum of products of q (up to 2^16) and codes (2^9), 256 of them, times the
// scale stays below 2^127.  Past it the product overflows before its last factor, which may be small, and a
// score that overflows to -inf would look like a masked one: such rows, too, are done by the definition.
constexpr int kMostScaleK = 127 + 127 - (16 + 9 + 8);

template <class T, bool E4M3, int DP>
struct Few {
    static constexpr bool kF32 = std::is_same<T, float>::value;
    using Prod = typename std::conditional<E4M3 && !kF32, __half, T>::type;   // type of the products' operands
    static constexpr int kElt = E4M3 ? 1 : (int)sizeof(T);
    static constexpr int kRow = DP * kElt;                                   // bytes of a staged row
    static constexpr int kLeast = kF32 ? 8 : 16;
    static constexpr int kBytes = kF32 && E4M3 && DP > 64 ? 2048 : 4096;     // of a step's K or V rows
    static constexpr int kStages = kRow < 128 ? 4 : 2;
    static constexpr int WK = (kBytes / kRow < kLeast) ? kLeast : (kBytes / kRow > 32 ? 32 : kBytes / kRow);   // cells of a warp's step
    static constexpr int kTile = kWarps * WK;
    static constexpr int kScaleBytes = E4M3 ? 2 * WK : 0;
    static constexpr int kStage = 2 * WK * kRow + kScaleBytes;               // K rows, V rows, scales
    static constexpr int kStageAl = (kStage + 127) / 128 * 128;
    static constexpr int kJoin = kWarps * kFewRows * (DP + 2) * 4 + kWarps * kFewRows * 4;   // (and the parts' weights)
    static constexpr int kRing = kWarps * kStages * kStageAl;
    // the fragments of q: in registers; for 256 values, fp32 and codes in shared memory (one copy for all warps)
    static constexpr bool kSharedQ = DP > 128 || kF32 || E4M3;
    static constexpr int kQSteps = kF32 ? DP / 8 : DP / 16;
    static constexpr int kQ = kSharedQ ? kQSteps * 32 * 16 : 0;
    static constexpr int kFactors = E4M3 ? kWarps * 3 * 32 * 4 : 0;          // a step's scales, as factors
    static constexpr int kSmem = (kRing > kJoin ? kRing : kJoin) + kQ + kFactors;
    static_assert(kSmem >= kMostParts * kFewRows * 4, "a unit's weights of parts do not fit");
    static constexpr int kBlocks = kSmem > 110 * 1024 ? 1 : DP > 128 || kSmem > 74 * 1024 || (kF32 && DP > 64) ? 2 : 3;   // per SM
};

struct FewParams {
    TokPool pool;
    TokBatch b;
    TokWork w;
    TokRows q, out;
    float *lse;
};

__device__ __forceinline__ uint32_t su32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// Byte `byte` of staged row `row`: the eight 16-byte chunks of a 128-byte line are exchanged by the
// row's (rows of 64 bytes: the line's) number, so that the loads meet no bank conflict: ldmatrix reads a
// chunk of eight rows; with fp32 cells eight lanes read four chunks of two rows of K, or two chunks of
// four rows, each second one, of V.
template <int ROW, bool F32>
__device__ __forceinline__ uint32_t swz(int row, int byte, bool v)
{
    const uint32_t o = row * ROW + byte;
    const int x = F32 ? (v ? row & 6 : (row & 1) << 2 | (row >> 1 & 3)) : (ROW >= 128 ? row : row >> 1) & 7;
    return o ^ (uint32_t)(x << 4);
}

__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool on)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp8(uint32_t dst, const void *src, bool on)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(on ? 8 : 0) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void *src, bool on)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(on ? 4 : 0) : "memory");
}

__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t *r)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t *r)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}

__device__ __forceinline__ float4 lds16(uint32_t a)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float2 lds8(uint32_t a)
{
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds4(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

// TF32 halves: the high one rounded to the nearest, the low one the exact remainder, of which the product
// reads the upper 19 bits (a NaN stays one in the remainder, whatever becomes of its bits in the high half).
__device__ __forceinline__ void halves(float x, uint32_t &hi, uint32_t &lo)
{
    hi = (__float_as_uint(x) + 0x1000u) & 0xFFFFE000u;
    lo = __float_as_uint(x - __uint_as_float(hi));
}

__device__ __forceinline__ void mma_tf32(float *c, const uint32_t *a, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// c += a_hi b_hi, x += the products with a low half (two accumulators: a product waits for the one before it
// on the same); b0, b1 as fp32 (EXACT: they are TF32 values).
template <bool EXACT>
__device__ __forceinline__ void mma_f32(float *c, float *x, const uint32_t *hi, const uint32_t *lo, float b0, float b1)
{
    if (EXACT) {
        mma_tf32(x, lo, __float_as_uint(b0), __float_as_uint(b1));
        mma_tf32(c, hi, __float_as_uint(b0), __float_as_uint(b1));
    } else {
        uint32_t h0, l0, h1, l1;
        halves(b0, h0, l0);
        halves(b1, h1, l1);
        mma_tf32(x, lo, h0, h1);
        mma_tf32(x, hi, l0, l1);
        mma_tf32(c, hi, h0, h1);
    }
}

template <class T> struct Mma;
template <> struct Mma<float> {     // (for the names alone: fp32 rows have products of their own)
    static __device__ __forceinline__ void go(float *, const uint32_t *, uint32_t, uint32_t) {}
    static __device__ __forceinline__ uint32_t pack(float, float) { return 0; }
};
template <> struct Mma<__nv_bfloat16> {
    static __device__ __forceinline__ void go(float *c, const uint32_t *a, uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};
template <> struct Mma<__half> {
    static __device__ __forceinline__ void go(float *c, const uint32_t *a, uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};

// Two e4m3 codes in the low 16 bits.
__device__ __forceinline__ uint32_t widen(uint32_t two)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    return h;
}

__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Two neighbouring values of a row of q (element offset even; rows may start anywhere).
template <class T>
__device__ __forceinline__ uint32_t load2(const T *p, int vec)
{
    if (vec) return __ldg(reinterpret_cast<const unsigned int *>(p));
    const uint16_t *u = reinterpret_cast<const uint16_t *>(p);
    return (uint32_t)u[0] | (uint32_t)u[1] << 16;
}

template <class T, bool E4M3, int DP, bool TREE>
__global__ void __launch_bounds__(kWarps * 32, Few<T, E4M3, DP>::kBlocks) k_tokens_few(FewParams p)
{
    using F = Few<T, E4M3, DP>;
    using M = Mma<typename F::Prod>;
    constexpr int KS = F::kQSteps, NT = F::WK / 8, ND = DP / 8, WK = F::WK;
    extern __shared__ __align__(128) char smem[];
    __shared__ TokItem w;
    __shared__ float row_factor[kFewRows];                   // bf16 rows on codes
    __shared__ int ends[2];                                  // positions of the first and the last row
    __shared__ int last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int D = p.pool.d, psz = 1 << p.pool.page_log2;
    const uint32_t ring = su32(smem) + warp * F::kStages * F::kStageAl;
    const int row_bytes = D * F::kElt;

    for (int it = p.w.first[blockIdx.x]; it < p.w.first[blockIdx.x + 1]; ++it) {
        if (threadIdx.x < sizeof(TokItem) / 8)
            reinterpret_cast<int2 *>(&w)[threadIdx.x] = __ldg(reinterpret_cast<const int2 *>(p.w.items + it) + threadIdx.x);
        __syncthreads();
        // (a tree's rows see all cells before its own, and lie no further than a chain's)
        if (threadIdx.x < 2)
            ends[threadIdx.x] = TREE && threadIdx.x == 0 ? w.pos - 1 : w.pos + (w.r0 + (threadIdx.x ? w.rows - 1 : 0)) / p.b.group;
        __syncthreads();
        const int nA = (w.a1 + F::kTile - 1) / F::kTile, b_al = w.b0 & ~(kAlign - 1);

        // one step of this warp: cells [start, start + WK), of which begin .. end - 1 take part
        auto range = [&](int tile, int &start, int &begin, int &end) {
            if (tile < nA) { start = tile * F::kTile; begin = 0; end = w.a1; }
            else { start = b_al + (tile - nA) * F::kTile; begin = w.b0; end = w.b1; }
            start += warp * WK;
        };
        // the page of group `lane` of eight cells of a step (0 where it has none that take part)
        auto pages = [&](int tile) {
            if (tile >= w.t1 || lane >= WK / 8) return 0;
            int start, begin, end;
            range(tile, start, begin, end);
            const int j = start + lane * 8;
            return j < end ? __ldg(p.b.table + w.table0 + (j >> p.pool.page_log2)) : 0;
        };
        auto issue = [&](int tile, int slot, int page_of_group) {
            if (tile < w.t1) {
                int start, begin, end;
                range(tile, start, begin, end);
                const uint32_t st = ring + slot * F::kStageAl;
                constexpr int CH = F::kRow / 16;               // chunks of a staged row
                constexpr int PER = CH < 32 ? 32 / CH : 1;     // rows that a warp's instruction covers,
                constexpr int REP = CH > 32 ? CH / 32 : 1;     // or instructions a row takes
                static_assert(PER * CH == 32 || REP * 32 == CH, "rows and lanes do not divide");
                const int r0 = CH < 32 ? lane / CH : 0;
                // whole steps of rows without padding (nearly all): plain copies
                if (start >= begin && start + WK <= end && row_bytes == F::kRow) {
                    // (groups of 16 cells, or of 8 for the smallest pages: 64 sequences on codes 176 -> 174 us)
                    auto copy = [&](auto cells_of_group) {
                        constexpr int GS = decltype(cells_of_group)::value;
#pragma unroll
                        for (int grp = 0; grp < WK / GS; ++grp) {
                            const int page = __shfl_sync(0xffffffffu, page_of_group, grp * (GS / 8));
                            const int64_t row = (((int64_t)page * p.pool.hk + w.h) << p.pool.page_log2) | ((start + grp * GS) & (psz - 1));
                            const int64_t at = row * F::kRow + r0 * F::kRow + (REP > 1 ? lane : lane % CH) * 16;
                            const char *kb = static_cast<const char *>(p.pool.k) + at, *vb = static_cast<const char *>(p.pool.v) + at;
#pragma unroll
                            for (int e = 0; e < GS * REP; e += PER) {
                                const int r = e / REP + r0, byte = (REP > 1 ? lane + e % REP * 32 : lane % CH) * 16;
                                const int off = e / REP * F::kRow + e % REP * 512;
                                cp16(st + swz<F::kRow, F::kF32 && !E4M3>(grp * GS + r, byte, false), kb + off);
                                cp16(st + WK * F::kRow + swz<F::kRow, F::kF32 && !E4M3>(grp * GS + r, byte, true), vb + off);
                            }
                        }
                    };
                    if constexpr (F::kF32) copy(std::integral_constant<int, 8>{});
                    else if (p.pool.page_log2 >= 4) copy(std::integral_constant<int, 16>{});
                    else copy(std::integral_constant<int, 8>{});
                } else {
#pragma unroll
                for (int grp = 0; grp < WK / 8; ++grp) {
                    const int page = __shfl_sync(0xffffffffu, page_of_group, grp);
                    const int j0 = start + grp * 8;
                    const int64_t row = (((int64_t)page * p.pool.hk + w.h) << p.pool.page_log2) | (j0 & (psz - 1));
                    const char *kb = static_cast<const char *>(p.pool.k) + row * row_bytes;
                    const char *vb = static_cast<const char *>(p.pool.v) + row * row_bytes;
                    if (j0 + 7 < begin || j0 >= end) kb = static_cast<const char *>(p.pool.k), vb = static_cast<const char *>(p.pool.v);
#pragma unroll(F::kF32 && DP > 128 ? 4 : 16)   // (fp32 of 256 values: 16 addresses at a time would spill)
                    for (int e = 0; e < 8 * REP; e += PER) {
                        const int r = e / REP + r0, byte = (REP > 1 ? lane + e % REP * 32 : lane % CH) * 16;
                        const bool in = j0 + r >= begin && j0 + r < end;
                        const uint32_t o = swz<F::kRow, F::kF32 && !E4M3>(grp * 8 + r, byte, false);
                        const uint32_t ov = WK * F::kRow + swz<F::kRow, F::kF32 && !E4M3>(grp * 8 + r, byte, true);
                        if (!E4M3 || D % 16 == 0) {
                            const bool on = in && byte < row_bytes;
                            const int64_t off = on ? (int64_t)r * row_bytes + byte : 0;
                            cp16(st + o, kb + off, on);
                            cp16(st + ov, vb + off, on);
                        } else {                               // rows of codes at 8-byte boundaries
#pragma unroll
                            for (int q = 0; q < 16; q += 8) {
                                const bool on = in && byte + q < row_bytes;
                                const int64_t off = on ? (int64_t)r * row_bytes + byte + q : 0;
                                cp8(st + o + q, kb + off, on);
                                cp8(st + ov + q, vb + off, on);
                            }
                        }
                    }
                }
                }
                const int scale_page = E4M3 ? __shfl_sync(0xffffffffu, page_of_group, lane / 2) : 0;
                if (E4M3 && lane < WK / 4) {
                    const int j = start + lane * 4, page = scale_page;
                    const bool on = j + 3 >= begin && j < end;
                    const int64_t row = on ? (((int64_t)page * p.pool.hk + w.h) << p.pool.page_log2) | (j & (psz - 1)) : 0;
                    cp4(st + 2 * WK * F::kRow + lane * 4, p.pool.ks + row, on);
                    cp4(st + 2 * WK * F::kRow + WK + lane * 4, p.pool.vs + row, on);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };

        // the first stages are on their way while q is fetched
        int next_pages = pages(w.t0);
#pragma unroll
        for (int i = 0; i < F::kStages - 1; ++i) {
            const int cur = next_pages;
            next_pages = pages(w.t0 + i + 1);
            issue(w.t0 + i, i, cur);
        }

        uint32_t qf[F::kSharedQ ? 1 : KS][4];
        uint4 *q_shared = reinterpret_cast<uint4 *>(smem + F::kSmem - F::kFactors - F::kQ);
        // every fragment of q (shared ones: `all`, or by warp 0 alone)
        auto for_q = [&](bool all, auto fn) {
            if (!F::kSharedQ) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) fn(qf[F::kSharedQ ? 0 : ks]);
            } else if (all || warp == 0) {
                for (int ks = 0; ks < KS; ++ks) fn(reinterpret_cast<uint32_t *>(q_shared + ks * 32 + lane));
            }
        };
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = w.r0 + g + half * 8;
            const bool on = g + half * 8 < w.rows && (!F::kSharedQ || warp == 0);
            const T *q = reinterpret_cast<const T *>(p.q.p) +
                         (on ? (int64_t)(w.row0 + r / p.b.group) * p.q.ts + (int64_t)(w.h * p.b.group + r % p.b.group) * p.q.hs : 0);
#pragma unroll(F::kSharedQ ? 4 : KS)
            for (int ks = 0; ks < KS; ++ks) {
                // the order of a row's values within a step only has to be that of the cells' values
                uint32_t x0, x1;
                if constexpr (F::kF32) {
                    const int d0 = ks / 2 * 16 + 4 * t + ks % 2 * 2;
                    x0 = on && d0 < D ? __float_as_uint(q[d0]) : 0u;
                    x1 = on && d0 < D ? __float_as_uint(q[d0 + 1]) : 0u;
                } else {
                    const int d0 = ks * 16 + (E4M3 ? 4 * t : 2 * t), d1 = d0 + (E4M3 ? 2 : 8);
                    x0 = on && d0 < D ? load2(q + d0, p.q.vec) : 0u;
                    x1 = on && d1 < D ? load2(q + d1, p.q.vec) : 0u;
                }
                if (!F::kSharedQ) {
                    qf[F::kSharedQ ? 0 : ks][half] = x0;
                    qf[F::kSharedQ ? 0 : ks][2 + half] = x1;
                } else if (warp == 0) {
                    uint32_t *f = reinterpret_cast<uint32_t *>(q_shared + ks * 32 + lane);
                    f[half] = x0;
                    f[2 + half] = x1;
                }
            }
        }
        // scores: products times rowf (and a cell's scale) are powers of two
        constexpr bool kRowFactor = E4M3 && std::is_same<T, __nv_bfloat16>::value;
        if constexpr (kRowFactor) {
            uint32_t top[2] = {0, 0};
            auto magnitude = [](uint32_t two) { return max(two & 0x7FFFu, two >> 16 & 0x7FFFu); };
            if (F::kSharedQ) __syncthreads();
            for_q(true, [&](uint32_t *f) {
                top[0] = max(top[0], max(magnitude(f[0]), magnitude(f[2])));
                top[1] = max(top[1], max(magnitude(f[1]), magnitude(f[3])));
            });
            float up[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                top[i] = max(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
                top[i] = max(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
                const uint32_t e = top[i] >> 7;                        // 255: an infinity or a NaN, left as it is
                const uint32_t f = e == 255u ? 127u : min(257u - e, 253u);
                up[i] = __uint_as_float(f << 23);
                if (warp == 0 && t == 0) row_factor[g + 8 * i] = p.b.scale_log2 * __uint_as_float((254u - f) << 23);
            }
            if (F::kSharedQ) __syncthreads();
            for_q(false, [&](uint32_t *f) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    f[i] = M::pack(__uint_as_float(f[i] << 16) * up[i & 1], __uint_as_float(f[i] & 0xFFFF0000u) * up[i & 1]);
            });
        }
        if (F::kSharedQ) __syncthreads();

        float o[ND][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        int v_top = 0, v_low = 255;                          // E4M3: the largest scale byte of V so far (o is in its unit); the
                                                             // least of this lane's cells
        int k_top = 0;                                       // E4M3: the largest scale byte of K of this lane's cells
#pragma unroll
        for (int i = 0; i < ND; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

        int slot = 0;
        for (int tile = w.t0; tile < w.t1; ++tile) {
            {
                const int cur = next_pages, nt = tile + F::kStages - 1;
                next_pages = pages(nt + 1);
                issue(nt, slot == 0 ? F::kStages - 1 : slot - 1, cur);
            }
            asm volatile("cp.async.wait_group %0;" ::"n"(F::kStages - 1) : "memory");
            __syncwarp();
            const uint32_t qs = su32(smem) + F::kSmem - F::kFactors - F::kQ + lane * 16;
            const uint32_t factors = su32(smem) + F::kSmem - F::kFactors + warp * 384;
            const uint32_t st = ring + slot * F::kStageAl;
            slot = slot + 1 == F::kStages ? 0 : slot + 1;
            int start, begin, end;
            range(tile, start, begin, end);
            if (start >= end || start + WK <= begin) { __syncwarp(); continue; }
            bool split = false;
            if constexpr (E4M3) {
                // a cell's scales by its lane: K's as a factor of its scores, V's of its probabilities,
                // relative to the largest scale of V so far
                const char *sc = smem + (st - su32(smem)) + 2 * WK * F::kRow;
                const bool in = lane < WK && start + lane >= begin && start + lane < end;
                const uint32_t yk = in ? *reinterpret_cast<const uint8_t *>(sc + lane) : 0u;
                const uint32_t yv = in ? *reinterpret_cast<const uint8_t *>(sc + WK + lane) : 0u;
                k_top = max(k_top, (int)yk);                 // (a NaN's byte counts too: rows that see it are done again anyway)
                // a scale that bears on the others' precision (not a NaN's, nor that of a row of zeros)
                bool bears = in && yv != 255u;
                if constexpr (!F::kF32) {
                    if (bears && yv == 0u) {
                        uint32_t any = 0;
#pragma unroll
                        for (int c = 0; c < F::kRow; c += 16) {
                            const float4 x = lds16(st + WK * F::kRow + swz<F::kRow, false>(lane, c, true));
                            any |= __float_as_uint(x.x) | __float_as_uint(x.y) | __float_as_uint(x.z) | __float_as_uint(x.w);
                        }
                        bears = (any & 0x7F7F7F7Fu) != 0;
                    }
                    const int most = (int)__reduce_max_sync(0xffffffffu, bears ? yv : 0u);
                    if (bears) v_low = min(v_low, (int)yv);
                    if (most > v_top) {
                        const float f = scale_of((uint32_t)max(127 + v_top - most, 0));
#pragma unroll
                        for (int i = 0; i < ND; ++i) { o[i][0] *= f; o[i][1] *= f; o[i][2] *= f; o[i][3] *= f; }
                        v_top = most;
                    }
                }
                float *mine = reinterpret_cast<float *>(smem + F::kSmem - F::kFactors) + warp * 96 + lane;   // of K, of V (to the
                // probability, to the value)
                // (a scale below 2^-7 of the largest: 2^-14 .. 1 of it goes to the values instead, so that the
                // probability keeps its bits in f16)
                const int low = F::kF32 || !bears ? 0 : (int)yv - v_top;
                split = !F::kF32 && __any_sync(0xffffffffu, low < -7);
                const int to_value = split ? max(low, -14) : 0;
                mine[0] = scale_of(yk);
                mine[32] = yv == 255u || F::kF32 ? scale_of(yv) : scale_of((uint32_t)max(127 + (int)yv - v_top - to_value, 0));
                if (split) mine[64] = __uint_as_float((uint32_t)(15 + to_value) << 10);   // 2^to_value in f16
                __syncwarp();
            }

            float s[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
            if constexpr (F::kF32) {
                float sx[NT][4] = {};
#pragma unroll(DP > 128 ? 2 : 4)
                for (int i = 0; i < DP / 16; ++i) {            // 16 values of a row: two steps
                    uint32_t hi[2][4], lo[2][4];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float4 a = lds16(qs + (2 * i + e) * 512);
                        halves(a.x, hi[e][0], lo[e][0]);
                        halves(a.y, hi[e][1], lo[e][1]);
                        halves(a.z, hi[e][2], lo[e][2]);
                        halves(a.w, hi[e][3], lo[e][3]);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float4 b;
                        if (E4M3) {
                            const uint32_t c = lds4(st + swz<F::kRow, false>(n * 8 + g, i * 16, false) + 4 * t);
                            const float2 u = e4m3_values((uint16_t)c), v = e4m3_values((uint16_t)(c >> 16));
                            b = make_float4(u.x, u.y, v.x, v.y);
                        } else {
                            b = lds16(st + swz<F::kRow, true>(n * 8 + g, (4 * i + t) * 16, false));
                        }
                        mma_f32<E4M3>(s[n], sx[n], hi[0], lo[0], b.x, b.y);
                        mma_f32<E4M3>(s[n], sx[n], hi[1], lo[1], b.z, b.w);
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[n][i] += sx[n][i];
            } else if constexpr (E4M3) {
#pragma unroll
                for (int kp = 0; kp < F::kRow / 64; ++kp) {        // four 16-byte chunks of eight rows
                    float4 qa[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) qa[i] = lds16(qs + (kp * 4 + i) * 512);
                    uint32_t r[NT][4];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        ldsm4(st + swz<F::kRow, false>(n * 8 + (lane & 7), (kp * 4 + (lane >> 3)) * 16, false), r[n]);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            M::go(s[n], reinterpret_cast<const uint32_t *>(&qa[i]), widen(r[n][i] & 0xffffu), widen(r[n][i] >> 16));
                }
            } else {
#pragma unroll
                for (int kp = 0; kp < F::kRow / 64; ++kp) {
                    float4 qa[2];
                    if (F::kSharedQ) { qa[0] = lds16(qs + kp * 1024); qa[1] = lds16(qs + kp * 1024 + 512); }
                    const uint32_t *q0 = F::kSharedQ ? reinterpret_cast<const uint32_t *>(&qa[0]) : qf[F::kSharedQ ? 0 : 2 * kp];
                    const uint32_t *q1 = F::kSharedQ ? reinterpret_cast<const uint32_t *>(&qa[1]) : qf[F::kSharedQ ? 0 : 2 * kp + 1];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        uint32_t r[4];
                        ldsm4(st + swz<F::kRow, false>(n * 8 + (lane & 7), (kp * 4 + (lane >> 3)) * 16, false), r);
                        M::go(s[n], q0, r[0], r[1]);
                        M::go(s[n], q1, r[2], r[3]);
                    }
                }
            }
            // scores in powers of two, masked
            const bool open = start >= begin && start + WK <= end && start + WK - 1 <= ends[0] &&
                              (p.b.window == 0 || start > ends[1] - p.b.window);
            const float rowf[2] = {kRowFactor ? row_factor[g] : p.b.scale_log2, kRowFactor ? row_factor[g + 8] : p.b.scale_log2};
            float top[2] = {-INFINITY, -INFINITY};
            uint32_t seen = 0;                               // not open: a bit per score
            int row_pos[2] = {0, 0};
            uint32_t tree[2] = {0, 0};                       // a tree's rows: a bit per cell of the step
            if (TREE && !open) {
                const uint32_t part = bits_below(end - start) & ~bits_below(begin - start);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    tree[i] = part & tree_seen(tree_row(p.b, w.row0 + (w.r0 + min(g + 8 * i, w.rows - 1)) / p.b.group), start,
                                               p.b.window, p.b.sinks);
            } else if (!open) {
                row_pos[0] = w.pos + (w.r0 + g) / p.b.group;
                row_pos[1] = w.pos + (w.r0 + g + 8) / p.b.group;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float f0 = 1.f, f1 = 1.f;
                if (E4M3) {
                    const float2 f = lds8(factors + (n * 8 + 2 * t) * 4);
                    f0 = f.x;
                    f1 = f.y;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = E4M3 ? s[n][i] * (i & 1 ? f1 : f0) : s[n][i];
                    if (!open) {
                        const int j = start + n * 8 + 2 * t + (i & 1);
                        const bool see = TREE ? tree[i >> 1] >> (n * 8 + 2 * t + (i & 1)) & 1u
                                              : j >= begin && j < end && tok_seen(j, row_pos[i >> 1], p.b.window, p.b.sinks);
                        x = see ? x : -INFINITY;
                        seen |= (uint32_t)see << (n * 4 + i);
                    }
                    s[n][i] = x;
                    top[i >> 1] = fmaxf(top[i >> 1], x);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2)) * rowf[i];
            }
            const bool up0 = top[0] > m[0] + 15.f, up1 = top[1] > m[1] + 15.f;
            if (__any_sync(0xffffffffu, up0 || up1)) {
                const float n0 = up0 ? top[0] - 7.f : m[0], n1 = up1 ? top[1] - 7.f : m[1];
                const float k0 = up0 ? ex2(m[0] - n0) : 1.f, k1 = up1 ? ex2(m[1] - n1) : 1.f;
                m[0] = n0;
                m[1] = n1;
                l[0] *= k0;
                l[1] *= k1;
#pragma unroll
                for (int i = 0; i < ND; ++i) {
                    o[i][0] *= k0; o[i][1] *= k0;
                    o[i][2] *= k1; o[i][3] *= k1;
                }
            }
            const float ref0 = m[0] == -INFINITY ? 0.f : -m[0], ref1 = m[1] == -INFINITY ? 0.f : -m[1];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s[n][0] = ex2(fmaf(s[n][0], rowf[0], ref0));
                s[n][1] = ex2(fmaf(s[n][1], rowf[0], ref0));
                s[n][2] = ex2(fmaf(s[n][2], rowf[1], ref1));
                s[n][3] = ex2(fmaf(s[n][3], rowf[1], ref1));
                l[0] += s[n][0] + s[n][1];
                l[1] += s[n][2] + s[n][3];
            }
            if constexpr (E4M3) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float *x = s[n];
                    const float2 f = lds8(factors + (32 + n * 8 + 2 * t) * 4);
                    if (open) {
                        x[0] *= f.x; x[1] *= f.y; x[2] *= f.x; x[3] *= f.y;
                    } else {                                 // a masked cell's scale may be anything
                        const uint32_t b = seen >> (4 * n);
                        x[0] = b & 1 ? x[0] * f.x : 0.f; x[1] = b & 2 ? x[1] * f.y : 0.f;
                        x[2] = b & 4 ? x[2] * f.x : 0.f; x[3] = b & 8 ? x[3] * f.y : 0.f;
                    }
                }
            }
            const uint32_t vst = st + WK * F::kRow;
            if constexpr (F::kF32) {
                uint32_t hi[NT][4], lo[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {                 // eight cells: the step's cells 2t and 2t + 1 are this lane's
                    halves(s[n][0], hi[n][0], lo[n][0]);
                    halves(s[n][2], hi[n][1], lo[n][1]);
                    halves(s[n][1], hi[n][2], lo[n][2]);
                    halves(s[n][3], hi[n][3], lo[n][3]);
                }
                // 32 values of a row at a time: lane group g has 4g .. 4g + 3
                constexpr int VW = 4;
#pragma unroll
                for (int J = 0; J < DP / 8; J += VW) {
                    // A step's products in accumulators of their own, added to the sums by rounded fp32
                    // additions: the tensor cores' truncate, and a long axis has thousands of them (of 256 values: 12 to
                    // 15 % of the time; sums straight in the accumulators were off by 7e-4 over 300,000 cells)
                    float d[VW][4] = {};
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float c[2][4];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int row = n * 8 + 2 * t + e;
                            if (E4M3) {
                                const uint32_t u = lds4(vst + swz<F::kRow, false>(row, (J / 4 * 2 + g / 4) * 16, true) + g % 4 * 4);
                                const float2 x = e4m3_values((uint16_t)u), y = e4m3_values((uint16_t)(u >> 16));
                                c[e][0] = x.x; c[e][1] = x.y; c[e][2] = y.x; c[e][3] = y.y;
                            } else {
                                const float4 x = lds16(vst + swz<F::kRow, true>(row, (J / 4 * 8 + g) * 16, true));
                                c[e][0] = x.x; c[e][1] = x.y; c[e][2] = x.z; c[e][3] = x.w;
                            }
                        }
                        uint32_t h0[VW], l0[VW], h1[VW], l1[VW];
#pragma unroll
                        for (int i = 0; i < VW; ++i) {
                            halves(c[0][i], h0[i], l0[i]);
                            halves(c[1][i], h1[i], l1[i]);
                        }
#pragma unroll
                        for (int i = 0; i < VW; ++i) mma_tf32(d[i], lo[n], h0[i], h1[i]);
                        if (!E4M3) {
#pragma unroll
                            for (int i = 0; i < VW; ++i) mma_tf32(d[i], hi[n], l0[i], l1[i]);
                        }
#pragma unroll
                        for (int i = 0; i < VW; ++i) mma_tf32(d[i], hi[n], h0[i], h1[i]);
                    }
#pragma unroll
                    for (int i = 0; i < VW; ++i)
#pragma unroll
                        for (int k = 0; k < 4; ++k) o[J + i][k] += d[i][k];
                }
            } else {
            auto products = [&](auto with_split) {
                constexpr bool kSplit = decltype(with_split)::value;
#pragma unroll
                for (int kg = 0; kg < WK / 16; ++kg) {
                    uint32_t a[4], vs[2] = {0, 0};
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        const float *x = s[2 * kg + hh];
                        a[2 * hh] = M::pack(x[0], x[1]);
                        a[2 * hh + 1] = M::pack(x[2], x[3]);
                        if (kSplit) {
                            const float2 f = lds8(factors + (64 + kg * 16 + hh * 8 + 2 * t) * 4);
                            vs[hh] = __float_as_uint(f.x) | __float_as_uint(f.y) << 16;
                        }
                    }
#pragma unroll
                    for (int c = 0; c < F::kRow / 16; c += 2) {
                        uint32_t r[4];
                        ldsm4t(vst + swz<F::kRow, false>(kg * 16 + (lane & 15), (c + (lane >> 4)) * 16, true), r);
                        if (E4M3) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                uint32_t e0 = widen(__byte_perm(r[2 * i], 0, 0x4420)), e1 = widen(__byte_perm(r[2 * i + 1], 0, 0x4420));
                                uint32_t u0 = widen(__byte_perm(r[2 * i], 0, 0x4431)), u1 = widen(__byte_perm(r[2 * i + 1], 0, 0x4431));
                                if (kSplit) {
                                    e0 = hmul2(e0, vs[0]); u0 = hmul2(u0, vs[0]);
                                    e1 = hmul2(e1, vs[1]); u1 = hmul2(u1, vs[1]);
                                }
                                M::go(o[2 * (c + i)], a, e0, e1);
                                M::go(o[2 * (c + i) + 1], a, u0, u1);
                            }
                        } else {
                            M::go(o[c], a, r[0], r[1]);
                            M::go(o[c + 1], a, r[2], r[3]);
                        }
                    }
                }
            };
            if (E4M3 && split) products(std::true_type{});
            else products(std::false_type{});
            }
            __syncwarp();
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
        }
        __syncthreads();                                     // every warp is done with its ring
        // the warps' sums, maxima and sums of powers, [warp][row][DP + 2]
        float *join = reinterpret_cast<float *>(smem);
        constexpr int JR = DP + 2;
        const float unit = E4M3 && !F::kF32 ? scale_of((uint32_t)v_top) : 1.f;
        // Scales of V further apart than kSpread: probabilities of the smallest ones' cells no longer fit f16, and
        // the largest may be of a cell that a row does not see, or that adds nothing to it.
        const bool far = E4M3 && __any_sync(0xffffffffu, (!F::kF32 && v_top - v_low > kSpread) || k_top > kMostScaleK);
        int bad = 0;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float *row = join + (warp * kFewRows + g + half * 8) * JR;
            bool fine = l[half] < INFINITY && !isnan(m[half]);
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                const int d = F::kF32 ? (i >> 2) * 32 + 8 * t + (i & 3) : E4M3 ? (i >> 1) * 16 + 4 * t + (i & 1) : i * 8 + 2 * t;
                const float x0 = o[i][2 * half] * unit, x1 = o[i][2 * half + 1] * unit;
                fine = fine && fabsf(x0) < INFINITY && fabsf(x1) < INFINITY;
                row[d] = x0;
                row[d + (F::kF32 ? 4 : E4M3 ? 2 : 1)] = x1;
            }
            if (t == 0) { row[DP] = m[half]; row[DP + 1] = l[half]; }
            bad |= (far || !fine) && g + half * 8 < w.rows;
        }
        const int chunks = D / 8;
        // rows whose sums are not numbers, or have lost bits to far larger scales, are done again by the definition,
        // from the cells they may attend to alone: a masked cell's NaN or infinity has met a probability of 0
        if (__syncthreads_or(bad)) {
            const int j0 = w.t0 < nA ? w.t0 * F::kTile : max(w.b0, b_al + (w.t0 - nA) * F::kTile);
            const int j1 = w.t1 <= nA ? min(w.a1, w.t1 * F::kTile) : min(w.b1, b_al + (w.t1 - nA) * F::kTile);
            for (int r = warp; r < w.rows; r += kWarps) {
                const int rr = w.r0 + r;
                const T *q = reinterpret_cast<const T *>(p.q.p) + (int64_t)(w.row0 + rr / p.b.group) * p.q.ts +
                             (int64_t)(w.h * p.b.group + rr % p.b.group) * p.q.hs;
                float x[8], mm, ll;
                TreeRow tree{};
                if (TREE) tree = tree_row(p.b, w.row0 + rr / p.b.group);
                attend_row<T, E4M3, TREE>(p.pool, p.b.table + w.table0, w.h, q, p.q.vec, TREE ? tree.pos : w.pos + rr / p.b.group, j0, j1,
                                          p.b.window, p.b.sinks, p.b.scale_log2, x, mm, ll, tree);
                for (int k = 0; k < kWarps; ++k) {
                    float *row = join + (k * kFewRows + r) * JR;
                    if (lane * 8 < D) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) row[lane * 8 + i] = k == 0 ? x[i] : 0.f;
                    }
                    if (lane == 0) { row[DP] = k == 0 ? mm : -INFINITY; row[DP + 1] = k == 0 ? ll : 0.f; }
                }
            }
            __syncthreads();
        }
        float *wt = join + kWarps * kFewRows * JR;             // (past the joined sums)
        // The weight of each of n parts of a row, at wt[row * n + i], and the row's maximum and sum of
        // powers: a thread per row for the block's own parts, a warp per row (parts along the lanes) for a
        // cut unit's.  src: a row's parts `step` apart.
        auto done = [&](int r, float mm, float ll, bool last_join) {
            if (last_join) {
                const int rr = w.r0 + r;
                if (p.lse)
                    p.lse[(int64_t)(w.row0 + rr / p.b.group) * p.b.n_heads + w.h * p.b.group + rr % p.b.group] =
                        ll == 0.f ? -INFINITY : (mm + log2f(ll)) * 0.693147180559945f;
            } else {
                float *mine = p.w.part + ((int64_t)w.part * kFewRows + r) * JR;
                mine[DP] = mm;
                mine[DP + 1] = ll;
            }
        };
        auto weigh_own = [&](bool last_join) {
            if ((int)threadIdx.x < w.rows) {
                const int r = threadIdx.x;
                float v[kWarps], mm = -INFINITY, ll = 0.f;
                bool nan = false;
#pragma unroll
                for (int i = 0; i < kWarps; ++i) {
                    v[i] = join[(i * kFewRows + r) * JR + DP];
                    nan = nan || isnan(v[i]);
                    mm = fmaxf(mm, v[i]);
                }
                mm = nan ? NAN : mm;
                const float ref = mm == -INFINITY ? 0.f : mm;
#pragma unroll
                for (int i = 0; i < kWarps; ++i) {
                    v[i] = ex2(v[i] - ref);
                    ll = fmaf(v[i], join[(i * kFewRows + r) * JR + DP + 1], ll);
                }
                const float inv = !last_join ? 1.f : ll == 0.f ? 0.f : 1.f / ll;
#pragma unroll
                for (int i = 0; i < kWarps; ++i) wt[r * kWarps + i] = v[i] * inv;
                done(r, mm, ll, last_join);
            }
            __syncthreads();
        };
        auto weigh = [&](const float *src, int64_t step, int n) {
            for (int r = warp; r < w.rows; r += kWarps) {
                float mm = -INFINITY, ll = 0.f;
                bool nan = false;
                for (int i = lane; i < n; i += 32) {
                    const float v = src[i * step + r * JR + DP];
                    wt[r * n + i] = v;
                    nan = nan || isnan(v);
                    mm = fmaxf(mm, v);
                }
#pragma unroll
                for (int s = 16; s; s >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, s));
                mm = __any_sync(0xffffffffu, nan) ? NAN : mm;
                const float ref = mm == -INFINITY ? 0.f : mm;
                for (int i = lane; i < n; i += 32) {
                    const float f = ex2(wt[r * n + i] - ref);
                    wt[r * n + i] = f;
                    ll = fmaf(f, src[i * step + r * JR + DP + 1], ll);
                }
#pragma unroll
                for (int s = 16; s; s >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, s);
                const float inv = ll == 0.f ? 0.f : 1.f / ll;
                for (int i = lane; i < n; i += 32) wt[r * n + i] *= inv;
                if (lane == 0) done(r, mm, ll, true);
            }
            __syncthreads();
        };
        // eight of a row's values, weighed and added in the order of the parts
        auto joined = [&](const float *src, int64_t step, int n, const float *wt, float *x) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
                const float2 *y = reinterpret_cast<const float2 *>(src + i * step);
                const float2 y0 = y[0], y1 = y[1], y2 = y[2], y3 = y[3];
                const float f = wt[i];
                x[0] = fmaf(f, y0.x, x[0]); x[1] = fmaf(f, y0.y, x[1]); x[2] = fmaf(f, y1.x, x[2]); x[3] = fmaf(f, y1.y, x[3]);
                x[4] = fmaf(f, y2.x, x[4]); x[5] = fmaf(f, y2.y, x[5]); x[6] = fmaf(f, y3.x, x[6]); x[7] = fmaf(f, y3.y, x[7]);
            }
        };
        const float *src = join;
        int64_t step = kFewRows * JR;
        int n = kWarps;
        if (w.parts > 1) {
            weigh_own(false);
            float *mine = p.w.part + (int64_t)w.part * kFewRows * JR;
            for (int u = threadIdx.x; u < w.rows * chunks; u += kWarps * 32) {
                const int r = u / chunks, c = (u % chunks) * 8;
                float x[8];
                joined(src + r * JR + c, step, n, wt + r * n, x);
#pragma unroll
                for (int i = 0; i < 8; i += 2) *reinterpret_cast<float2 *>(mine + r * JR + c + i) = make_float2(x[i], x[i + 1]);
            }
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) {
                last = atomicAdd(p.w.count + w.unit, 1) == w.parts - 1;
                if (last) p.w.count[w.unit] = 0;
            }
            __syncthreads();
            if (!last) continue;                             // (the barrier above is the item's last)
            __threadfence();
            src = p.w.part + (int64_t)w.part0 * kFewRows * JR;
            n = w.parts;
            wt = join;
            weigh(src, step, n);
        } else {
            weigh_own(true);
        }
        for (int u = threadIdx.x; u < w.rows * chunks; u += kWarps * 32) {
            const int r = u / chunks, c = (u % chunks) * 8, rr = w.r0 + r;
            float x[8];
            joined(src + r * JR + c, step, n, wt + r * n, x);
            const int token = w.row0 + rr / p.b.group, head = w.h * p.b.group + rr % p.b.group;
            store8(reinterpret_cast<T *>(p.out.p) + token * p.out.ts + head * p.out.hs + c, p.out.vec, x);
        }
        __syncthreads();                                     // the joined sums' memory is the next ring
    }
}

template <class T, bool E4M3, int DP, bool TREE>
int go(const FewParams &p, cudaStream_t s)
{
    using F = Few<T, E4M3, DP>;
    allow_dynamic_smem_once<k_tokens_few<T, E4M3, DP, TREE>>(F::kSmem);
    k_tokens_few<T, E4M3, DP, TREE><<<p.w.blocks, kWarps * 32, F::kSmem, s>>>(p);
    return 1;
}

template <class T, bool E4M3, int DP>
int go(const FewParams &p, cudaStream_t s)
{
    return p.b.node ? go<T, E4M3, DP, true>(p, s) : go<T, E4M3, DP, false>(p, s);
}

template <class T, bool E4M3>
int by_dim(const FewParams &p, cudaStream_t s)
{
    if (p.pool.d <= 64) return go<T, E4M3, 64>(p, s);
    if (p.pool.d <= 128) return go<T, E4M3, 128>(p, s);
    return go<T, E4M3, 256>(p, s);
}

}  // namespace

template <class T, bool E4M3>
static FewShape shape_of(int d)
{
    if (d <= 64) return {Few<T, E4M3, 64>::kTile, Few<T, E4M3, 64>::kBlocks};
    if (d <= 128) return {Few<T, E4M3, 128>::kTile, Few<T, E4M3, 128>::kBlocks};
    return {Few<T, E4M3, 256>::kTile, Few<T, E4M3, 256>::kBlocks};
}

FewShape few_shape(int dtype, int form, int d)
{
    const bool e = form == MURE_FORM_E4M3;
    FewShape f = dtype == MURE_F32 ? (e ? shape_of<float, true>(d) : shape_of<float, false>(d))
                                   : (e ? shape_of<__half, true>(d) : shape_of<__half, false>(d));
    f.blocks *= sm_count();
    return f;
}

int few_part_floats(int d) { return kFewRows * ((d <= 64 ? 64 : d <= 128 ? 128 : 256) + 2); }

int launch_tokens_few(const TokPool &pool, const TokBatch &b, const TokWork &w, int dtype, int form, TokRows q, TokRows out,
                      float *lse, cudaStream_t s)
{
    if (w.blocks == 0) return 0;
    const FewParams p{pool, b, w, q, out, lse};
    const bool e = form == MURE_FORM_E4M3;
    if (dtype == MURE_F32) return e ? by_dim<float, true>(p, s) : by_dim<float, false>(p, s);
    if (dtype == MURE_F16) return e ? by_dim<__half, true>(p, s) : by_dim<__half, false>(p, s);
    return e ? by_dim<__nv_bfloat16, true>(p, s) : by_dim<__nv_bfloat16, false>(p, s);
}

}  // namespace mure
