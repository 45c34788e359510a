// Token caches: attention of chunks of new tokens in 16-bit types on the 5th-generation tensor cores.
//
// A CTA takes up to 256 rows (new token, query head) of one sequence and cached head, as two tiles
// of 128, over tiles of 128 cells:
//   S = Q K^T    tcgen05, both operands from shared memory, S in tensor memory;
//   P = 2^(s - m) in 16 bits, written over half of S in tensor memory;
//   O += P V     tcgen05, P from tensor memory, V from shared memory (its rows are the product's
//                K axis: an MN-major operand), O in tensor memory.
// While the softmax of one tile of rows runs on the CUDA cores, the tensor pipe works on the other
// tile's products.  Warps:
//   0-3, 4-7  softmax of the two row tiles, a thread per row: no shuffles; they also fetch Q and
//             write the rows out;
//   8, 11     issue the MMAs of either row tile;
//   9, 10     copy K and V tiles by tensor maps, a box per page (or 128 cells of a larger page);
//   12-15     (on codes) widen them, see below.
// What a row's scores are taken relative to lies 7 below their running maximum and moves only when that
// grows by more than 8 (in powers of two; f16 holds powers up to 2^15, and those down to 2^-21 of the
// largest keep all its bits), so O is hardly ever rescaled; where it is, S's arrival (or, where P lies
// beside S, a barrier of the product's own) has shown that every earlier product is done.  Whole units of work
// go to the CTAs, the longest first; the ones that do not fit an even share are cut along the cells and joined
// by a second kernel in the order of their parts.
//
// One pass over the cells with a running maximum and sum is the online softmax of Milakov and Gimelshein (2018),
// with attention's sums carried along as Rabe and Staats (2021) do.  P is rounded to the cells' type because
// that is what the product takes (as low halves of its own it would cost a third more tensor work); the row's
// sum is of the powers before that rounding, and everything else is held in fp32: 1.35 to 1.4 times the error of
// an output rounded once.  Powers come from the hardware's approximation (2 units in fp32's last place).
// Every wait is bounded, as in the GEMM kernel.
//
// Measured (GB300): 8,192 new tokens over 16,384 cells, 32 heads of 128 bf16 values on 8: 1,155 to 1,184 us,
// 1,390 to 1,430 TFLOP/s (0.74 to 0.76 of cuBLAS's burst rate); a 256 x 128 tile takes 2,750 cycles, the
// tensor pipe is busy for 2,270.  Twelve ragged chunks of 90 to 700 tokens over up to 6,000 cells: 261 us
// (pieces of a few dozen tiles, 12,000 cycles of beginning and end each).  Chunks within a window
// (64 values): 72 us: the softmax's latency, 1,800 cycles per tile of which 1,024 exponentials, and a beginning
// and end for every ten tiles, not measured by themselves for 64 values.
//
// Trees (TREE): a row sees all cells before its sequence's new ones that its position allows, and of the new ones' those
// whose bits are set.  On e4m3 cells (CODES) a tree's pieces may widen the codes themselves: warp 9 copies tiles of codes into
// slots of their own, and warps 12 to 15 turn them into the 16-bit tiles that the products read, a thread per cell.
// Widening whole pages first moves 5 bytes for each code, which only readers of a page in numbers are worth: 48 trees of 17
// to 64 tokens over 500 to 6,000 cells of 8 heads of 128, 345 us so (191 of them the widening), 189 us by the pieces
// themselves.  What bounds these is the chain from a tile of codes to the products (2.75 us per tile of 256 rows; the same
// with the codes copied as they are, 2.4 us without touching them), not the conversions.  Trees of 200 to 256 rows over
// 100,000 to 131,000 cells of 16 bits: 187 to 202 us and 8 to 12 for the join, 201 to 221 both (one card and another), 4.4 to 4.9
// TB/s, 1.75 us per tile as in any chunk.
#include <type_traits>

#include "simt_tile.cuh"
#include "tokens_tc.cuh"

namespace mure {

namespace {

// CODES: the cells are e4m3 codes, widened on their way to the products (trees, whose cells are read once or little more).
template <int DP, bool CODES>
struct Chunk {
    static constexpr int kThreads = CODES ? 512 : 384;
    static constexpr int kPanels = DP / 64;
    static constexpr uint32_t kQ = 2 * kPanels * kPanel;            // two row tiles
    static constexpr uint32_t kStage = kPanels * kPanel;            // a K or V tile
    static constexpr int kStages = DP == 64 ? 8 : CODES ? 3 : 4;
    static constexpr uint32_t kK = CODES && DP == 128 ? 1 : kStages / 2, kV = kStages - kK;    // of K, and of V behind them
    // Tensor memory: S of both row tiles in columns 0 .. 255, O from 256.  P lies over half of S, or for
    // up to 64 values, where O leaves room, beside it: the next scores then need not wait for P V.
    static constexpr bool kApart = DP == 64;
    static __device__ __forceinline__ uint32_t col_p(int h) { return kApart ? 384 + h * 64 : h * 128 + 64; }
    static __device__ __forceinline__ uint32_t col_o(int h) { return 256 + h * DP; }
    // CODES: tiles of codes that are copied ahead of their widening
    static constexpr uint32_t kSlot = kCells * DP, kSlots = !CODES ? 1 : DP == 64 ? 6 : 4;
    static constexpr uint32_t kSmem = kQ + kStages * kStage + (CODES ? kSlots * kSlot : 0) + 1024; // (+ room to align to 1024)
};

// Two e4m3 codes of a cell whose scale byte is `byte` as 16-bit values, as the cells' pages widened whole would hold them.
// Scales at which every product is exact and in range (from 2^-15; to 2^7 for f16, to 2^15 for bf16) go by 16-bit
// factors, f16's codes by one product for both, bf16's by one for each into fp32; others by fp32 (bits shifted into
// place and a product of both for bf16, which need a look for NaNs beside: 64 trees' tiles 208 -> 231 us).
template <class T>
struct Widen {
    static constexpr bool kHalf = std::is_same<T, __half>::value;
    static __device__ __forceinline__ bool fast(uint32_t byte) { return byte - 112u <= (kHalf ? 22u : 30u); }
    static __device__ __forceinline__ uint32_t unit(uint32_t byte)      // 2^(byte - 127), 2^-15 is subnormal
    {
        return byte == 112u ? 0x02000200u : (byte - 112u) * 0x04000400u;
    }
    static __device__ __forceinline__ uint32_t pair(uint32_t four, uint32_t which, uint32_t unit)
    {
        uint32_t h, r;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(which ? four >> 16 : four)));
        if constexpr (kHalf) asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(h), "r"(unit));
        else {
            float lo, hi;
            asm("fma.rn.f32.f16 %0, %1, %2, %3;" : "=f"(lo) : "h"((uint16_t)h), "h"((uint16_t)unit), "f"(-0.f));
            asm("fma.rn.f32.f16 %0, %1, %2, %3;" : "=f"(hi) : "h"((uint16_t)(h >> 16)), "h"((uint16_t)unit), "f"(-0.f));
            r = narrow2<T>(lo, hi);
        }
        return r;
    }
};

struct ChunkParams {
    TokPool pool;
    TokBatch b;
    TokWork w;
    TokRows q, out;
    float *lse;
    float *ml;               // partial results' maxima and sums, [parts][256][2]
    int64_t n_pages;
    int box;                 // cells of a copied box
    TokPool codes;           // widened cells: where they were widened from,
    const int32_t *code_table = nullptr;      // and the pages there (null: the cells are what the caches hold)
    int *err;
    long long spin;
    CUtensorMap map_k, map_v;
};

// A value of a widened page: what f16 does not reach is a NaN.
template <class T>
__device__ __forceinline__ float widened(float x) { return std::is_same<T, __half>::value && !(fabsf(x) <= 65504.f) ? NAN : x; }

template <class T, int DP, bool TREE, bool CODES>
__global__ void __launch_bounds__(Chunk<DP, CODES>::kThreads, 1) k_tokens_chunk(const __grid_constant__ ChunkParams p)
{
    using C = Chunk<DP, CODES>;
    extern __shared__ char smem_raw[];
    // the first kK stages hold K tiles, the others V tiles
    __shared__ __align__(8) uint64_t bar_full[C::kStages], bar_empty[C::kStages], bar_q[2], bar_s[2], bar_p[2][2], bar_o[2], bar_pv[2], bar_turn[2], bar_drain[2];
    __shared__ uint32_t tmem_sh;
    __shared__ int again_sh;                  // rows are marked
    __shared__ WaitCtl ctl_sh;
    __shared__ __align__(8) uint64_t bar_code[C::kSlots], bar_read[C::kSlots];   // codes there, and read
    __shared__ TokItem item_sh[C::kThreads / 32];   // each warp's piece of work
    __shared__ TokItem copy_sh;               // CODES: the copies' piece of work
    __shared__ int page_sh[2][2][16];         // copying warps: the pages of a tile's boxes
    volatile WaitCtl *ctl = &ctl_sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_smem = base, ring = base + C::kQ;
    const int D = p.pool.d;

    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_sh)), "r"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (threadIdx.x == 0) {
        again_sh = 0;
        ctl_sh.abort = 0;
        ctl_sh.limit = p.spin > 0 ? p.spin : kSpin;
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(smem_u32(&bar_full[i]), CODES ? 4 : 1);
            mbar_init(smem_u32(&bar_empty[i]), 2);      // the products of both row tiles
        }
        for (int h = 0; h < 2; ++h) {
            mbar_init(smem_u32(&bar_q[h]), 4);
            mbar_init(smem_u32(&bar_s[h]), 1);
            mbar_init(smem_u32(&bar_p[h][0]), 4);
            mbar_init(smem_u32(&bar_p[h][1]), 4);
            mbar_init(smem_u32(&bar_o[h]), 1);
            mbar_init(smem_u32(&bar_pv[h]), 1);
            mbar_init(smem_u32(&bar_turn[h]), 1);
            mbar_init(smem_u32(&bar_drain[h]), 1);
        }
        for (uint32_t i = 0; i < C::kSlots; ++i) {
            mbar_init(smem_u32(&bar_code[i]), 1);
            mbar_init(smem_u32(&bar_read[i]), 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_sh;
    const int it0 = p.w.first[blockIdx.x], it1 = p.w.first[blockIdx.x + 1];
    const TokItem &w = item_sh[warp];
    auto take = [&](int it) {
        __syncwarp();
        if (lane < (int)sizeof(TokItem) / 4)
            reinterpret_cast<int32_t *>(&item_sh[warp])[lane] = __ldg(reinterpret_cast<const int32_t *>(p.w.items + it) + lane);
        __syncwarp();
    };

    if (warp < 8) {
        // ------------------------------------------------------------------ softmax --
        const int h = warp >> 2, r = threadIdx.x & 127;              // row tile, row of it
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lanes + h * 128, tP = tmem + lanes + C::col_p(h), tO = tmem + lanes + C::col_o(h);
        const uint32_t qs = q_smem + h * C::kPanels * kPanel;
        uint32_t n_s = 0, n_o = 0;                                   // phases waited for
        bool ok = true;
        for (int it = it0; it < it1 && ok; ++it) {
            take(it);
            const int rows = w.rows;
            if (h * 128 >= rows) continue;
            const int r0 = w.r0 + h * 128, t0 = w.t0, t1 = w.t1, pos = w.pos;
            const int row = r0 + r;
            const bool real = h * 128 + r < rows;
            const bool have = t1 > t0;                               // (no cells: zeros, no products)
            // Q into the K-major swizzled tile (all products with the last one have finished), the lanes
            // of a warp along the rows: kLanes 16-byte chunks of one row, the next rows beside it.  Rows without
            // cells leave Q and its barrier alone: every arrival is then followed by a wait for this piece's first
            // scores, so that the issuing warp is never more than one phase behind (a parity names no more).
            constexpr int kLanes = DP / 8, kPer = 32 / kLanes;
            const int chunk = lane % kLanes;
            if (have) {
                const int64_t q_at = real ? (w.row0 + row / p.b.group) * p.q.ts + (w.h * p.b.group + row % p.b.group) * p.q.hs : -1;
                uint4 v[kLanes];
#pragma unroll
                for (int i = 0; i < kLanes; ++i) {                   // (all on their way before the first is stored)
                    const int64_t off = __shfl_sync(0xffffffffu, q_at, i * kPer + lane / kLanes);
                    v[i] = make_uint4(0, 0, 0, 0);
                    if (off < 0 || chunk * 8 >= D) continue;
                    const T *q = reinterpret_cast<const T *>(p.q.p) + off + chunk * 8;
                    if (p.q.vec) v[i] = __ldg(reinterpret_cast<const uint4 *>(q));
                    else {
                        const uint16_t *u = reinterpret_cast<const uint16_t *>(q);
                        v[i].x = u[0] | (uint32_t)u[1] << 16; v[i].y = u[2] | (uint32_t)u[3] << 16;
                        v[i].z = u[4] | (uint32_t)u[5] << 16; v[i].w = u[6] | (uint32_t)u[7] << 16;
                    }
                }
#pragma unroll
                for (int i = 0; i < kLanes; ++i)
                    st_shared16(qs + (chunk >> 3) * kPanel + sw128_off((r & ~31) + i * kPer + lane / kLanes, chunk & 7), v[i]);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_q[h]));
            }

            const int at = pos + row / p.b.group;                                  // the row's position
            // (a tree's rows see all cells before its own, and lie no further than a chain's)
            const int lo = TREE ? pos - 1 : pos + r0 / p.b.group, hi = pos + (r0 + 127) / p.b.group;
            TreeRow tree{};
            if (TREE) tree = tree_row(p.b, w.row0 + min(row, w.r0 + rows - 1) / p.b.group);
            float m = -INFINITY, l = 0.f;
            for (int t = t0; t < t1; ++t) {
                const TileCells tc = tile_cells(w, t, p.box);
                const bool open = tc.start + kCells <= tc.end && tc.start + kCells - 1 <= lo &&
                                  (p.b.window == 0 || tc.start > hi - p.b.window);
                ok = warp_wait(smem_u32(&bar_s[h]), n_s & 1, ctl);
                if (!ok) break;
                ++n_s;
                fence_after();
                // a cell of the tile a row may attend to: i <= last and (i >= first or i < sink)
                const int last = min(tc.end - 1, at) - tc.start, sink = p.b.sinks - tc.start;
                const int first = p.b.window ? at - p.b.window + 1 - tc.start : 0;
                auto mask = [&](uint32_t *x, int i0) {               // 32 cells: a bit each
                    if (open) return;
                    auto below = [&](int n) { return n <= i0 ? 0u : n >= i0 + 32 ? ~0u : (1u << (n - i0)) - 1u; };
                    const uint32_t bits = TREE ? below(tc.end - tc.start) & tree_seen(tree, tc.start + i0, p.b.window, p.b.sinks) : below(last + 1) & (~below(first) | below(sink));
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = bits & (1u << i) ? x[i] : 0xFF800000u;
                };
                // short: at most 64 cells take part (sinks, ends)
                auto softmax = [&](auto of_short) {
                constexpr bool kShort = decltype(of_short)::value;
                // The maximum of the scores; those of the second 64 cells stay in registers.
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                uint32_t s[64];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (c == 1 && kShort) continue;
                    tmem_ld32(tS + c * 64, s);
                    tmem_ld32(tS + c * 64 + 32, s + 32);
                    tmem_wait_ld();
                    mask(s, c * 64);
                    mask(s + 32, c * 64 + 32);
#pragma unroll
                    for (int i = 0; i < 64; ++i) top[i & 3] = fmaxf(top[i & 3], __uint_as_float(s[i]));
                }
                const float mt = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * p.b.scale_log2;
                // the product before (the last piece's at first, whose arrival no other wait stands for) has read P and
                // added to O
                if (C::kApart && n_s > 1) {
                    ok = warp_wait(smem_u32(&bar_pv[h]), (n_s - 2) & 1, ctl);
                    if (!ok) return;
                    fence_after();
                }
                const bool up = mt > m + 15.f;
                if (__any_sync(0xffffffffu, up)) {
                    const float mn = up ? mt - 7.f : m, keep = up ? ex2(m - mn) : 1.f;
                    m = mn;
                    l *= keep;
                    if (t > t0) {
#pragma unroll 1
                        for (int c = 0; c < D; c += 8) {             // (few at a time: the scores are in registers)
                            uint32_t x[8];
                            tmem_ld8(tO + c, x);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * keep);
                            tmem_st8(tO + c, x);
                        }
                    }
                }
                const float ref = m == -INFINITY ? 0.f : -m;
                const f32x2 scale2 = pack2(p.b.scale_log2, p.b.scale_log2), ref2 = pack2(ref, ref);
                f32x2 sum = 0;
                // powers of 32 scores -> 16 columns of P
                auto powers = [&](const uint32_t *x, uint32_t to) {
                    uint32_t y[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 e = unpack2(fma2(pack2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), scale2, ref2));
                        const float e0 = ex2(e.x), e1 = ex2(e.y);
                        sum = add2(sum, pack2(e0, e1));
                        y[i] = narrow2<T>(e0, e1);
                    }
                    tmem_st16(to, y);
                };
                // P lies over the scores of the second 64 cells, which go first; those of the first 64 are
                // fetched once more.  The products with all but cells 32 .. 63 start as soon as those are there.
                uint32_t x[32];
                tmem_ld32(tS, x);
                if (!kShort) {
                    powers(s, tP + 32);
                    powers(s + 32, tP + 48);
                }
                tmem_wait_ld();
                mask(x, 0);
                powers(x, tP);
                tmem_ld32(tS + 32, x);
                tmem_wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_p[h][1]));
                tmem_wait_ld();
                mask(x, 32);
                powers(x, tP + 16);
                l += unpack2(sum).x + unpack2(sum).y;
                tmem_wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_p[h][0]));
                };
                // (with D = 128 the second body's registers cost more than the short tiles: 1,170 -> 1,207 us)
                if (DP == 64 && tc.end - tc.start <= 64) softmax(std::integral_constant<bool, DP == 64>{});
                else softmax(std::false_type{});
                if (!ok) break;
            }
            if (!ok) break;
            // the next piece's row of Q, to be at hand when this one's rows are out (not in registers: with
            // 64 of them kept for it the rest spills)
            const TokItem *after = p.w.items + min(it + 1, it1 - 1);
            const int next_r0 = __ldg(&after->r0) + h * 128 + r, next_rows = __ldg(&after->rows);
            const int next_row0 = __ldg(&after->row0), next_h = __ldg(&after->h);
            if (have) {
                ok = warp_wait(smem_u32(&bar_o[h]), n_o & 1, ctl);
                if (!ok) break;
                ++n_o;
                fence_after();
            }
            if (it + 1 < it1 && h * 128 + r < next_rows) {
                const T *q = reinterpret_cast<const T *>(p.q.p) + (next_row0 + next_r0 / p.b.group) * p.q.ts +
                             (next_h * p.b.group + next_r0 % p.b.group) * p.q.hs;
                asm volatile("prefetch.global.L1 [%0];" ::"l"(q));
                if (D > 64) asm volatile("prefetch.global.L1 [%0];" ::"l"(q + 64));
            }
            const int parts = w.parts, part = w.part;
            const int token = w.row0 + row / p.b.group, head = w.h * p.b.group + row % p.b.group;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            bool bad = !(fabsf(l) < INFINITY) || isnan(m);
            // The rows leave through the warp's part of Q's tile (no product reads it any more), in its
            // swizzle: the lanes then lie along the rows again.  Partial results (fp32) in two passes.
            const int64_t out_at = !real ? -1 : parts > 1 ? ((int64_t)part * 256 + h * 128 + r) * DP
                                                          : token * p.out.ts + head * p.out.hs;
            for (int pass = 0; pass < (parts > 1 ? 2 : 1); ++pass) {
                __syncwarp();
                const int c0 = pass * (DP / 2), c1 = parts > 1 ? c0 + DP / 2 : DP;
#pragma unroll 1
                for (int c = c0; c < c1; c += 32) {
                    uint32_t x[32];
                    if (have) {
                        tmem_ld32(tO + c, x);
                        tmem_wait_ld();
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = 0u;
                    }
#pragma unroll
                    for (int k = 0; k < 32; k += 8) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) bad = bad || (c + k < D && !(fabsf(__uint_as_float(x[k + i])) < INFINITY));
                        if (parts > 1) {
#pragma unroll
                            for (int i = 0; i < 8; i += 4) {
                                const int at = (c - c0 + k + i) / 4;       // 16-byte chunk of the row's DP / 2 sums
                                st_shared16(qs + (at >> 3) * kPanel + sw128_off(r, at & 7),
                                            make_uint4(x[k + i], x[k + i + 1], x[k + i + 2], x[k + i + 3]));
                            }
                        } else {
                            uint32_t y[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                y[i] = narrow2<T>(__uint_as_float(x[k + 2 * i]) * inv, __uint_as_float(x[k + 2 * i + 1]) * inv);
                            const int at = (c + k) / 8;
                            st_shared16(qs + (at >> 3) * kPanel + sw128_off(r, at & 7), make_uint4(y[0], y[1], y[2], y[3]));
                        }
                    }
                }
                __syncwarp();
#pragma unroll 8
                for (int i = 0; i < 32; i += kPer) {
                    const int64_t off = __shfl_sync(0xffffffffu, out_at, i + lane / kLanes);
                    const uint4 v = ld_shared16(qs + (chunk >> 3) * kPanel + sw128_off((r & ~31) + i + lane / kLanes, chunk & 7));
                    if (off < 0) continue;
                    if (parts > 1) {
                        *reinterpret_cast<uint4 *>(p.w.part + off + c0 + chunk * 4) = v;
                    } else if (chunk * 8 < D) {
                        T *o = reinterpret_cast<T *>(p.out.p) + off + chunk * 8;
                        if (p.out.vec) *reinterpret_cast<uint4 *>(o) = v;
                        else {
                            uint16_t *u = reinterpret_cast<uint16_t *>(o);
                            const uint32_t e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k) { u[2 * k] = (uint16_t)e[k]; u[2 * k + 1] = (uint16_t)(e[k] >> 16); }
                        }
                    }
                }
            }
            if (real) {
                if (parts > 1) {
                    float *ml = p.ml + ((int64_t)part * 256 + h * 128 + r) * 2;
                    ml[0] = m;
                    ml[1] = l;
                } else if (p.lse) {
                    p.lse[(int64_t)token * p.b.n_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945f;
                }
            }
            // rows whose sums are not numbers are marked, to be done again once every role is through
            const uint32_t again = __ballot_sync(0xffffffffu, bad && real);
            if (lane == 0) {
                p.w.again[(int64_t)it * (kChunkRows / 32) + warp] = again;
                if (again) again_sh = 1;
            }
        }
    } else if (warp == 8 || warp == 11) {
        // ------------------------------------------- MMA issue: warp 8 rows 0-127, warp 11 the others --
        // The two take turns, a turn being a tile's P V and the next tile's Q K^T, handed over half-way
        // through the latter: each row tile's softmax then runs while the other one's products do.
        // Measured per 256 rows x 128 cells (D = 128; 2,270 cycles of tensor pipe): one warp for both 3,200
        // cycles (what it does between two batches leaves the pipe empty), two warps without turns 3,300
        // (the pipe interleaves them and both softmaxes wait at a time), with turns 2,800.
        constexpr uint32_t NK = C::kK, NV = C::kV;
        const int h = warp == 8 ? 0 : 1;
        uint32_t n_q = 0, n_p = 0, n_turn = 0, n_k = 0, n_v = 0;     // phases; K and V tiles taken
        const uint32_t id_s = idesc_16<T>(kCells, false), id_o = idesc_16<T>((D + 15) & ~15, true);
        const uint32_t tS = tmem + h * 128, tP = tmem + C::col_p(h), tO = tmem + C::col_o(h);
        const int ks_q = (D + 15) / 16;
        const uint64_t qd = sw128_desc(q_smem + h * C::kPanels * kPanel);
        bool ok = true;
        auto scores = [&](uint32_t stage, bool pass) {               // S = Q K^T from a stage; pass: the turn, half-way
            const uint64_t b = sw128_desc(ring + stage * C::kStage);
            if (elect_one()) {
                if (ks_q == DP / 16) {
#pragma unroll
                    for (int ks = 0; ks < DP / 16; ++ks) {
                        const uint64_t o = (uint64_t)((ks >> 2) * (kPanel >> 4) + 2 * (ks & 3));
                        mma_ss(tS, qd + o, b + o, id_s, ks > 0);
                        if (ks == DP / 32 - 1 && pass) mbar_arrive(smem_u32(&bar_turn[1 - h]));
                    }
                } else {
                    for (int ks = 0; ks < ks_q; ++ks) {
                        const uint64_t o = (uint64_t)((ks >> 2) * (kPanel >> 4) + 2 * (ks & 3));
                        mma_ss(tS, qd + o, b + o, id_s, ks > 0);
                        if (ks == (ks_q - 1) / 2 && pass) mbar_arrive(smem_u32(&bar_turn[1 - h]));
                    }
                }
                mma_commit(smem_u32(&bar_s[h]));
                mma_commit(smem_u32(&bar_empty[stage]));
            }
            __syncwarp();
        };
        for (int it = it0; it < it1 && ok; ++it) {
            take(it);
            const int rows = w.rows, t0 = w.t0, t1 = w.t1;
            if (h * 128 >= rows) {
                // no rows here: the stages go by one at a time (a barrier's parity names a phase only to
                // a waiter that is at most one behind)
                for (int t = t0; t < t1 && ok; ++t, ++n_k, ++n_v) {
                    ok = warp_wait(smem_u32(&bar_full[n_k % NK]), (n_k / NK) & 1, ctl);
                    if (ok && lane == 0) mbar_arrive(smem_u32(&bar_empty[n_k % NK]));
                    ok = ok && warp_wait(smem_u32(&bar_full[NK + n_v % NV]), (n_v / NV) & 1, ctl);
                    if (ok && lane == 0) mbar_arrive(smem_u32(&bar_empty[NK + n_v % NV]));
                }
                continue;
            }
            if (t1 <= t0) continue;                                  // (rows without cells: no Q, no products)
            ok = warp_wait(smem_u32(&bar_q[h]), n_q++ & 1, ctl);
            if (!ok) break;
            ok = warp_wait(smem_u32(&bar_full[n_k % NK]), (n_k / NK) & 1, ctl);
            if (!ok) break;
            fence_after();
            scores(n_k % NK, false);
            ++n_k;
            for (int t = t0; t < t1; ++t, ++n_v) {
                const TileCells tc = tile_cells(w, t, p.box);
                const int ks_v = min(kCells, tc.end - tc.start + 15) / 16;   // cells past the end have probability 0
                const uint32_t v_stage = NK + n_v % NV;
                const bool more = t + 1 < t1;
                const uint64_t b = mn_desc(ring + v_stage * C::kStage);
                // (turn n of warp 8 follows turn n - 1 of warp 11, turn n of warp 11 turn n of warp 8)
                ok = warp_wait(smem_u32(&bar_full[v_stage]), (n_v / NV) & 1, ctl) &&
                     warp_wait(smem_u32(&bar_p[h][1]), n_p & 1, ctl) &&
                     (rows <= 128 || (h == 0 && n_turn == 0) || warp_wait(smem_u32(&bar_turn[h]), (n_turn - (h == 0)) & 1, ctl));
                if (!ok) break;
                fence_after();
                auto product = [&](int ks, uint32_t acc) { mma_ts(tO, tP + ks * 8, b + (uint64_t)(ks * (2048 >> 4)), id_o, acc); };
                if (elect_one()) {                                   // cells 64 .. 127 and 0 .. 31
                    if (ks_v == 8) {
                        product(4, t > t0);
#pragma unroll
                        for (int ks = 5; ks < 10; ++ks) product(ks & 7, 1);
                    } else {
                        for (int ks = 4; ks < ks_v; ++ks) product(ks, t > t0 || ks > 4);
                        for (int ks = 0; ks < min(ks_v, 2); ++ks) product(ks, t > t0 || ks > 0 || ks_v > 4);
                    }
                }
                __syncwarp();
                ok = warp_wait(smem_u32(&bar_p[h][0]), n_p & 1, ctl);
                if (!ok) break;
                ++n_p;
                fence_after();
                if (C::kApart && more) {
                    ok = warp_wait(smem_u32(&bar_full[n_k % NK]), (n_k / NK) & 1, ctl);
                    if (!ok) break;
                    fence_after();
                    scores(n_k % NK, false);
                    ++n_k;
                }
                if (elect_one()) {                                   // cells 32 .. 63
                    if (ks_v > 2) product(2, 1);
                    if (C::kApart && rows > 128) mbar_arrive(smem_u32(&bar_turn[1 - h]));
                    if (ks_v > 3) product(3, 1);
                    mma_commit(smem_u32(&bar_empty[v_stage]));
                    if (C::kApart) mma_commit(smem_u32(&bar_pv[h]));
                    if (!more) mma_commit(smem_u32(&bar_o[h]));
                }
                __syncwarp();
                if (C::kApart) {
                } else if (more) {
                    ok = warp_wait(smem_u32(&bar_full[n_k % NK]), (n_k / NK) & 1, ctl);
                    if (!ok) break;
                    fence_after();
                    scores(n_k % NK, rows > 128);
                    ++n_k;
                } else if (rows > 128 && lane == 0) {
                    mbar_arrive(smem_u32(&bar_turn[1 - h]));
                }
                n_turn += rows > 128;
            }
        }
        // products in flight finish before shared and tensor memory are released
        if (elect_one()) mma_commit(smem_u32(&bar_drain[h]));
        __syncwarp();
        wait_phase_drain(smem_u32(&bar_drain[h]), 0);
    } else if (CODES && warp == 9) {
        // ------------------------------------- copies of codes: a tile's K, then its V, into slots in turn --
        const uint32_t codes = ring + C::kStages * C::kStage;
        // the next one: the tile c_t of the piece c_it (c_which: its V)
        const int boxes = kCells / p.box, page_mask = (1 << p.pool.page_log2) - 1;
        uint32_t copied = 0;
        int c_it = it0 - 1, c_t = 0, c_which = 0, page_next = 0;
        auto page_of = [&](int t) {                                  // the page of box `lane` (none: past the last one, zeros)
            if (t >= copy_sh.t1 || lane >= boxes) return 0;
            const TileCells tc = tile_cells(copy_sh, t, p.box);
            const int j = tc.start + lane * p.box;
            return j < tc.end ? __ldg(p.b.table + copy_sh.table0 + (j >> p.pool.page_log2)) : (int)p.n_pages;
        };
        auto copy = [&] {                                            // false: no more, or a wait ran out
            while (c_it < it1 && (c_it < it0 || c_t >= copy_sh.t1)) {
                if (++c_it == it1) break;
                __syncwarp();
                if (lane < (int)sizeof(TokItem) / 4)
                    reinterpret_cast<int32_t *>(&copy_sh)[lane] = __ldg(reinterpret_cast<const int32_t *>(p.w.items + c_it) + lane);
                __syncwarp();
                c_t = copy_sh.t0;
                page_next = page_of(c_t);
            }
            if (c_it >= it1) return false;
            const uint32_t s = copied % C::kSlots, bar = smem_u32(&bar_code[s]);
            if (copied >= C::kSlots && !warp_wait(smem_u32(&bar_read[s]), (copied / C::kSlots - 1) & 1, ctl)) return false;
            int *pages = page_sh[0][c_t & 1];
            if (c_which == 0) {
                if (lane < 16) pages[lane] = page_next;
                page_next = page_of(c_t + 1);
            }
            __syncwarp();
            const int start = tile_cells(copy_sh, c_t, p.box).start;
            if (elect_one()) {
                const CUtensorMap *map = c_which ? &p.map_v : &p.map_k;
                mbar_expect_tx(bar, C::kSlot);
                uint32_t dst = codes + s * C::kSlot;
                for (int bx = 0; bx < boxes; ++bx, dst += p.box * DP)
                    copy_box(dst, map, 0, (start + bx * p.box) & page_mask, copy_sh.h, pages[bx], bar);
            }
            __syncwarp();
            ++copied;
            if (c_which) ++c_t;
            c_which ^= 1;
            return true;
        };
        while (c_it < it1 && copy()) {
        }
        // copies in flight land before shared memory is released
        for (uint32_t i = copied > C::kSlots ? copied - C::kSlots : 0; i < copied; ++i)
            wait_phase_drain(smem_u32(&bar_code[i % C::kSlots]), (i / C::kSlots) & 1);
    } else if (CODES && warp >= 12) {
        // ------------------------------------------------ widening: a thread per cell of a tile --
        // Its row of codes, 16 at a time and each thread of a phase at another sixteen (no bank conflicts), goes into the
        // swizzled tile that the products read, with the row's scale on the way.
        const int r = threadIdx.x - 384;
        const uint32_t codes = ring + C::kStages * C::kStage;
        bool ok = true;
        uint32_t load = 0, tiles = 0;                                // slots, and tiles of K and of V, done
        for (int it = it0; it < it1 && ok; ++it) {
            take(it);
            const int t1 = w.t1, hh = w.h;
            const int32_t *table = p.b.table + w.table0;
            // the scale bytes of the thread's cell, K's and V's (past the end: 256), a tile ahead, and as they are loaded: what
            // would work on them at once would wait for them
            uint32_t next[2];
            auto scales = [&](int t) {
                const TileCells tc = tile_cells(w, t, p.box);
                const int j = tc.start + r;
                next[0] = next[1] = 256u;
                if (t < t1 && j < tc.end) {
                    const int64_t row = cell_row(p.pool, table, hh, j);
                    next[0] = __ldg(p.pool.ks + row);
                    next[1] = __ldg(p.pool.vs + row);
                }
            };
            scales(w.t0);
            for (int t = w.t0; t < t1 && ok; ++t, ++tiles) {
                const uint32_t bytes[2] = {next[0], next[1]};
                scales(t + 1);
#pragma unroll 1
                for (int which = 0; which < 2; ++which, ++load) {
                    const uint32_t slot = load % C::kSlots, of = which ? C::kV : C::kK, stage = which ? C::kK + tiles % C::kV : tiles % C::kK;
                    ok = warp_wait(smem_u32(&bar_code[slot]), (load / C::kSlots) & 1, ctl) &&
                         (tiles < of || warp_wait(smem_u32(&bar_empty[stage]), (tiles / of - 1) & 1, ctl));
                    if (!ok) break;
                    const uint32_t to = ring + stage * C::kStage;
                    const uint32_t byte = which ? bytes[1] : bytes[0];
                    const uint32_t from = codes + slot * C::kSlot + r * DP;
                    const uint32_t unit = Widen<T>::unit(byte);
                    const bool fast = Widen<T>::fast(byte);
                    auto put = [&](int k, uint4 lo, uint4 hi) {
                        const uint32_t panel = to + (k >> 2) * kPanel;
                        st_shared16(panel + sw128_off(r, 2 * k & 7), lo);
                        st_shared16(panel + sw128_off(r, (2 * k & 7) + 1), hi);
                    };
                    if (fast) {
                        // (two at a time: the loop unrolled whole costs more in instruction fetches, 189 -> 209 us)
#pragma unroll 1
                        for (int c0 = 0; c0 < DP / 16; c0 += 2) {
                            uint4 v[2];
                            int k[2];
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                k[c] = DP == 128 ? (c0 + c + r) & 7 : (c0 + c + (r >> 1)) & 3;
                                v[c] = ld_shared16(from + k[c] * 16);
                            }
#pragma unroll
                            for (int c = 0; c < 2; ++c)
                                put(k[c],
                                    make_uint4(Widen<T>::pair(v[c].x, 0, unit), Widen<T>::pair(v[c].x, 1, unit),
                                               Widen<T>::pair(v[c].y, 0, unit), Widen<T>::pair(v[c].y, 1, unit)),
                                    make_uint4(Widen<T>::pair(v[c].z, 0, unit), Widen<T>::pair(v[c].z, 1, unit),
                                               Widen<T>::pair(v[c].w, 0, unit), Widen<T>::pair(v[c].w, 1, unit)));
                        }
                    } else {
                        const float s = scale_of(byte & 255u);
                        auto slow = [&](uint32_t four, int half) {
                            const float2 f = e4m3_values((uint16_t)(half ? four >> 16 : four));
                            return byte == 256u ? 0u : narrow2<T>(widened<T>(f.x * s), widened<T>(f.y * s));
                        };
#pragma unroll 1
                        for (int k = 0; k < DP / 16; ++k) {
                            const uint4 v = ld_shared16(from + k * 16);
                            put(k, make_uint4(slow(v.x, 0), slow(v.x, 1), slow(v.y, 0), slow(v.y, 1)),
                                make_uint4(slow(v.z, 0), slow(v.z, 1), slow(v.w, 0), slow(v.w, 1)));
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(smem_u32(&bar_read[slot]));
                        mbar_arrive(smem_u32(&bar_full[stage]));
                    }
                }
            }
        }
    } else if (!CODES) {
        // -------------------------------------------- copies: warp 9 K tiles, warp 10 V tiles --
        constexpr uint32_t NS = C::kStages / 2;
        const int which = warp - 9, boxes = kCells / p.box, slots = (1 << p.pool.page_log2) - 1;
        const CUtensorMap *map = which ? &p.map_v : &p.map_k;
        uint32_t load = 0;
        bool ok = true;
        for (int it = it0; it < it1 && ok; ++it) {
            take(it);
            const int t1 = w.t1, hh = w.h;
            const int32_t *table = p.b.table + w.table0;
            // the page of box `lane` (a box without cells lies past the last page: zeros), a tile ahead
            auto page_of = [&](int t) {
                if (t >= t1 || lane >= boxes) return 0;
                const TileCells tc = tile_cells(w, t, p.box);
                const int j = tc.start + lane * p.box;
                return j < tc.end ? __ldg(table + (j >> p.pool.page_log2)) : (int)p.n_pages;
            };
            int next = page_of(w.t0);
            for (int t = w.t0; t < t1; ++t) {
                int *pages = page_sh[which][load & 1];
                if (lane < 16) pages[lane] = next;
                next = page_of(t + 1);
                const int start = tile_cells(w, t, p.box).start;
                const uint32_t s = which * NS + load % NS, bar = smem_u32(&bar_full[s]);
                if (load >= NS) {
                    ok = warp_wait(smem_u32(&bar_empty[s]), (load / NS - 1) & 1, ctl);
                    if (!ok) break;
                }
                __syncwarp();
                if (elect_one()) {
                    mbar_expect_tx(bar, C::kStage);
                    uint32_t dst = ring + s * C::kStage;
#pragma unroll 2
                    for (int bx = 0; bx < boxes; ++bx, dst += p.box * 128) {
                        const int page = pages[bx], slot = (start + bx * p.box) & slots;
#pragma unroll
                        for (int x = 0; x < C::kPanels; ++x) copy_box(dst + x * kPanel, map, x * 64, slot, hh, page, bar);
                    }
                }
                __syncwarp();
                ++load;
            }
        }
        // copies in flight land before shared memory is released
        for (uint32_t i = load > NS ? load - NS : 0; i < load; ++i)
            wait_phase_drain(smem_u32(&bar_full[which * NS + i % NS]), (i / NS) & 1);
    }
    fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && ctl_sh.abort) atomicExch(p.err, MURE_ERR_TIMEOUT);
    if (warp == 8) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
    }
    if (!again_sh || ctl_sh.abort) return;

    // Marked rows by the definition, a warp per row, from the cells they may attend to alone: a masked cell's NaN or
    // infinity has met a probability of 0.  Here, where no wait is left that their time could run out on.
    for (int it = it0; it < it1; ++it) {
        take(it);
        for (int r = warp; r < w.rows; r += C::kThreads / 32) {
            if (!(p.w.again[(int64_t)it * (kChunkRows / 32) + r / 32] >> (r & 31) & 1)) continue;
            const int row = w.r0 + r, token = w.row0 + row / p.b.group, head = w.h * p.b.group + row % p.b.group;
            const T *q = reinterpret_cast<const T *>(p.q.p) + token * p.q.ts + head * p.q.hs;
            const TileCells first = tile_cells(w, w.t0, p.box), end = tile_cells(w, w.t1 - 1, p.box);
            float y[8], m, l;
            TreeRow tree{};
            if (TREE) tree = tree_row(p.b, token);
            const int pos = TREE ? tree.pos : w.pos + row / p.b.group, j0 = first.start, j1 = min(end.end, end.start + kCells);
            if (CODES || p.code_table)
                attend_row<T, true, TREE>(p.codes, p.code_table + w.table0, w.h, q, p.q.vec, pos, j0, j1, p.b.window, p.b.sinks,
                                          p.b.scale_log2, y, m, l, tree);
            else
                attend_row<T, false, TREE>(p.pool, p.b.table + w.table0, w.h, q, p.q.vec, pos, j0, j1, p.b.window, p.b.sinks,
                                           p.b.scale_log2, y, m, l, tree);
            if (w.parts > 1) {
                const int64_t pr = (int64_t)w.part * kChunkRows + r;
                if (lane * 8 < D) store8(p.w.part + pr * DP + lane * 8, 1, y);
                if (lane == 0) { p.ml[pr * 2] = m; p.ml[pr * 2 + 1] = l; }
            } else {
                const float f = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] *= f;
                if (lane * 8 < D)
                    store8(reinterpret_cast<T *>(p.out.p) + token * p.out.ts + head * p.out.hs + lane * 8, p.out.vec, y);
                if (p.lse && lane == 0) p.lse[(int64_t)token * p.b.n_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945f;
            }
        }
    }
}

// Joins the parts of rows that were cut: a warp per row, the parts in their order.  of: rows of a part.
template <class T>
__global__ void __launch_bounds__(256) k_tokens_join(const TokItem *cut, int of, int DP, TokBatch b, int D, TokRows out, float *lse,
                                                     const float *part, const float *ml)
{
    // (launched while the parts are still made, see launch_tokens_join, or after them: then this waits for nothing)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const TokItem &w = cut[blockIdx.x];
    const int r = blockIdx.y * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (r >= w.rows) return;
    const int64_t first = (int64_t)w.part0 * of + r;
    float m = -INFINITY;
    for (int i = 0; i < w.parts; ++i) {
        const float v = ml[(first + (int64_t)i * of) * 2];
        m = isnan(v) || isnan(m) ? NAN : fmaxf(m, v);
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < w.parts; ++i) {
        const int64_t at = first + (int64_t)i * of;
        const float f = ex2(ml[at * 2] - ref);
        l = fmaf(f, ml[at * 2 + 1], l);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k * 32 + lane < D) x[k] = fmaf(f, part[at * DP + k * 32 + lane], x[k]);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int row = w.r0 + r, token = w.row0 + row / b.group, head = w.h * b.group + row % b.group;
    T *o = reinterpret_cast<T *>(out.p) + token * out.ts + head * out.hs;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k * 32 + lane < D) o[k * 32 + lane] = TokType<T>::down(x[k] * inv);
    if (lse && lane == 0) lse[(int64_t)token * b.n_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945f;
}

template <class T, int DP, bool TREE, bool CODES>
void pieces(const ChunkParams &p, cudaStream_t s)
{
    using C = Chunk<DP, CODES>;
    allow_dynamic_smem_once<k_tokens_chunk<T, DP, TREE, CODES>>(C::kSmem);
    k_tokens_chunk<T, DP, TREE, CODES><<<p.w.blocks, C::kThreads, C::kSmem, s>>>(p);
}

template <class T, int DP>
int go(const ChunkParams &p, const TokChunk &c, bool fused, cudaStream_t s)
{
    if (p.b.node && fused) pieces<T, DP, true, true>(p, s);
    else if (p.b.node) pieces<T, DP, true, false>(p, s);
    else pieces<T, DP, false, false>(p, s);
    return 1 + launch_tokens_join(c, kChunkRows, p.b, std::is_same<T, __half>::value ? MURE_F16 : MURE_BF16, p.pool.d, p.out, p.lse, false, s);
}

}  // namespace

int launch_tokens_join(const TokChunk &c, int of, const TokBatch &b, int dtype, int d, TokRows out, float *lse, bool early, cudaStream_t s)
{
    if (c.n_cut == 0) return 0;
    const int dp = d <= 64 ? 64 : 128;
    // early: the parts' kernel lets this launch begin at once, and its blocks wait for it (one tree's two launches 20 -> 19 us;
    // behind the two-tile kernel's long runs 189 -> 194).
    cudaLaunchAttribute attribute{};
    attribute.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attribute.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3(c.n_cut, of / 8);
    config.blockDim = 256;
    config.stream = s;
    config.attrs = &attribute;
    config.numAttrs = early ? 1 : 0;
    const float *part = c.w.part, *ml = c.ml;
    if (dtype == MURE_F16) cudaLaunchKernelEx(&config, k_tokens_join<__half>, c.cut, of, dp, b, d, out, lse, part, ml);
    else cudaLaunchKernelEx(&config, k_tokens_join<__nv_bfloat16>, c.cut, of, dp, b, d, out, lse, part, ml);
    return 1;
}

int chunk_blocks() { return sm_count(); }

int chunk_box(int page_size) { return page_size < kChunkTile ? page_size : kChunkTile; }

int64_t chunk_part_floats(int d) { return (int64_t)256 * ((d <= 64 ? 64 : 128) + 2); }

bool chunk_map(CUtensorMap &map, void *pool, int dtype, int hk, int d, int page_size, int64_t n_pages)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = tensor_map_encoder();
    if (!enc) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)page_size, (cuuint64_t)hk, (cuuint64_t)n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)d * 2, (cuuint64_t)d * 2 * page_size, (cuuint64_t)d * 2 * page_size * hk};
    const cuuint32_t box[4] = {64, (cuuint32_t)chunk_box(page_size), 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return enc(&map, dtype == MURE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, pool, dims, strides, box,
               estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool chunk_code_map(CUtensorMap &map, void *pool, int hk, int d, int page_size, int64_t n_pages)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = tensor_map_encoder();
    if (!enc) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)page_size, (cuuint64_t)hk, (cuuint64_t)n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)d, (cuuint64_t)d * page_size, (cuuint64_t)d * page_size * hk};
    const cuuint32_t box[4] = {d <= 64 ? 64u : 128u, (cuuint32_t)chunk_box(page_size), 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return enc(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, pool, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int launch_tokens_chunk(const TokPool &pool, const TokBatch &b, const TokChunk &c, int dtype, TokRows q, TokRows out, float *lse,
                        int64_t n_pages, const CUtensorMap &map_k, const CUtensorMap &map_v, const TokPool *codes,
                        const int32_t *code_table, bool fused, int *err, int64_t spin, cudaStream_t s)
{
    if (c.w.blocks == 0) return 0;
    ChunkParams p{};
    p.pool = pool; p.b = b; p.w = c.w; p.q = q; p.out = out; p.lse = lse;
    p.ml = c.ml;
    p.n_pages = n_pages;
    if (codes) {
        p.codes = *codes;
        p.code_table = code_table;
    }
    p.box = chunk_box(1 << pool.page_log2);
    p.err = err;
    p.spin = spin;
    p.map_k = map_k;
    p.map_v = map_v;
    if (dtype == MURE_F16) return pool.d <= 64 ? go<__half, 64>(p, c, fused, s) : go<__half, 128>(p, c, fused, s);
    return pool.d <= 64 ? go<__nv_bfloat16, 64>(p, c, fused, s) : go<__nv_bfloat16, 128>(p, c, fused, s);
}

}  // namespace mure
