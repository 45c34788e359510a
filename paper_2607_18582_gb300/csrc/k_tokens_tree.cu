// Token caches: attention of trees of new tokens over 16-bit cells, in pieces of up to 128 rows (new token, query head) of one
// sequence and cached head, on the 5th-generation tensor cores.
//
// The products and the softmax are those of the kernel for chunks (S = Q K^T and O += P V in tensor memory, a thread per
// row, scores relative to a value near their running maximum).  What differs is the shape of the work: a tree has few rows
// and its cells are many, or neither, so that a piece is a few tiles of cells, and what takes the time is the chain from a
// tile's scores to its product, and a piece's beginning and end.  So a CTA takes one tile of 128 rows
// alone, in half of an SM's registers, shared and tensor memory, and two CTAs share an SM: while one waits the other works.
// Warps:
//   0-3  softmax, a thread per row; they also fetch Q and write the rows out;
//   4    issues the MMAs;
//   5    copies K and V tiles by tensor maps.
// A cell before the tree's is seen by its position, as anywhere; of the tree's own a row sees those whose bits are set
// (its token and its ancestors), 32 at a time.
//
// Measured (GB300): 64 trees of 3 to 40 tokens within a window of 1,024, 15 heads of 64 f16 values on 5: 37 us and 4 for the
// join (the kernel for chunks: 55 and 3; with the few rows' kernel before this one for the smaller trees, 27 and 18).  One
// tree of 24 tokens over 700 cells: 15 us, of which a piece's beginning and end are some 9 (sequence, piece, page and cells in a
// chain of loads, then scores, softmax and product) and a tile 2.1.  Trees of more than 128 rows are slower here than where two row
// tiles share each K and V tile: 200 to 256 rows over 100,000 cells 215 us against 192, 120 to 256 over 700 to 3,000 71
// against 66.
#include "simt_tile.cuh"
#include "tokens_tc.cuh"

namespace mure {

namespace {

constexpr int kThreads = 192;

template <int DP>
struct TreeShape {
    static constexpr int kPanels = DP / 64;
    static constexpr uint32_t kQ = kPanels * kPanel;
    static constexpr uint32_t kStage = kPanels * kPanel;            // a K or V tile
    static constexpr uint32_t kStages = DP == 64 ? 2 : 1;           // of K, and of V
    // Tensor memory, 256 columns: S in 0 .. 127, O from 128; P over half of S, or for up to 64 values, where O leaves room,
    // beside O: the next scores then need not wait for P V.
    static constexpr bool kApart = DP == 64;
    static constexpr uint32_t kColP = kApart ? 192 : 64, kColO = 128;
    static constexpr uint32_t kSmem = kQ + 2 * kStages * kStage + 1024;     // (+ room to align to 1024)
    static_assert(2 * (kSmem + 1024 + 1024) <= 228 * 1024, "two CTAs do not fit an SM");
};

struct TreeParams {
    TokPool pool;
    TokBatch b;
    TokWork w;
    TokRows q, out;
    float *lse;
    float *ml;               // partial results' maxima and sums, [parts][kTreeRows][2]
    int64_t n_pages;
    int box;                 // cells of a copied box
    int *err;
    long long spin;
    CUtensorMap map_k, map_v;
};

template <class T, int DP>
__global__ void __launch_bounds__(kThreads, 2) k_tokens_tree(const __grid_constant__ TreeParams p)
{
    using C = TreeShape<DP>;
    constexpr uint32_t NS = C::kStages;
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) uint64_t bar_full[2 * NS], bar_empty[2 * NS], bar_q, bar_s, bar_p[2], bar_o, bar_pv, bar_drain;
    __shared__ uint32_t tmem_sh;
    __shared__ int again_sh;                  // rows are marked
    __shared__ WaitCtl ctl_sh;
    __shared__ TokItem item_sh[6];            // each warp's piece of work
    __shared__ int page_sh[2][16];            // the copying warp: the pages of a tile's boxes
    volatile WaitCtl *ctl = &ctl_sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_smem = base, ring = base + C::kQ;
    const int D = p.pool.d;

    if (warp == 4) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_sh)), "r"(256));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (threadIdx.x == 0) {
        again_sh = 0;
        ctl_sh.abort = 0;
        ctl_sh.limit = p.spin > 0 ? p.spin : kSpin;
        for (uint32_t i = 0; i < 2 * NS; ++i) {
            mbar_init(smem_u32(&bar_full[i]), 1);
            mbar_init(smem_u32(&bar_empty[i]), 1);
        }
        mbar_init(smem_u32(&bar_q), 4);
        mbar_init(smem_u32(&bar_s), 1);
        mbar_init(smem_u32(&bar_p[0]), 4);
        mbar_init(smem_u32(&bar_p[1]), 4);
        mbar_init(smem_u32(&bar_o), 1);
        mbar_init(smem_u32(&bar_pv), 1);
        mbar_init(smem_u32(&bar_drain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_sh;
    asm volatile("griddepcontrol.launch_dependents;");               // (the join may begin; it waits for this grid's end)
    const int it0 = p.w.first[blockIdx.x], it1 = p.w.first[blockIdx.x + 1];
    const TokItem &w = item_sh[warp];
    auto take = [&](int it) {
        __syncwarp();
        if (lane < (int)sizeof(TokItem) / 4)
            reinterpret_cast<int32_t *>(&item_sh[warp])[lane] = __ldg(reinterpret_cast<const int32_t *>(p.w.items + it) + lane);
        __syncwarp();
    };

    if (warp < 4) {
        // ------------------------------------------------------------------ softmax --
        const int r = threadIdx.x;                                   // row of the tile
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        const uint32_t tS = tmem + lanes, tP = tmem + lanes + C::kColP, tO = tmem + lanes + C::kColO;
        uint32_t n_s = 0, n_o = 0;                                   // phases waited for
        bool ok = true;
        for (int it = it0; it < it1 && ok; ++it) {
            take(it);
            const int rows = w.rows, t0 = w.t0, t1 = w.t1, pos = w.pos;
            const int row = w.r0 + r;
            const bool real = r < rows;
            const bool have = t1 > t0;                               // (no cells: zeros, no products)
            // Q into the K-major swizzled tile, the lanes of a warp along the rows: kLanes 16-byte chunks of one row, the next
            // rows beside it.  Rows without cells leave Q and its barrier alone.
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
                    st_shared16(q_smem + (chunk >> 3) * kPanel + sw128_off((r & ~31) + i * kPer + lane / kLanes, chunk & 7), v[i]);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_q));
            }

            // (all rows see all cells before the tree's, and lie no further than a chain's)
            const int hi = pos + (w.r0 + 127) / p.b.group;
            const TreeRow tree = tree_row(p.b, w.row0 + min(row, w.r0 + rows - 1) / p.b.group);
            float m = -INFINITY, l = 0.f;
            for (int t = t0; t < t1; ++t) {
                const TileCells tc = tile_cells(w, t, p.box);
                const bool open = tc.start + kCells <= min(tc.end, pos) && (p.b.window == 0 || tc.start > hi - p.b.window);
                // the cells that the row may attend to, a bit each (before the wait: they come from memory)
                uint32_t bits[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    bits[i] = open ? ~0u : bits_below(tc.end - tc.start - 32 * i) & tree_seen(tree, tc.start + 32 * i, p.b.window, p.b.sinks);
                ok = warp_wait(smem_u32(&bar_s), n_s & 1, ctl);
                if (!ok) break;
                ++n_s;
                fence_after();
                auto mask = [&](uint32_t *x, uint32_t of) {
                    if (open) return;
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = of & (1u << i) ? x[i] : 0xFF800000u;
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
                    mask(s, bits[2 * c]);
                    mask(s + 32, bits[2 * c + 1]);
#pragma unroll
                    for (int i = 0; i < 64; ++i) top[i & 3] = fmaxf(top[i & 3], __uint_as_float(s[i]));
                }
                const float mt = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * p.b.scale_log2;
                // the product before (the last piece's at first, whose arrival no other wait stands for) has read P and
                // added to O
                if (C::kApart && n_s > 1) {
                    ok = warp_wait(smem_u32(&bar_pv), (n_s - 2) & 1, ctl);
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
                mask(x, bits[0]);
                powers(x, tP);
                tmem_ld32(tS + 32, x);
                tmem_wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_p[1]));
                tmem_wait_ld();
                mask(x, bits[1]);
                powers(x, tP + 16);
                l += unpack2(sum).x + unpack2(sum).y;
                tmem_wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_p[0]));
                };
                if (DP == 64 && tc.end - tc.start <= 64) softmax(std::integral_constant<bool, DP == 64>{});
                else softmax(std::false_type{});
                if (!ok) break;
            }
            if (!ok) break;
            // the next piece's row of Q, to be at hand when this one's rows are out
            const TokItem *after = p.w.items + min(it + 1, it1 - 1);
            const int next_r0 = __ldg(&after->r0) + r, next_rows = __ldg(&after->rows);
            const int next_row0 = __ldg(&after->row0), next_h = __ldg(&after->h);
            if (have) {
                ok = warp_wait(smem_u32(&bar_o), n_o & 1, ctl);
                if (!ok) break;
                ++n_o;
                fence_after();
            }
            if (it + 1 < it1 && r < next_rows) {
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
            const int64_t out_at = !real ? -1 : parts > 1 ? ((int64_t)part * kTreeRows + r) * DP : token * p.out.ts + head * p.out.hs;
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
                                st_shared16(q_smem + (at >> 3) * kPanel + sw128_off(r, at & 7),
                                            make_uint4(x[k + i], x[k + i + 1], x[k + i + 2], x[k + i + 3]));
                            }
                        } else {
                            uint32_t y[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                y[i] = narrow2<T>(__uint_as_float(x[k + 2 * i]) * inv, __uint_as_float(x[k + 2 * i + 1]) * inv);
                            const int at = (c + k) / 8;
                            st_shared16(q_smem + (at >> 3) * kPanel + sw128_off(r, at & 7), make_uint4(y[0], y[1], y[2], y[3]));
                        }
                    }
                }
                __syncwarp();
#pragma unroll 8
                for (int i = 0; i < 32; i += kPer) {
                    const int64_t off = __shfl_sync(0xffffffffu, out_at, i + lane / kLanes);
                    const uint4 v = ld_shared16(q_smem + (chunk >> 3) * kPanel + sw128_off((r & ~31) + i + lane / kLanes, chunk & 7));
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
                    float *ml = p.ml + ((int64_t)part * kTreeRows + r) * 2;
                    ml[0] = m;
                    ml[1] = l;
                } else if (p.lse) {
                    p.lse[(int64_t)token * p.b.n_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945f;
                }
            }
            // rows whose sums are not numbers are marked, to be done again once every role is through
            const uint32_t again = __ballot_sync(0xffffffffu, bad && real);
            if (lane == 0) {
                p.w.again[(int64_t)it * (kTreeRows / 32) + warp] = again;
                if (again) again_sh = 1;
            }
        }
    } else if (warp == 4) {
        // -------------------------------------------------------------- MMA issue --
        uint32_t n_q = 0, n_p = 0, n_k = 0, n_v = 0;                 // phases; K and V tiles taken
        const uint32_t id_s = idesc_16<T>(kCells, false), id_o = idesc_16<T>((D + 15) & ~15, true);
        const uint32_t tS = tmem, tP = tmem + C::kColP, tO = tmem + C::kColO;
        const int ks_q = (D + 15) / 16;
        const uint64_t qd = sw128_desc(q_smem);
        bool ok = true;
        auto scores = [&](uint32_t stage) {                          // S = Q K^T from a stage
            const uint64_t b = sw128_desc(ring + stage * C::kStage);
            if (elect_one()) {
                for (int ks = 0; ks < ks_q; ++ks) {
                    const uint64_t o = (uint64_t)((ks >> 2) * (kPanel >> 4) + 2 * (ks & 3));
                    mma_ss(tS, qd + o, b + o, id_s, ks > 0);
                }
                mma_commit(smem_u32(&bar_s));
                mma_commit(smem_u32(&bar_empty[stage]));
            }
            __syncwarp();
        };
        for (int it = it0; it < it1 && ok; ++it) {
            take(it);
            const int t0 = w.t0, t1 = w.t1;
            if (t1 <= t0) continue;                                  // (rows without cells: no Q, no products)
            ok = warp_wait(smem_u32(&bar_q), n_q++ & 1, ctl);
            if (!ok) break;
            ok = warp_wait(smem_u32(&bar_full[n_k % NS]), (n_k / NS) & 1, ctl);
            if (!ok) break;
            fence_after();
            scores(n_k % NS);
            ++n_k;
            for (int t = t0; t < t1; ++t, ++n_v) {
                const TileCells tc = tile_cells(w, t, p.box);
                const int ks_v = min(kCells, tc.end - tc.start + 15) / 16;   // cells past the end have probability 0
                const uint32_t v_stage = NS + n_v % NS;
                const bool more = t + 1 < t1;
                const uint64_t b = mn_desc(ring + v_stage * C::kStage);
                ok = warp_wait(smem_u32(&bar_full[v_stage]), (n_v / NS) & 1, ctl) && warp_wait(smem_u32(&bar_p[1]), n_p & 1, ctl);
                if (!ok) break;
                fence_after();
                auto product = [&](int ks, uint32_t acc) { mma_ts(tO, tP + ks * 8, b + (uint64_t)(ks * (2048 >> 4)), id_o, acc); };
                if (elect_one()) {                                   // cells 64 .. 127 and 0 .. 31
                    for (int ks = 4; ks < ks_v; ++ks) product(ks, t > t0 || ks > 4);
                    for (int ks = 0; ks < min(ks_v, 2); ++ks) product(ks, t > t0 || ks > 0 || ks_v > 4);
                }
                __syncwarp();
                ok = warp_wait(smem_u32(&bar_p[0]), n_p & 1, ctl);
                if (!ok) break;
                ++n_p;
                fence_after();
                if (C::kApart && more) {
                    ok = warp_wait(smem_u32(&bar_full[n_k % NS]), (n_k / NS) & 1, ctl);
                    if (!ok) break;
                    fence_after();
                    scores(n_k % NS);
                    ++n_k;
                }
                if (elect_one()) {                                   // cells 32 .. 63
                    if (ks_v > 2) product(2, 1);
                    if (ks_v > 3) product(3, 1);
                    mma_commit(smem_u32(&bar_empty[v_stage]));
                    if (C::kApart) mma_commit(smem_u32(&bar_pv));
                    if (!more) mma_commit(smem_u32(&bar_o));
                }
                __syncwarp();
                if (!C::kApart && more) {
                    ok = warp_wait(smem_u32(&bar_full[n_k % NS]), (n_k / NS) & 1, ctl);
                    if (!ok) break;
                    fence_after();
                    scores(n_k % NS);
                    ++n_k;
                }
            }
        }
        // products in flight finish before shared and tensor memory are released
        if (elect_one()) mma_commit(smem_u32(&bar_drain));
        __syncwarp();
        wait_phase_drain(smem_u32(&bar_drain), 0);
    } else {
        // ---------------------------------------------- copies: a tile's K, then its V --
        const int boxes = kCells / p.box, slots = (1 << p.pool.page_log2) - 1;
        uint32_t load = 0, begun[2] = {0, 0};
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
            for (int t = w.t0; t < t1 && ok; ++t, ++load) {
                int *pages = page_sh[load & 1];
                if (lane < 16) pages[lane] = next;
                next = page_of(t + 1);
                const int start = tile_cells(w, t, p.box).start;
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    const uint32_t s = which * NS + load % NS, bar = smem_u32(&bar_full[s]);
                    if (load >= NS) {
                        ok = warp_wait(smem_u32(&bar_empty[s]), (load / NS - 1) & 1, ctl);
                        if (!ok) break;
                    }
                    __syncwarp();
                    if (elect_one()) {
                        const CUtensorMap *map = which ? &p.map_v : &p.map_k;
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
                    ++begun[which];
                }
                if (!ok) break;
            }
        }
        // copies in flight land before shared memory is released
#pragma unroll
        for (int which = 0; which < 2; ++which)
            for (uint32_t i = begun[which] > NS ? begun[which] - NS : 0; i < begun[which]; ++i)
                wait_phase_drain(smem_u32(&bar_full[which * NS + i % NS]), (i / NS) & 1);
    }
    fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && ctl_sh.abort) atomicExch(p.err, MURE_ERR_TIMEOUT);
    if (warp == 4) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(256));
    }
    if (!again_sh || ctl_sh.abort) return;

    // Marked rows by the definition, a warp per row, from the cells they may attend to alone: a masked cell's NaN or
    // infinity has met a probability of 0.  Here, where no wait is left that their time could run out on.
    for (int it = it0; it < it1; ++it) {
        take(it);
        for (int r = warp; r < w.rows; r += kThreads / 32) {
            if (!(p.w.again[(int64_t)it * (kTreeRows / 32) + r / 32] >> (r & 31) & 1)) continue;
            const int row = w.r0 + r, token = w.row0 + row / p.b.group, head = w.h * p.b.group + row % p.b.group;
            const T *q = reinterpret_cast<const T *>(p.q.p) + token * p.q.ts + head * p.q.hs;
            const TileCells first = tile_cells(w, w.t0, p.box), end = tile_cells(w, w.t1 - 1, p.box);
            float y[8], m, l;
            const TreeRow tree = tree_row(p.b, token);
            attend_row<T, false, true>(p.pool, p.b.table + w.table0, w.h, q, p.q.vec, tree.pos, first.start,
                                       min(end.end, end.start + kCells), p.b.window, p.b.sinks, p.b.scale_log2, y, m, l, tree);
            if (w.parts > 1) {
                const int64_t pr = (int64_t)w.part * kTreeRows + r;
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

template <class T, int DP>
int go(const TreeParams &p, cudaStream_t s)
{
    allow_dynamic_smem_once<k_tokens_tree<T, DP>>(TreeShape<DP>::kSmem);
    k_tokens_tree<T, DP><<<p.w.blocks, kThreads, TreeShape<DP>::kSmem, s>>>(p);
    return 1;
}

}  // namespace

int tree_blocks() { return 2 * sm_count(); }

int64_t tree_part_floats(int d) { return (int64_t)kTreeRows * ((d <= 64 ? 64 : 128) + 2); }

int launch_tokens_tree(const TokPool &pool, const TokBatch &b, const TokChunk &c, int dtype, TokRows q, TokRows out, float *lse,
                       int64_t n_pages, const CUtensorMap &map_k, const CUtensorMap &map_v, int *err, int64_t spin, cudaStream_t s)
{
    if (c.w.blocks == 0) return 0;
    TreeParams p{};
    p.pool = pool; p.b = b; p.w = c.w; p.q = q; p.out = out; p.lse = lse;
    p.ml = c.ml;
    p.n_pages = n_pages;
    p.box = chunk_box(1 << pool.page_log2);
    p.err = err;
    p.spin = spin;
    p.map_k = map_k;
    p.map_v = map_v;
    const int launches = dtype == MURE_F16 ? (pool.d <= 64 ? go<__half, 64>(p, s) : go<__half, 128>(p, s))
                                           : (pool.d <= 64 ? go<__nv_bfloat16, 64>(p, s) : go<__nv_bfloat16, 128>(p, s));
    return launches + launch_tokens_join(c, kTreeRows, b, dtype, pool.d, out, lse, true, s);
}

}  // namespace mure
