// Token caches: writing new tokens' keys and values into their cells and gathering cells into
// dense rows.
//
// Both are copies that touch each byte once and are bound by device memory.  A thread takes eight
// values of a row (16 bytes of a 16-bit type, 8 bytes of codes), the threads of a row are a
// power-of-two group of a warp, so the row's largest magnitude is a few shuffles away and an e4m3
// row is quantised in the pass that copies it.  A block takes a tile of tokens of one sequence.
#include "tokens_util.cuh"

namespace mure {

namespace {

constexpr int kThreads = 256;

struct CellParams {
    TokPool pool;
    TokBatch b;
    TokRows k, v;
    int lanes;       // threads per row: a power of two, at least d / 8
    int part;        // read: 0 all cells, 1 the new tokens'
};

// A block's tile: sequence, first token of the tile, tokens.
struct Tile {
    int seq, i0, n;
};

__device__ __forceinline__ Tile tile_of(const TokBatch &b, bool all, TokSeq &sq)
{
    const int32_t *prefix = all ? b.tile_all : b.tile_new;
    const int per = all ? kTokTileAll : kTokTileNew;
    Tile t;
    t.seq = find_prefix(prefix, b.n_seqs, (int)blockIdx.x);
    sq = b.seq[t.seq];
    t.i0 = ((int)blockIdx.x - prefix[t.seq]) * per;
    t.n = min(per, (all ? sq.kv : sq.n_new) - t.i0);
    return t;
}

template <class T, bool E4M3>
__global__ void __launch_bounds__(kThreads) k_tokens_append(CellParams p)
{
    TokSeq sq;
    const Tile t = tile_of(p.b, false, sq);
    const int lane = threadIdx.x & (p.lanes - 1), D = p.pool.d, c = lane * 8;
    const int32_t *table = p.b.table + sq.table0;
    const int rows = t.n * p.pool.hk * 2;
    // (all lanes of a warp take part in the shuffles: rows are handed out to whole warps)
    const int per = kThreads / p.lanes, first = threadIdx.x / p.lanes;
    for (int r0 = 0; r0 < rows; r0 += per) {
        const int r = r0 + first;
        const bool on = r < rows && c < D;
        const int which = r & 1, h = (r >> 1) % p.pool.hk, i = (r >> 1) / p.pool.hk;
        float x[8];
        int64_t row = 0;
        if (on) {
            const TokRows &in = which ? p.v : p.k;
            row = cell_row(p.pool, table, h, sq.pos + t.i0 + i);
            load8(reinterpret_cast<const T *>(in.p) + (int64_t)(sq.row0 + t.i0 + i) * in.ts + h * in.hs + c, in.vec, x);
        }
        void *pool = which ? p.pool.v : p.pool.k;
        if (!E4M3) {
            if (on) store8(static_cast<T *>(pool) + row * D + c, 1, x);
        } else {
            uint32_t a = 0;
            if (on) {
#pragma unroll
                for (int q = 0; q < 8; ++q) a = max(a, __float_as_uint(x[q]) & 0x7FFFFFFFu);
            }
            for (int s = p.lanes >> 1; s; s >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, s));
            const uint32_t byte = scale_byte(a);
            if (on) {
                uint32_t w[2];
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    w[q] = byte == 255u ? 0u : e4m3_pair(unscale(x[4 * q], byte), unscale(x[4 * q + 1], byte)) |
                                                   e4m3_pair(unscale(x[4 * q + 2], byte), unscale(x[4 * q + 3], byte)) << 16;
                *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(pool) + row * D + c) = make_uint2(w[0], w[1]);
                if (lane == 0) (which ? p.pool.vs : p.pool.ks)[row] = (uint8_t)byte;
            }
        }
    }
}

template <class T, bool E4M3>
__global__ void __launch_bounds__(kThreads) k_tokens_read(CellParams p)
{
    TokSeq sq;
    const Tile t = tile_of(p.b, p.part == 0, sq);
    const int lane = threadIdx.x & (p.lanes - 1), D = p.pool.d, c = lane * 8;
    if (c >= D) return;
    const int32_t *table = p.b.table + sq.table0;
    const int rows = t.n * p.pool.hk;
    const int64_t out0 = (p.part == 0 ? sq.cell0 : (int64_t)sq.row0) + t.i0;
    const int cell0 = (p.part == 0 ? 0 : sq.pos) + t.i0;
    for (int r = threadIdx.x / p.lanes; r < rows; r += kThreads / p.lanes) {
        const int h = r % p.pool.hk, i = r / p.pool.hk;
        const int64_t row = cell_row(p.pool, table, h, cell0 + i);
        float k[8], v[8];
        cell8<T, E4M3>(p.pool.k, p.pool.ks, row, D, c, k);
        cell8<T, E4M3>(p.pool.v, p.pool.vs, row, D, c, v);
        store8(reinterpret_cast<T *>(p.k.p) + (out0 + i) * p.k.ts + h * p.k.hs + c, p.k.vec, k);
        store8(reinterpret_cast<T *>(p.v.p) + (out0 + i) * p.v.ts + h * p.v.hs + c, p.v.vec, v);
    }
}

// Whole pages of codes as 16-bit pages, in the order of the list.
template <class T>
__global__ void __launch_bounds__(kThreads) k_tokens_widen(TokPool p, const int32_t *pages, int64_t rows, int lanes, T *k, T *v)
{
    const int c = (threadIdx.x & (lanes - 1)) * 8;
    if (c >= p.d) return;
    const int64_t per_page = (int64_t)p.hk << p.page_log2;
    for (int64_t r = (int64_t)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes; r < rows; r += (int64_t)gridDim.x * (kThreads / lanes)) {
        const int64_t i = r / per_page, row = __ldg(pages + i) * per_page + (r - i * per_page);
        float x[8], y[8];
        cell8<T, true>(p.k, p.ks, row, p.d, c, x);
        cell8<T, true>(p.v, p.vs, row, p.d, c, y);
        store8(k + r * p.d + c, 1, x);
        store8(v + r * p.d + c, 1, y);
    }
}

template <class T, bool E4M3>
int go(const CellParams &p, bool read, int64_t tiles, cudaStream_t s)
{
    if (read) k_tokens_read<T, E4M3><<<(unsigned)tiles, kThreads, 0, s>>>(p);
    else k_tokens_append<T, E4M3><<<(unsigned)tiles, kThreads, 0, s>>>(p);
    return 1;
}

int dispatch(const CellParams &p, bool read, int dtype, int form, int64_t tiles, cudaStream_t s)
{
    if (tiles == 0) return 0;
    const bool e = form == MURE_FORM_E4M3;
    if (dtype == MURE_F32) return e ? go<float, true>(p, read, tiles, s) : go<float, false>(p, read, tiles, s);
    if (dtype == MURE_F16) return e ? go<__half, true>(p, read, tiles, s) : go<__half, false>(p, read, tiles, s);
    return e ? go<__nv_bfloat16, true>(p, read, tiles, s) : go<__nv_bfloat16, false>(p, read, tiles, s);
}

int row_lanes(int d)
{
    int n = 1;
    while (n * 8 < d) n *= 2;
    return n;
}

}  // namespace

int launch_tokens_widen(const TokPool &pool, int dtype, const int32_t *pages, int64_t n_list, void *k, void *v, cudaStream_t s)
{
    const int lanes = row_lanes(pool.d);
    const int64_t rows = n_list * pool.hk << pool.page_log2;
    const int64_t blocks = (rows + kThreads / lanes - 1) / (kThreads / lanes);
    if (blocks == 0) return 0;
    const unsigned grid = (unsigned)(blocks < (1 << 20) ? blocks : (1 << 20));
    if (dtype == MURE_F16)
        k_tokens_widen<__half><<<grid, kThreads, 0, s>>>(pool, pages, rows, lanes, static_cast<__half *>(k), static_cast<__half *>(v));
    else
        k_tokens_widen<__nv_bfloat16><<<grid, kThreads, 0, s>>>(pool, pages, rows, lanes, static_cast<__nv_bfloat16 *>(k),
                                                                static_cast<__nv_bfloat16 *>(v));
    return 1;
}

int launch_tokens_append(const TokPool &pool, const TokBatch &b, int dtype, int form, TokRows k, TokRows v, int64_t tiles,
                         cudaStream_t s)
{
    return dispatch({pool, b, k, v, row_lanes(pool.d), 1}, false, dtype, form, tiles, s);
}

int launch_tokens_read(const TokPool &pool, const TokBatch &b, int dtype, int form, int part, TokRows k, TokRows v,
                       int64_t tiles, cudaStream_t s)
{
    return dispatch({pool, b, k, v, row_lanes(pool.d), part}, true, dtype, form, tiles, s);
}

}  // namespace mure
