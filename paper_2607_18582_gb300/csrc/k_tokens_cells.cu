// Token caches: writing new tokens' keys and values into their cells and gathering cells into
// dense rows.
//
// Both are copies that touch each byte once and are bound by device memory.  A thread takes eight
// values of a row of K and the same of V (16 bytes each of a 16-bit type, 8 bytes of codes), kRows
// rows at a time: all its loads are on their way before the first is used.  The threads of a row are a
// power-of-two group of a warp, so the row's largest magnitude is a few shuffles away and an e4m3 row is
// quantised in the pass that copies it.  A block takes a tile of 16 tokens of one sequence.
// Measured (GB300, 8 heads of 128 bf16 values): 163,000 e4m3 cells gathered in 184 us, 6.5 TB/s; 57,000
// tokens written as e4m3 and read back in 141 us, 82 of them the writing: 4.3 TB/s, its issue slots 77 %
// busy (74 million warp instructions, the integer pipe 58 %): bound by instructions more than by memory.
#include <type_traits>

#include "tokens_util.cuh"

namespace mure {

namespace {

constexpr int kThreads = 128;    // (with 4 rows a thread: 256 threads 3 %, 2 rows 8-11 %, 8 rows 22-48 % slower)
constexpr int kRows = 4;         // rows of K and of V that a thread has on their way

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
    Tile t;
    // (one tile for each sequence, as in a decoding step: no search)
    t.seq = !all && b.one_new ? (int)blockIdx.x : find_prefix(prefix, b.n_seqs, (int)blockIdx.x);
    sq = b.seq[t.seq];
    t.i0 = !all && b.one_new ? 0 : ((int)blockIdx.x - __ldg(prefix + t.seq)) * kTokTile;
    t.n = min(kTokTile, (all ? sq.kv : sq.n_new) - t.i0);
    return t;
}

// Eight values as they lie in memory.
template <class T, bool E4M3>
struct Raw {
    uint4 w[E4M3 ? 1 : sizeof(T) / 2];
    uint32_t scale;
};

template <class T>
__device__ __forceinline__ void raw_row(Raw<T, false> &r, const T *p, int vec)
{
    if (vec) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = reinterpret_cast<const uint4 *>(p)[i];
    } else {
        T *t = reinterpret_cast<T *>(r.w);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = p[i];
    }
}

template <class T, bool E4M3>
__device__ __forceinline__ void raw_cell(Raw<T, E4M3> &r, const void *pool, const uint8_t *scales, int64_t row, int D, int c)
{
    if constexpr (E4M3) {
        const uint2 u = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(pool) + row * D + c);
        r.w[0] = make_uint4(u.x, u.y, 0, 0);
        r.scale = scales[row];
    } else {
        raw_row(r, static_cast<const T *>(pool) + row * D + c, 1);
    }
}

template <class T, bool E4M3>
__device__ __forceinline__ void raw_values(const Raw<T, E4M3> &r, float *x)
{
    if constexpr (E4M3) {
        const float s = scale_of(r.scale);
        const uint32_t u[2] = {r.w[0].x, r.w[0].y};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = e4m3_values((uint16_t)(u[i >> 1] >> (16 * (i & 1))));
            x[2 * i] = f.x * s;
            x[2 * i + 1] = f.y * s;
        }
    } else {
        const T *t = reinterpret_cast<const T *>(r.w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = TokType<T>::up(t[i]);
    }
}

// One row of a pool from eight values per lane (all lanes of the warp take part in the shuffles).
template <class T, bool E4M3>
__device__ __forceinline__ void put_row(const Raw<T, false> &raw, bool on, void *pool, uint8_t *scales, int64_t row, int D, int c, int lanes)
{
    if constexpr (!E4M3) {
        if (on) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(static_cast<T *>(pool) + row * D + c)[i] = raw.w[i];
        }
    } else {
        float x[8];
        uint32_t a = 0;                                  // the largest magnitude's bits (16-bit types: two at a time)
        if constexpr (sizeof(T) == 2) {
            const uint32_t u[4] = {raw.w[0].x, raw.w[0].y, raw.w[0].z, raw.w[0].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) a = __vmaxu2(a, u[q] & 0x7FFF7FFFu);
            a = max(a & 0xFFFFu, a >> 16);
        } else {
            const uint32_t *u = reinterpret_cast<const uint32_t *>(raw.w);
#pragma unroll
            for (int q = 0; q < 8; ++q) a = max(a, u[q] & 0x7FFFFFFFu);
        }
        a = on ? a : 0u;
        for (int s = lanes >> 1; s; s >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, s));
        if constexpr (sizeof(T) == 2) {
            const uint16_t h = (uint16_t)a;
            a = __float_as_uint(TokType<T>::up(*reinterpret_cast<const T *>(&h)));
        }
        raw_values(raw, x);
        const uint32_t byte = scale_byte(a);
        if (on) {
            uint32_t w[2];
#pragma unroll
            for (int q = 0; q < 2; ++q)
                w[q] = e4m3_pair(unscale(x[4 * q], byte), unscale(x[4 * q + 1], byte)) |
                       e4m3_pair(unscale(x[4 * q + 2], byte), unscale(x[4 * q + 3], byte)) << 16;
            *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(pool) + row * D + c) = byte == 255u ? make_uint2(0, 0) : make_uint2(w[0], w[1]);
            if (c == 0) scales[row] = (uint8_t)byte;
        }
    }
}

template <class T, bool E4M3>
__global__ void __launch_bounds__(kThreads) k_tokens_append(CellParams p)
{
    TokSeq sq;
    const Tile t = tile_of(p.b, false, sq);
    const int D = p.pool.d, c = (threadIdx.x & (p.lanes - 1)) * 8;
    const int32_t *table = p.b.table + sq.table0;
    const int rows = t.n * p.pool.hk, per = kThreads / p.lanes;
    for (int r0 = threadIdx.x / p.lanes; r0 - (int)(threadIdx.x / p.lanes) < rows; r0 += per * kRows) {
        Raw<T, false> k[kRows], v[kRows];
        int64_t row[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int r = r0 + u * per, h = r % p.pool.hk, i = r / p.pool.hk;
            k[u] = Raw<T, false>{};
            v[u] = Raw<T, false>{};
            row[u] = -1;
            if (r < rows && c < D) {
                row[u] = cell_row(p.pool, table, h, sq.pos + t.i0 + i);
                const int64_t token = sq.row0 + t.i0 + i;
                raw_row(k[u], reinterpret_cast<const T *>(p.k.p) + token * p.k.ts + h * p.k.hs + c, p.k.vec);
                raw_row(v[u], reinterpret_cast<const T *>(p.v.p) + token * p.v.ts + h * p.v.hs + c, p.v.vec);
            }
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            if (r0 - (int)(threadIdx.x / p.lanes) + u * per >= rows) break;      // (for all threads alike)
            put_row<T, E4M3>(k[u], row[u] >= 0, p.pool.k, p.pool.ks, row[u], D, c, p.lanes);
            put_row<T, E4M3>(v[u], row[u] >= 0, p.pool.v, p.pool.vs, row[u], D, c, p.lanes);
        }
    }
}

template <class T, bool E4M3>
__global__ void __launch_bounds__(kThreads) k_tokens_read(CellParams p)
{
    TokSeq sq;
    const Tile t = tile_of(p.b, p.part == 0, sq);
    const int D = p.pool.d, c = (threadIdx.x & (p.lanes - 1)) * 8;
    if (c >= D) return;
    const int32_t *table = p.b.table + sq.table0;
    const int rows = t.n * p.pool.hk, per = kThreads / p.lanes;
    const int64_t out0 = (p.part == 0 ? sq.cell0 : (int64_t)sq.row0) + t.i0;
    const int cell0 = (p.part == 0 ? 0 : sq.pos) + t.i0;
    for (int r0 = threadIdx.x / p.lanes; r0 < rows; r0 += per * kRows) {
        Raw<T, E4M3> k[kRows], v[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int r = r0 + u * per;
            if (r >= rows) break;
            const int64_t row = cell_row(p.pool, table, r % p.pool.hk, cell0 + r / p.pool.hk);
            raw_cell<T, E4M3>(k[u], p.pool.k, p.pool.ks, row, D, c);
            raw_cell<T, E4M3>(v[u], p.pool.v, p.pool.vs, row, D, c);
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int r = r0 + u * per;
            if (r >= rows) break;
            const int h = r % p.pool.hk;
            const int64_t at = out0 + r / p.pool.hk;
            float x[8], y[8];
            raw_values(k[u], x);
            raw_values(v[u], y);
            store8(reinterpret_cast<T *>(p.k.p) + at * p.k.ts + h * p.k.hs + c, p.k.vec, x);
            store8(reinterpret_cast<T *>(p.v.p) + at * p.v.ts + h * p.v.hs + c, p.v.vec, y);
        }
    }
}

// Whole pages of codes as 16-bit pages, in the order of the list.  bf16 holds every code times its scale (but for
// the last places of subnormals); f16 those of f16 rows that were appended, except the largest, whose code may
// have been rounded up past 65,504.  Values beyond become NaN: an infinity times a q of the other sign would look
// like a masked cell's score.
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
        if constexpr (std::is_same<T, __half>::value) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = fabsf(x[i]) <= 65504.f ? x[i] : NAN;
                y[i] = fabsf(y[i]) <= 65504.f ? y[i] : NAN;
            }
        }
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
