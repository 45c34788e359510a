// Token caches: pages copied, and cells of kept new tokens moved up.
//
// Both are copies that touch each byte once, bound by device memory where they are large and by the launch where they
// are small.  What is copied goes with the launch, as kernel arguments: a call needs no workspace, two calls share nothing,
// and nothing waits for an upload.
// Measured (GB300): 9,100 pages of 32 KB, keys and values, in three launches 193 us, 6.2 TB/s; 64 pages 3.7 us; kept paths
// of 24 trees, 8 heads of 128 bf16 values, 3.9 us: sequence, page and cell in a chain of loads.
#include <cstring>

#include "tokens_util.cuh"

namespace mure {

namespace {

// ------------------------------------------------------------------- pages --
constexpr int kThreads = 256;
constexpr int kWords = 4;                    // 16-byte words that a thread has on their way

// Pairs of a launch: three sizes, so that a short list does not carry a long one's arguments (65 to 512 small pages with
// arguments for 4,000: 1.1 us more).
template <int N>
struct PageParams {
    const char *from[4];                     // k, v, and their scales
    char *to[4];
    int64_t bytes[2];                        // of a page of codes or values, of its scales
    int32_t page[2 * N];
};

// blockIdx.x: a pair of pages; y: k or v; z: a share of the page.
template <int N>
__global__ void __launch_bounds__(kThreads) k_tokens_copy(const __grid_constant__ PageParams<N> p)
{
    const int64_t a = p.page[2 * blockIdx.x], b = p.page[2 * blockIdx.x + 1];
    const int which = blockIdx.y;
    {
        const uint4 *from = reinterpret_cast<const uint4 *>(p.from[which] + a * p.bytes[0]);
        uint4 *to = reinterpret_cast<uint4 *>(p.to[which] + b * p.bytes[0]);
        const int n = (int)(p.bytes[0] / 16);
        for (int i = blockIdx.z * kThreads * kWords + threadIdx.x; i < n; i += gridDim.z * kThreads * kWords) {
            uint4 w[kWords];
#pragma unroll
            for (int u = 0; u < kWords; ++u)
                if (i + u * kThreads < n) w[u] = from[i + u * kThreads];
#pragma unroll
            for (int u = 0; u < kWords; ++u)
                if (i + u * kThreads < n) to[i + u * kThreads] = w[u];
        }
    }
    if (p.bytes[1] && blockIdx.z == 0) {                             // (pages of 8 cells and up: a multiple of 8 bytes)
        const uint2 *from = reinterpret_cast<const uint2 *>(p.from[2 + which] + a * p.bytes[1]);
        uint2 *to = reinterpret_cast<uint2 *>(p.to[2 + which] + b * p.bytes[1]);
        for (int i = threadIdx.x; i < (int)(p.bytes[1] / 8); i += kThreads) to[i] = from[i];
    }
}

template <int N>
void copy(const TokPool &from, const TokPool &to, int64_t bytes, int64_t scale_bytes, const int32_t *pages, int n, cudaStream_t s)
{
    static_assert(sizeof(PageParams<N>) <= 32764, "more than a kernel's arguments");
    PageParams<N> p;
    p.from[0] = static_cast<const char *>(from.k); p.from[1] = static_cast<const char *>(from.v);
    p.from[2] = reinterpret_cast<const char *>(from.ks); p.from[3] = reinterpret_cast<const char *>(from.vs);
    p.to[0] = static_cast<char *>(to.k); p.to[1] = static_cast<char *>(to.v);
    p.to[2] = reinterpret_cast<char *>(to.ks); p.to[3] = reinterpret_cast<char *>(to.vs);
    p.bytes[0] = bytes; p.bytes[1] = scale_bytes;
    memcpy(p.page, pages, (size_t)n * 2 * sizeof(int32_t));
    const int64_t z = (bytes / 16 + kThreads * kWords - 1) / (kThreads * kWords);
    k_tokens_copy<N><<<dim3(n, 2, (unsigned)(z < 1024 ? z : 1024)), kThreads, 0, s>>>(p);
}

// ------------------------------------------------------------------- cells --
template <int S, int I>                      // sequences and indexes of a launch: two sizes, as above
struct KeepParams {
    TokPool pool;
    const TokSeq *seq;
    const int32_t *table;
    int elt;                                 // bytes of a value, or of a code
    int scales;
    int lanes;                               // threads of a row, a power of two: 8 values each
    int32_t of[S], first[S + 1], to[S];
    int32_t index[I];
};

struct alignas(16) Wide { uint4 a, b; };

// A block moves the cells of one sequence and cached head, a group of threads one cell's rows: four cells a group are
// in registers before any is written.  As the indexes ascend, a later source lies behind every target before it, so that
// the next round's sources are still whole.
template <class W, int S, int I>             // eight values: Wide (fp32), uint4 (16 bits), uint2 (codes)
__global__ void __launch_bounds__(128) k_tokens_keep(const __grid_constant__ KeepParams<S, I> p)
{
    const int b = blockIdx.x, h = blockIdx.y;
    const TokSeq sq = p.seq[p.of[b]];
    const int32_t *table = p.table + sq.table0;
    const int D = p.pool.d, slot = threadIdx.x & (p.lanes - 1), c = slot * 8, group = threadIdx.x / p.lanes, groups = 128 / p.lanes;
    const int i0 = p.first[b], n = p.first[b + 1] - i0;
    constexpr int U = 4;
    for (int base = 0; base < n; base += groups * U) {
        W k[U], v[U];
        uint32_t scale[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + group + u * groups;
            if (i < n && c < D) {
                const int64_t row = cell_row(p.pool, table, h, sq.pos + p.index[i0 + i]);
                k[u] = *reinterpret_cast<const W *>(static_cast<const char *>(p.pool.k) + (row * D + c) * p.elt);
                v[u] = *reinterpret_cast<const W *>(static_cast<const char *>(p.pool.v) + (row * D + c) * p.elt);
                if (p.scales && slot == 0) scale[u] = p.pool.ks[row] | (uint32_t)p.pool.vs[row] << 8;
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + group + u * groups;
            if (i < n && c < D) {
                const int64_t row = cell_row(p.pool, table, h, sq.pos + p.to[b] + i);
                *reinterpret_cast<W *>(static_cast<char *>(p.pool.k) + (row * D + c) * p.elt) = k[u];
                *reinterpret_cast<W *>(static_cast<char *>(p.pool.v) + (row * D + c) * p.elt) = v[u];
                if (p.scales && slot == 0) {
                    p.pool.ks[row] = (uint8_t)scale[u];
                    p.pool.vs[row] = (uint8_t)(scale[u] >> 8);
                }
            }
        }
    }
}

template <int S, int I>
int keep(const TokPool &pool, const TokBatch &b, int elt, bool scales, const int32_t *seq, const int32_t *first, const int32_t *end,
         const int32_t *to, const int32_t *index, int64_t n, cudaStream_t s)
{
    static_assert(sizeof(KeepParams<S, I>) <= 32764, "more than a kernel's arguments");
    const int lanes = row_lanes(pool.d);
    int launches = 0;
    int64_t i = 0;
    int32_t at = first[0];                   // the next index of sequence i's
    while (i < n) {
        KeepParams<S, I> p;
        p.pool = pool; p.seq = b.seq; p.table = b.table;
        p.elt = elt; p.scales = scales; p.lanes = lanes;
        int seqs = 0, used = 0;
        while (i < n && seqs < S && used < I) {
            const int take = end[i] - at < I - used ? end[i] - at : I - used;
            p.of[seqs] = seq[i];
            p.first[seqs] = used;
            p.to[seqs] = to[i] + (at - first[i]);
            memcpy(p.index + used, index + at, (size_t)take * sizeof(int32_t));
            used += take;
            at += take;
            ++seqs;
            if (at < end[i]) break;          // the rest of a long list follows in the stream's order
            ++i;
            if (i < n) at = first[i];
        }
        p.first[seqs] = used;
        const dim3 grid(seqs, pool.hk);
        if (elt == 4) k_tokens_keep<Wide, S, I><<<grid, 128, 0, s>>>(p);
        else if (elt == 2) k_tokens_keep<uint4, S, I><<<grid, 128, 0, s>>>(p);
        else k_tokens_keep<uint2, S, I><<<grid, 128, 0, s>>>(p);
        ++launches;
    }
    return launches;
}

}  // namespace

int launch_tokens_copy_pages(const TokPool &from, const TokPool &to, int elt, bool scales, const int32_t *pages, int64_t n, cudaStream_t s)
{
    constexpr int kShort = 64, kMiddle = 512, kLong = 4000;
    const int64_t cells = (int64_t)from.hk << from.page_log2;
    int launches = 0;
    for (int64_t i = 0; i < n;) {
        const int take = (int)(n - i < kLong ? n - i : kLong);
        if (take <= kShort) copy<kShort>(from, to, cells * from.d * elt, scales ? cells : 0, pages + 2 * i, take, s);
        else if (take <= kMiddle) copy<kMiddle>(from, to, cells * from.d * elt, scales ? cells : 0, pages + 2 * i, take, s);
        else copy<kLong>(from, to, cells * from.d * elt, scales ? cells : 0, pages + 2 * i, take, s);
        i += take;
        ++launches;
    }
    return launches;
}

int launch_tokens_keep(const TokPool &pool, const TokBatch &b, int elt, bool scales, const int32_t *seq, const int32_t *first,
                       const int32_t *end, const int32_t *to, const int32_t *index, int64_t n, cudaStream_t s)
{
    if (n == 0) return 0;
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i) total += end[i] - first[i];
    return n <= 64 && total <= 768 ? keep<64, 768>(pool, b, elt, scales, seq, first, end, to, index, n, s)
                                   : keep<512, 6000>(pool, b, elt, scales, seq, first, end, to, index, n, s);
}

}  // namespace mure
