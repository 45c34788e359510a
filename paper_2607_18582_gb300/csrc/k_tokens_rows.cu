// Token caches: attention by the definition, a warp per (new token, query head).
#include "tokens_util.cuh"

namespace mure {

namespace {

constexpr int kWarps = 4;

struct RowParams {
    TokPool pool;
    TokBatch b;
    TokRows q, out;
    float *lse;
    int64_t n_tokens;
};

template <class T, bool E4M3>
__global__ void __launch_bounds__(kWarps * 32) k_tokens_attend_rows(RowParams p)
{
    const int lane = threadIdx.x & 31;
    for (int64_t r = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; r < p.n_tokens * p.b.n_heads;
         r += (int64_t)gridDim.x * kWarps) {
        const int token = (int)(r / p.b.n_heads), head = (int)(r % p.b.n_heads);
        // the sequence: the last one that starts at or before the token and has new tokens
        int lo = 0, len = p.b.n_seqs;
        while (len > 1) {
            const int half = len / 2;
            if (p.b.seq[lo + half].row0 <= token) { lo += half; len -= half; }
            else len = half;
        }
        const TokSeq sq = p.b.seq[lo];
        const T *q = reinterpret_cast<const T *>(p.q.p) + token * p.q.ts + head * p.q.hs;
        float o[8], m, l;
        attend_row<T, E4M3>(p.pool, p.b.table + sq.table0, head / p.b.group, q, p.q.vec,
                            sq.pos + token - sq.row0, 0, sq.kv, p.b.window, p.b.sinks, p.b.scale_log2, o, m, l);
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] *= inv;
        if (lane * 8 < p.pool.d)
            store8(reinterpret_cast<T *>(p.out.p) + token * p.out.ts + head * p.out.hs + lane * 8, p.out.vec, o);
        if (p.lse && lane == 0) p.lse[r] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945f;
    }
}

template <class T>
int go(const RowParams &p, int form, cudaStream_t s)
{
    const int64_t rows = p.n_tokens * p.b.n_heads;
    const unsigned grid = (unsigned)(rows / kWarps + 1 < 65536 ? rows / kWarps + 1 : 65536);
    if (form == MURE_FORM_E4M3) k_tokens_attend_rows<T, true><<<grid, kWarps * 32, 0, s>>>(p);
    else k_tokens_attend_rows<T, false><<<grid, kWarps * 32, 0, s>>>(p);
    return 1;
}

}  // namespace

int launch_tokens_attend_rows(const TokPool &pool, const TokBatch &b, int dtype, int form, int64_t n_tokens, TokRows q,
                              TokRows out, float *lse, cudaStream_t s)
{
    if (n_tokens == 0) return 0;
    const RowParams p{pool, b, q, out, lse, n_tokens};
    if (dtype == MURE_F32) return go<float>(p, form, s);
    if (dtype == MURE_F16) return go<__half>(p, form, s);
    return go<__nv_bfloat16>(p, form, s);
}

}  // namespace mure
