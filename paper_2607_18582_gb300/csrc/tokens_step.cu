// Token caches: the C entry points of what surrounds an attention call: norm and rotation of the new tokens' queries and
// keys, pages copied, cells of kept tokens moved up.
#include <cmath>
#include <memory>

#include "tokens_host.cuh"

using namespace mure;

struct mure_rotary {
    mure_ctx *ctx = nullptr;
    int head_dim = 0;
    TokRotary r;
    void *mem = nullptr;
};

namespace {

// Turns per position of `radians` per position as a 64-bit fraction, modulo 1.  1 / (2 pi) as the sum of two doubles, so that
// the product's error lies far below 2^-64 of a turn for magnitudes up to 2^20.
uint64_t turn_of(double radians)
{
    if (radians < 0) return 0 - turn_of(-radians);
    constexpr double kHi = 0x1.45f306dc9c883p-3, kLo = -0x1.6b01ec5417056p-57;      // 1 / (2 pi), to some 2^-112
    const double hi = radians * kHi, lo = std::fma(radians, kHi, -hi) + radians * kLo;
    const double part = hi - std::floor(hi);                                        // exact, as what follows
    const double up = std::floor(part * 0x1p32), rest = part * 0x1p32 - up;
    // (lo is at most 2^-35: in units of 2^-64 a signed number)
    return ((uint64_t)up << 32) + (uint64_t)std::floor(rest * 0x1p32) + (uint64_t)(int64_t)std::nearbyint(lo * 0x1p64);
}

void check_rotary(mure_ctx *c, const mure_tokens *t, const mure_tokens_plan *p, const mure_rotary *r, const int32_t *positions,
                  int64_t stride)
{
    FAILIF(!r, c, MURE_ERR_INVALID_ARG, "NULL rotary");
    FAILIF(r->ctx != c, c, MURE_ERR_INVALID_ARG, "cache and rotary belong to different contexts");
    FAILIF(r->head_dim != t->d.head_dim, c, MURE_ERR_INVALID_ARG, "the rotary has heads of %d values, the cache of %d", r->head_dim,
           t->d.head_dim);
    FAILIF((uintptr_t)positions % 4 != 0, c, MURE_ERR_INVALID_ARG, "positions are not aligned");
    FAILIF(positions && (stride < p->n_new || stride > kMostStride), c, MURE_ERR_INVALID_ARG,
           "position_stride %lld is not in %lld..2^40", (long long)stride, (long long)p->n_new);
}

int cell_bytes(const mure_tokens_desc &d) { return d.form == MURE_FORM_E4M3 ? 1 : elt_bytes(d.dtype); }

}  // namespace

extern "C" {

mure_status mure_rotary_create(mure_ctx *c, const mure_rotary_desc *desc, mure_rotary **out)
{
    if (!c) return MURE_ERR_INVALID_ARG;
    return run(c, [&] {
        FAILIF(!out, c, MURE_ERR_INVALID_ARG, "NULL out");
        *out = nullptr;
        FAILIF(!desc, c, MURE_ERR_INVALID_ARG, "NULL description");
        const mure_rotary_desc &d = *desc;
        FAILIF(d.head_dim < 8 || d.head_dim > 256 || d.head_dim % 8, c, MURE_ERR_INVALID_ARG,
               "head_dim %d is not a multiple of 8 in 8..256", d.head_dim);
        FAILIF(d.rot_dim < 0 || d.rot_dim > d.head_dim || d.rot_dim % 8, c, MURE_ERR_INVALID_ARG,
               "rot_dim %d is not a multiple of 8 in 0..%d", d.rot_dim, d.head_dim);
        FAILIF(d.pairs != MURE_PAIRS_HALVES && d.pairs != MURE_PAIRS_ADJACENT, c, MURE_ERR_UNSUPPORTED, "unknown pairs %d", d.pairs);
        FAILIF(d.n_axes < 1 || d.n_axes > 8, c, MURE_ERR_INVALID_ARG, "n_axes %d not in 1..8", d.n_axes);
        FAILIF(!(d.eps >= 0.f && d.eps <= 1.f), c, MURE_ERR_INVALID_ARG, "eps must be in 0..1");
        FAILIF(d.reserved != 0, c, MURE_ERR_INVALID_ARG, "reserved fields must be 0");
        FAILIF(!d.freq && d.rot_dim > 0 && !(d.base > 0 && std::isfinite(d.base)), c, MURE_ERR_INVALID_ARG, "base must be positive");
        const int half = d.rot_dim / 2, D = d.head_dim;
        std::vector<char> image((size_t)half * 8 + 2 * D * 4 + half);
        uint64_t *turn = reinterpret_cast<uint64_t *>(image.data());
        float *weight = reinterpret_cast<float *>(image.data() + half * 8);
        uint8_t *axis = reinterpret_cast<uint8_t *>(image.data() + half * 8 + 2 * D * 4);
        for (int i = 0; i < half; ++i) {
            const double f = d.freq ? d.freq[i] : std::pow(d.base, -2.0 * i / d.rot_dim);
            FAILIF(!(std::fabs(f) <= 0x1p20), c, MURE_ERR_INVALID_ARG, "frequency %d is not in -2^20..2^20", i);
            FAILIF(d.axis && d.axis[i] >= d.n_axes, c, MURE_ERR_INVALID_ARG, "pair %d: axis %d of %d", i, d.axis[i], d.n_axes);
            turn[i] = turn_of(f);
            axis[i] = d.axis ? d.axis[i] : 0;
        }
        for (int i = 0; i < D; ++i) {
            weight[i] = d.q_weight ? d.q_weight[i] : 1.f;
            weight[D + i] = d.k_weight ? d.k_weight[i] : 1.f;
        }
        CK(c, cudaSetDevice(c->device));
        auto r = std::make_unique<mure_rotary>();
        r->ctx = c;
        r->head_dim = D;
        char *m = static_cast<char *>(dalloc(c, image.size()));
        // (a few KB from pageable memory: taken in when the call returns)
        const cudaError_t e = cudaMemcpyAsync(m, image.data(), image.size(), cudaMemcpyHostToDevice, c->stream);
        if (e != cudaSuccess) dfree(c, m);
        CK(c, e);
        r->mem = m;
        r->r.turn = reinterpret_cast<uint64_t *>(m);
        r->r.weight = reinterpret_cast<float *>(m + half * 8);
        r->r.axis = reinterpret_cast<uint8_t *>(m + half * 8 + 2 * D * 4);
        r->r.rot = d.rot_dim;
        r->r.adjacent = d.pairs == MURE_PAIRS_ADJACENT;
        r->r.norm_q = d.q_weight != nullptr;
        r->r.norm_k = d.k_weight != nullptr;
        r->r.eps = d.eps;
        *out = r.release();
    });
}

void mure_rotary_free(mure_rotary *r)
{
    if (!r) return;
    dfree(r->ctx, r->mem);
    delete r;
}

mure_status mure_tokens_rotate(mure_tokens *t, mure_tokens_plan *p, const mure_rotary *rotary, const int32_t *positions,
                               int64_t position_stride, const mure_tokens_rows *q, const mure_tokens_rows *k,
                               const mure_tokens_rows *q_out, const mure_tokens_rows *k_out)
{
    if (!t) return MURE_ERR_INVALID_ARG;
    mure_ctx *c = t->ctx;
    return run(c, [&] {
        check_pair(c, t, p);
        check_rotary(c, t, p, rotary, positions, position_stride);
        FAILIF(!q != !q_out || !k != !k_out, c, MURE_ERR_INVALID_ARG, "an input without its output, or an output without its input");
        const int hq = q ? p->b.n_heads : 0, hk = k ? t->d.n_kv_heads : 0;
        const int64_t n = p->n_new;
        TokRows qr, kr, qo, ko;
        if (q) {
            qr = check_rows(c, q, t->d, n, hq, "q");
            qo = check_rows(c, q_out, t->d, n, hq, "q_out");
            check_apart(c, qo, t->d, n, hq, "q_out");
        }
        if (k) {
            kr = check_rows(c, k, t->d, n, hk, "k");
            ko = check_rows(c, k_out, t->d, n, hk, "k_out");
            check_apart(c, ko, t->d, n, hk, "k_out");
        }
        CK(c, cudaSetDevice(c->device));
        TokRotary r = rotary->r;
        r.positions = positions;
        r.position_stride = position_stride;
        c->launches += launch_tokens_rotate(pool_of(t), p->b, r, t->d.dtype, t->d.form, false, hq, hk, qr, kr, TokRows{}, qo, ko,
                                            n, p->tiles_new, c->stream);
        check_launch(c);
    });
}

mure_status mure_tokens_append_rotated(mure_tokens *t, mure_tokens_plan *p, const mure_rotary *rotary, const int32_t *positions,
                                       int64_t position_stride, const mure_tokens_rows *q, const mure_tokens_rows *k,
                                       const mure_tokens_rows *v, const mure_tokens_rows *q_out)
{
    if (!t) return MURE_ERR_INVALID_ARG;
    mure_ctx *c = t->ctx;
    return run(c, [&] {
        check_pair(c, t, p);
        check_rotary(c, t, p, rotary, positions, position_stride);
        FAILIF(!p->append_fault.empty(), c, MURE_ERR_INVALID_ARG, "%s", p->append_fault.c_str());
        FAILIF(!q != !q_out, c, MURE_ERR_INVALID_ARG, "an input without its output, or an output without its input");
        const int hq = q ? p->b.n_heads : 0, hk = t->d.n_kv_heads;
        const int64_t n = p->n_new;
        TokRows qr, qo;
        if (q) {
            qr = check_rows(c, q, t->d, n, hq, "q");
            qo = check_rows(c, q_out, t->d, n, hq, "q_out");
            check_apart(c, qo, t->d, n, hq, "q_out");
        }
        const TokRows kr = check_rows(c, k, t->d, n, hk, "k"), vr = check_rows(c, v, t->d, n, hk, "v");
        CK(c, cudaSetDevice(c->device));
        TokRotary r = rotary->r;
        r.positions = positions;
        r.position_stride = position_stride;
        c->launches += launch_tokens_rotate(pool_of(t), p->b, r, t->d.dtype, t->d.form, true, hq, hk, qr, kr, vr, qo, TokRows{},
                                            n, p->tiles_new, c->stream);
        check_launch(c);
    });
}

mure_status mure_tokens_copy_pages(mure_tokens *to, const mure_tokens *from, int64_t n, const int32_t *from_pages,
                                   const int32_t *to_pages)
{
    if (!to) return MURE_ERR_INVALID_ARG;
    mure_ctx *c = to->ctx;
    return run(c, [&] {
        FAILIF(!from, c, MURE_ERR_INVALID_ARG, "NULL cache");
        FAILIF(from->ctx != c, c, MURE_ERR_INVALID_ARG, "the caches belong to different contexts");
        const mure_tokens_desc &a = from->d, &b = to->d;
        FAILIF(a.n_kv_heads != b.n_kv_heads || a.head_dim != b.head_dim || a.page_size != b.page_size || a.dtype != b.dtype ||
                   a.form != b.form,
               c, MURE_ERR_INVALID_ARG, "the caches have different geometries");
        FAILIF(n < 0, c, MURE_ERR_INVALID_ARG, "a negative number of pages");
        if (n == 0) return;
        FAILIF(!from_pages || !to_pages, c, MURE_ERR_INVALID_ARG, "NULL pages");
        FAILIF(n > b.n_pages, c, MURE_ERR_INVALID_ARG, "%lld targets, and %lld pages", (long long)n, (long long)b.n_pages);
        // two handles on one memory (a caller's pools) are one cache, whole or not at all
        const bool same = a.k == b.k && a.v == b.v && a.k_scale == b.k_scale && a.v_scale == b.v_scale;
        const int64_t page = (int64_t)a.n_kv_heads * a.page_size, bytes = page * a.head_dim * cell_bytes(a);
        if (!same) {
            const struct { const void *p; int64_t n; } in[4] = {{a.k, a.n_pages * bytes}, {a.v, a.n_pages * bytes},
                                                               {a.k_scale, a.n_pages * page}, {a.v_scale, a.n_pages * page}},
                                                       at[4] = {{b.k, b.n_pages * bytes}, {b.v, b.n_pages * bytes},
                                                                {b.k_scale, b.n_pages * page}, {b.v_scale, b.n_pages * page}};
            for (const auto &x : in)
                for (const auto &y : at)
                    FAILIF(x.p && y.p && (uintptr_t)x.p < (uintptr_t)y.p + y.n && (uintptr_t)y.p < (uintptr_t)x.p + x.n, c,
                           MURE_ERR_INVALID_ARG, "the caches' pools overlap in part");
        }
        IdSet targets(n);
        std::vector<int32_t> pairs((size_t)n * 2);
        for (int64_t i = 0; i < n; ++i) {
            FAILIF(from_pages[i] < 0 || from_pages[i] >= a.n_pages, c, MURE_ERR_INVALID_ARG, "page %d not in 0..%lld", from_pages[i],
                   (long long)a.n_pages - 1);
            FAILIF(to_pages[i] < 0 || to_pages[i] >= b.n_pages, c, MURE_ERR_INVALID_ARG, "page %d not in 0..%lld", to_pages[i],
                   (long long)b.n_pages - 1);
            FAILIF(!targets.insert(to_pages[i]), c, MURE_ERR_INVALID_ARG, "page %d is a target twice", to_pages[i]);
            pairs[2 * i] = from_pages[i];
            pairs[2 * i + 1] = to_pages[i];
        }
        for (int64_t i = 0; same && i < n; ++i)
            FAILIF(targets.has(from_pages[i]), c, MURE_ERR_INVALID_ARG, "page %d is both a source and a target", from_pages[i]);
        CK(c, cudaSetDevice(c->device));
        c->launches += launch_tokens_copy_pages(pool_of(from), pool_of(to), cell_bytes(a), a.form == MURE_FORM_E4M3, pairs.data(), n,
                                                c->stream);
        check_launch(c);
    });
}

mure_status mure_tokens_keep(mure_tokens *t, mure_tokens_plan *p, const int32_t *count, const int32_t *index)
{
    if (!t) return MURE_ERR_INVALID_ARG;
    mure_ctx *c = t->ctx;
    return run(c, [&] {
        check_pair(c, t, p);
        FAILIF(!p->append_fault.empty(), c, MURE_ERR_INVALID_ARG, "%s", p->append_fault.c_str());
        const int n = (int)p->seq.size();
        if (n == 0) return;
        FAILIF(!count, c, MURE_ERR_INVALID_ARG, "NULL count");
        std::vector<int32_t> seq, first, end, to;
        int64_t at = 0;
        for (int b = 0; b < n; ++b)              // (all of them before any index, whose number they add up to)
            FAILIF(count[b] < 0 || count[b] > p->seq[b].n_new, c, MURE_ERR_INVALID_ARG, "sequence %d: %d kept of %d new tokens", b, count[b],
                   p->seq[b].n_new);
        for (int b = 0; b < n; ++b) {
            if (count[b] == 0) continue;
            FAILIF(!index, c, MURE_ERR_INVALID_ARG, "NULL index");
            int still = 0;                       // the first ones that are where they are to be
            for (int k = 0; k < count[b]; ++k) {
                const int32_t i = index[at + k];
                FAILIF(i < 0 || i >= p->seq[b].n_new || (k > 0 && i <= index[at + k - 1]), c, MURE_ERR_INVALID_ARG,
                       "sequence %d: kept token %d is %d: not an ascending index of its %d new tokens", b, k, i, p->seq[b].n_new);
                still += i == k;                 // (indexes ascend: once one is past its place, all are)
            }
            if (still < count[b]) {
                seq.push_back(b);
                first.push_back((int32_t)(at + still));
                to.push_back(still);
                end.push_back((int32_t)(at + count[b]));
            }
            at += count[b];
        }
        if (seq.empty()) return;
        CK(c, cudaSetDevice(c->device));
        c->launches += launch_tokens_keep(pool_of(t), p->b, cell_bytes(t->d), t->d.form == MURE_FORM_E4M3, seq.data(), first.data(),
                                          end.data(), to.data(), index, (int64_t)seq.size(), c->stream);
        check_launch(c);
    });
}

}  // extern "C"
