// Token caches: the handles behind the C entry points, and the checks that their calls share.
#pragma once

#include "host.cuh"
#include "tokens.cuh"

struct mure_tokens {
    mure_ctx *ctx = nullptr;
    mure_tokens_desc d{};
    void *own = nullptr;      // the library's allocation of the pools (null: the caller's pools)
    CUtensorMap map_k, map_v; // 16-bit types of up to kChunkDim values: the pools (codes: of multiples of 16 values)
};

struct mure_tokens_plan {
    mure_ctx *ctx = nullptr;
    mure_tokens_desc d{};     // the geometry it serves (pools ignored)
    bool ready = false;
    std::vector<mure::TokSeq> seq;           // the batch's sequences, as on the device
    mure::TokBatch b;
    int64_t n_new = 0, n_cells = 0;          // packed rows of the new tokens / of all cells
    int64_t tiles_new = 0, tiles_all = 0;
    int new_past_end = -1;                   // a sequence whose new tokens end past its cells
    std::string append_fault;                // why the batch's new tokens cannot be written ("" if they can)
    mure::TokWork few;                             // 16-bit types: the rows that the kernel for few rows takes
    mure::TokChunk chunk;                          // ... and those that the kernel for chunks takes
    mure::TokChunk tree;                           // ... and those that the kernel for trees takes
    // E4M3: the pages that chunks read, as 16-bit pages
    const int32_t *wide_pages = nullptr, *wide_table = nullptr;
    int64_t n_wide = 0;
    bool fused = false;                      // E4M3 trees: the pieces widen codes themselves
    CUtensorMap map_k, map_v;
    void *mem = nullptr, *part = nullptr, *wide = nullptr;    // tables; partial results; 16-bit pages
    size_t mem_bytes = 0, part_bytes = 0, wide_bytes = 0;
};

namespace mure {

constexpr int64_t kMostStride = int64_t(1) << 40;

// Ids of a set, by open addressing: whether one of them, twice or a probe, is there.  A slot goes by the product's high bits,
// which all of an id's bits reach: by its low ones, ids that are multiples of a power of two would share few slots.
struct IdSet {
    std::vector<int32_t> slot;
    uint32_t mask;
    int shift = 28;                             // 32 less the bits of a slot's number
    explicit IdSet(int64_t n)
    {
        uint32_t size = 16;
        for (; size < 2 * (uint64_t)n && size < (1u << 31); size *= 2) --shift;
        slot.assign(size, -1);
        mask = size - 1;
    }
    uint32_t at(int32_t id) const
    {
        uint32_t i = (uint32_t)id * 2654435761u >> shift;
        while (slot[i] != -1 && slot[i] != id) i = (i + 1) & mask;
        return i;
    }
    bool insert(int32_t id)                     // false: it was there
    {
        const uint32_t i = at(id);
        if (slot[i] == id) return false;
        slot[i] = id;
        return true;
    }
    bool has(int32_t id) const { return slot[at(id)] == id; }
};

inline int elt_bytes(int dtype) { return dtype == MURE_F32 ? 4 : 2; }

inline int log2_of(int n)
{
    int l = 0;
    while ((1 << l) < n) ++l;
    return l;
}

inline TokPool pool_of(const mure_tokens *t)
{
    TokPool p;
    p.k = t->d.k; p.v = t->d.v; p.ks = t->d.k_scale; p.vs = t->d.v_scale;
    p.hk = t->d.n_kv_heads; p.d = t->d.head_dim; p.page_log2 = log2_of(t->d.page_size);
    return p;
}

// A call's cache and plan.
inline void check_pair(mure_ctx *c, const mure_tokens *t, const mure_tokens_plan *p)
{
    FAILIF(!p, c, MURE_ERR_INVALID_ARG, "NULL plan");
    FAILIF(p->ctx != c, c, MURE_ERR_INVALID_ARG, "cache and plan belong to different contexts");
    FAILIF(!p->ready, c, MURE_ERR_INVALID_ARG, "the plan holds no batch");
    const mure_tokens_desc &a = t->d, &b = p->d;
    FAILIF(a.n_kv_heads != b.n_kv_heads || a.head_dim != b.head_dim || a.page_size != b.page_size || a.dtype != b.dtype ||
               a.form != b.form || a.n_pages != b.n_pages,
           c, MURE_ERR_INVALID_ARG, "the plan was made for caches of another geometry");
}

inline TokRows check_rows(mure_ctx *c, const mure_tokens_rows *r, const mure_tokens_desc &d, int64_t rows, int heads, const char *name)
{
    TokRows o;
    if (rows == 0) return o;
    const int e = elt_bytes(d.dtype);
    FAILIF(!r || !r->p, c, MURE_ERR_INVALID_ARG, "NULL %s", name);
    FAILIF((uintptr_t)r->p % e != 0, c, MURE_ERR_INVALID_ARG, "%s is not aligned to its type", name);
    o.p = static_cast<char *>(r->p);
    FAILIF(r->token_stride < 0 || r->head_stride < 0 || r->token_stride > kMostStride || r->head_stride > kMostStride, c,
           MURE_ERR_INVALID_ARG, "a stride of %s is not in 0..2^40", name);
    o.ts = r->token_stride;
    o.hs = r->head_stride;
    const int per = 16 / e;
    o.vec = (uintptr_t)r->p % 16 == 0 && (rows == 1 || o.ts % per == 0) && (heads == 1 || o.hs % per == 0);
    return o;
}

// Rows that are written must not lie on one another.
inline void check_apart(mure_ctx *c, const TokRows &r, const mure_tokens_desc &d, int64_t rows, int heads, const char *name)
{
    if (rows == 0) return;
    const int64_t ts = r.ts, hs = r.hs, D = d.head_dim;
    const bool ok = (heads == 1 || rows == 1) ? (heads == 1 || hs >= D) && (rows == 1 || ts >= D)
                                              : (hs >= D && ts >= hs * (heads - 1) + D) || (ts >= D && hs >= ts * (rows - 1) + D);
    FAILIF(!ok, c, MURE_ERR_INVALID_ARG, "rows of %s overlap", name);
}

}  // namespace mure
