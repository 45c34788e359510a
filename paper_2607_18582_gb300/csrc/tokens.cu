// Token caches: the C entry points, and the host's layout of a batch's work.
//
// Lengths and page tables are host arrays, as the mutant tables are.  So every check runs before
// anything is queued, no kernel can meet a page or a length out of range, and the work can be
// laid out knowing every sequence's length.  A plan holds a batch's tables on the device; all
// layers' calls of a step share it.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <numeric>
#include <queue>
#include <unordered_map>

#include "tokens_host.cuh"

using namespace mure;

namespace {

// Rows of a sequence and cached head up to which the kernel for few rows takes them; it reads the cells
// again for every 16.  16 sequences of 4,000 cells, 8 heads (few rows / chunk, us): 128 values, 32 rows
// 70 / 58; 64 values, 32 rows 45 / 50, 64 rows 70 / 51; codes, whose pages a chunk's kernel wants
// widened first, 128 values, 64 rows 126 / 137, 128 rows 225 / 138, 64 values 90 / 92 and 164 / 93.
// (Measured at that one shape.  fp32 rows, and heads of more than 128 values, have no other kernel.)
int few_rows_up_to(bool codes, int d) { return codes ? 64 : d <= 64 ? 32 : 16; }
// Trees, whose pieces widen codes themselves (48 sequences of 4,000 cells, 8 heads, no other shape; few / the others, us): codes of 128
// values, 24 rows 177 / 200, 32 177 / 201, 48 248 / 202, of 64 values, 32 128 / 193, 48 182 / 193, 64 236 / 193; cells as they are, of
// 128 values, 16 rows 144 / 154, 24 163 / 155, of 64 values, 32 95 / 115, 48 124 / 112.
int few_tree_rows_up_to(bool codes, int d) { return codes && d % 16 == 0 ? (d <= 64 ? 48 : 32) : few_rows_up_to(codes, d); }

constexpr int64_t kMostPos = int64_t(1) << 30, kMostUnits = int64_t(1) << 24;

void check_geometry(mure_ctx *c, const mure_tokens_desc &d)
{
    FAILIF(d.dtype != MURE_F32 && d.dtype != MURE_F16 && d.dtype != MURE_BF16, c, MURE_ERR_UNSUPPORTED, "unknown dtype %d",
           d.dtype);
    FAILIF(d.form != MURE_FORM_SAME && d.form != MURE_FORM_E4M3, c, MURE_ERR_UNSUPPORTED, "unknown form %d", d.form);
    FAILIF(d.n_kv_heads < 1 || d.n_kv_heads > 1024, c, MURE_ERR_INVALID_ARG, "n_kv_heads %d not in 1..1024", d.n_kv_heads);
    FAILIF(d.head_dim < 8 || d.head_dim > 256 || d.head_dim % 8, c, MURE_ERR_INVALID_ARG,
           "head_dim %d is not a multiple of 8 in 8..256", d.head_dim);
    FAILIF(d.page_size < 8 || d.page_size > 1024 || (d.page_size & (d.page_size - 1)), c, MURE_ERR_INVALID_ARG,
           "page_size %d is not a power of two in 8..1024", d.page_size);
    FAILIF(d.n_pages < 1 || d.n_pages > INT32_MAX, c, MURE_ERR_INVALID_ARG, "n_pages %lld not in 1..2^31 - 1",
           (long long)d.n_pages);
    FAILIF(d.reserved != 0, c, MURE_ERR_INVALID_ARG, "reserved fields must be 0");
}

// At least `bytes` of device memory, and up to 16 MiB more where it grows (the next steps' tables do).
void reserve(mure_ctx *c, void *&mem, size_t &have, size_t bytes)
{
    if (bytes <= have) return;
    dfree(c, mem);
    mem = nullptr;
    have = 0;
    const size_t room = bytes + std::min<size_t>(bytes / 4, 16 << 20);
    mem = dalloc(c, room);
    have = room;
}

// Host bytes to the device, in the stream's order.  A copy from pageable memory has taken its source when it
// returns; up to 64 KB of it return without waiting for the stream, more do wait.  So larger tables go in
// pieces, up to the 1 MiB that the driver takes in without waiting in its turn (150 KB behind 17 ms of
// queued work: 17 ms in one copy, 31 us in three; 1 MiB 93 us; 8 MiB wait in pieces too).
void upload(mure_ctx *c, void *dst, const char *src, size_t bytes)
{
    constexpr size_t kPiece = 64 << 10, kInPieces = 1 << 20;
    const size_t piece = bytes <= kInPieces ? kPiece : bytes;
    for (size_t at = 0; at < bytes; at += piece)
        CK(c, cudaMemcpyAsync(static_cast<char *>(dst) + at, src + at, std::min(piece, bytes - at), cudaMemcpyHostToDevice, c->stream));
}

// Rows [r0, r0 + rows) of sequence s and head h and the tiles of the cells that they may attend to.
struct Unit {
    TokItem item;
    int tiles;
};

// What a kernel's pieces are made of.  (`start` and `half` were set on ragged chunks, 12 of 90 to 700 tokens over up to
// 6,000 cells; they decide how the work is shared out, not what comes out.)
struct Shape {
    int rows;      // of a piece
    int tile;      // cells
    int align;     // of the first tile past the sinks
    int blocks;    // that run at a time
    int least;     // tiles of a part, at least
    double start;  // a unit's beginning and end, in tiles
    double half;   // a tile of at most half the rows, in tiles (chunks, 0.6 -> 0.9: ragged ones 278 -> 258 us)
};

// node: a tree's tokens (null: a chain).
void add_units(std::vector<Unit> &units, const TokSeq &q, const TokNode *node, int hk, int group, int window, int sinks, const Shape &sh)
{
    const int64_t n_rows = (int64_t)q.n_new * group;
    for (int h = 0; h < hk; ++h)
        for (int64_t r0 = 0; r0 < n_rows; r0 += sh.rows) {
            Unit u{};
            TokItem &w = u.item;
            w.h = h; w.r0 = (int)r0; w.rows = (int)std::min<int64_t>(sh.rows, n_rows - r0);
            w.pos = q.pos; w.row0 = q.row0; w.table0 = q.table0;
            const int i0 = (int)(r0 / group), i1 = (int)((r0 + w.rows - 1) / group);
            int lo = q.pos + i0;
            if (node) {
                int depth = node[i0].depth;
                for (int i = i0 + 1; i <= i1; ++i) depth = std::min(depth, node[i].depth);
                lo = q.pos + depth;
            }
            const int end = std::min(q.kv, q.pos + i1 + 1);          // (an ancestor comes before its token)
            w.b1 = end;
            if (window > 0 && lo >= window) {
                w.b0 = std::min(node ? std::min(lo - window + 1, q.pos) : lo - window + 1, end);
                w.a1 = std::min(sinks, end);
                if (w.a1 >= w.b0 / sh.align * sh.align) w.a1 = w.b0 = 0;   // one run from the first cell on
            }
            const int from = w.b0 / sh.align * sh.align;
            u.tiles = (w.a1 + sh.tile - 1) / sh.tile + (w.b0 < end ? (end - from + sh.tile - 1) / sh.tile : 0);
            units.push_back(u);
        }
}

// A kernel's pieces, block by block.
struct Shares {
    std::vector<TokItem> items, cut;   // cut: the first part of every cut unit
    std::vector<int32_t> first;
    int parts = 0;
};

// Whole units, the longest first, each to the block with the least work, while they fit its share; the
// units that are left are cut to fill the blocks up.  Units of one sequence have about one length, so
// blocks that work at a time read the same cells (chunks of a batch whose cells exceed the L2 cache:
// 880 MB from device memory where shares were cut along the line).  A unit that is cut writes and
// reads its sums once more and starts twice, so few are: one that is little longer than a share and
// has a block to itself stays whole.
Shares pack(const std::vector<Unit> &units, const Shape &sh)
{
    Shares r;
    r.first.push_back(0);
    if (units.empty()) return r;
    constexpr double kWhole = 1.3;
    auto tile_cost = [&](const Unit &u) { return u.item.rows > sh.rows / 2 ? 1.0 : sh.half; };
    auto cost = [&](const Unit &u) { return u.tiles * tile_cost(u) + sh.start; };
    std::vector<int> order(units.size());
    std::iota(order.begin(), order.end(), 0);
    std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return cost(units[a]) > cost(units[b]); });
    double total = 0;
    for (const Unit &u : units) total += cost(u);
    int64_t most = 0;                                               // parts of the least size
    for (const Unit &u : units) most += std::max(1, u.tiles / sh.least);
    const int blocks = (int)std::min<int64_t>(sh.blocks, most);
    const double share = total / blocks * 1.02;
    using Load = std::pair<double, int>;                            // work so far, block
    std::priority_queue<Load, std::vector<Load>, std::greater<Load>> least;
    for (int b = 0; b < blocks; ++b) least.push({0.0, b});
    std::vector<std::vector<TokItem>> mine(blocks);
    std::vector<int> left;
    for (int i : order) {
        const Unit &u = units[i];
        const Load l = least.top();
        if (l.first + cost(u) > (l.first == 0 ? share * kWhole : share)) { left.push_back(i); continue; }
        least.pop();
        least.push({l.first + cost(u), l.second});
        TokItem w = u.item;
        w.t0 = 0; w.t1 = u.tiles; w.parts = 1;
        mine[l.second].push_back(w);
    }
    const double fill = share + sh.start;                             // (a part of a unit starts once more)
    for (int i : left) {
        const Unit &u = units[i];
        const int least_tiles = std::max(sh.least, (u.tiles + kMostParts - 1) / kMostParts);
        std::vector<std::pair<int, TokItem>> parts;
        for (int t = 0; t < u.tiles || (u.tiles == 0 && t == 0);) {
            const Load l = least.top();
            least.pop();
            int take = std::max((int)((fill - l.first - sh.start) / tile_cost(u)), least_tiles);
            if (u.tiles - t - take < sh.least) take = u.tiles - t;
            TokItem w = u.item;
            w.t0 = t; w.t1 = t + take;
            parts.push_back({l.second, w});
            least.push({l.first + take * tile_cost(u) + sh.start, l.second});
            t += std::max(take, 1);
        }
        for (size_t k = 0; k < parts.size(); ++k) {
            TokItem &w = parts[k].second;
            w.parts = (int)parts.size();
            if (parts.size() > 1) {
                w.part0 = r.parts; w.part = r.parts + (int)k; w.unit = (int)r.cut.size();
            }
            mine[parts[k].first].push_back(w);
        }
        if (parts.size() > 1) {
            r.parts += (int)parts.size();
            r.cut.push_back(parts[0].second);
        }
    }
    for (const auto &m : mine) {
        r.items.insert(r.items.end(), m.begin(), m.end());
        r.first.push_back((int32_t)r.items.size());
    }
    return r;
}

// A tree's tokens and their bits, or why its parents are none.
std::string add_tree(std::vector<TokNode> &nodes, std::vector<uint32_t> &bits, const int32_t *parents, int n, int pos, int window, int sinks)
{
    const int words = (n + 31) / 32;     // (65,535 trees of the most tokens: 2^31 words)
    const size_t node0 = nodes.size(), bit0 = bits.size();
    nodes.resize(node0 + n);
    bits.resize(bit0 + (size_t)n * words);
    TokNode *node = nodes.data() + node0;
    for (int i = 0; i < n; ++i) {
        const int p = parents[i];
        if (p < -1 || p >= i) return "new token " + std::to_string(i) + ": parent " + std::to_string(p) + " is not in -1.." + std::to_string(i - 1);
        uint32_t *mine = bits.data() + bit0 + (size_t)i * words;
        node[i] = {p < 0 ? 0 : node[p].depth + 1, pos, words, (uint32_t)(mine - bits.data())};
        if (window == 0) {
            if (p >= 0) std::copy(mine - (size_t)(i - p) * words, mine - (size_t)(i - p - 1) * words, mine);
            mine[i / 32] |= 1u << i % 32;
        } else {
            for (int a = i; a >= 0; a = parents[a])
                if (node[a].depth > node[i].depth - window || pos + node[a].depth < sinks) mine[a / 32] |= 1u << a % 32;
        }
    }
    return "";
}

// The packed device image of a plan's tables: parts at 16-byte boundaries of one host buffer.
struct Image {
    std::vector<char> bytes;
    template <class T>
    size_t add(const std::vector<T> &v)
    {
        const size_t at = (bytes.size() + 15) / 16 * 16;
        bytes.resize(at + std::max<size_t>(v.size() * sizeof(T), 16));
        if (!v.empty()) memcpy(bytes.data() + at, v.data(), v.size() * sizeof(T));
        return at;
    }
};

void set_plan(mure_tokens_plan *p, const mure_tokens_batch *bp, bool tree = false, const int32_t *parents = nullptr)
{
    mure_ctx *c = p->ctx;
    p->ready = false;
    FAILIF(!bp, c, MURE_ERR_INVALID_ARG, "NULL batch");
    const mure_tokens_batch &b = *bp;
    const mure_tokens_desc &d = p->d;
    FAILIF(b.reserved != 0, c, MURE_ERR_INVALID_ARG, "reserved fields must be 0");
    FAILIF(b.n_seqs < 0 || b.n_seqs > 65535, c, MURE_ERR_INVALID_ARG, "n_seqs %d not in 0..65535", b.n_seqs);
    FAILIF(b.n_heads < 1 || b.n_heads % d.n_kv_heads != 0, c, MURE_ERR_INVALID_ARG,
           "n_heads %d is not a positive multiple of n_kv_heads %d", b.n_heads, d.n_kv_heads);
    FAILIF(b.n_heads > 65536, c, MURE_ERR_UNSUPPORTED, "more than 65,536 query heads");
    FAILIF(b.n_seqs > 0 && (!b.new_len || !b.pos || !b.kv_len), c, MURE_ERR_INVALID_ARG, "NULL lengths");
    FAILIF(b.window < 0 || b.sinks < 0, c, MURE_ERR_INVALID_ARG, "negative window or sinks");
    FAILIF(b.window == 0 && b.sinks != 0, c, MURE_ERR_INVALID_ARG, "sinks without a window");
    // (of powers of two, as the kernels take it: its product with log2 e, too, has to be a number)
    const float scale_log2 = (float)((b.scale > 0.f ? (double)b.scale : 1.0 / std::sqrt((double)d.head_dim)) * 1.4426950408889634);
    FAILIF(!(b.scale >= 0.f) || !std::isfinite(scale_log2), c, MURE_ERR_INVALID_ARG, "scale must be in 0..2.3e38");

    const int page_log2 = log2_of(d.page_size), n = b.n_seqs;
    std::vector<TokSeq> seq(n);
    std::vector<int32_t> tile_new(n + 1, 0), tile_all(n + 1, 0), table;
    int64_t n_new = 0, n_cells = 0, t_new = 0, t_all = 0;
    struct Span {
        int64_t page;
        int first, last;   // slots
    };
    std::vector<Span> written;
    std::string fault;
    int past_end = -1;
    std::vector<TokNode> nodes;
    std::vector<uint32_t> bits;
    // (all of them before any list is read whose length they add up to)
    for (int s = 0; s < n; ++s)
        FAILIF(b.new_len[s] < 0 || b.pos[s] < 0 || b.kv_len[s] < 0, c, MURE_ERR_INVALID_ARG, "sequence %d: a negative length or position", s);
    for (int s = 0; s < n; ++s) {
        const int64_t nn = b.new_len[s], pos = b.pos[s], kv = b.kv_len[s];
        FAILIF(pos + nn > kMostPos || kv > kMostPos, c, MURE_ERR_INVALID_ARG, "sequence %d: positions past 2^30", s);
        const int64_t pages = (kv + d.page_size - 1) >> page_log2;
        FAILIF(pages > 0 && (!b.page_table || b.table_stride < pages), c, MURE_ERR_INVALID_ARG,
               "sequence %d: %lld pages, a table of %lld", s, (long long)pages, (long long)(b.page_table ? b.table_stride : 0));
        const int32_t *ids = b.page_table + (b.page_table ? s * b.table_stride : 0);
        for (int64_t i = 0; i < pages; ++i)
            FAILIF(ids[i] < 0 || ids[i] >= d.n_pages, c, MURE_ERR_INVALID_ARG, "sequence %d: page %d not in 0..%lld", s, ids[i],
                   (long long)d.n_pages - 1);
        seq[s] = {(int32_t)n_new, (int32_t)nn, (int32_t)pos, (int32_t)kv, (int64_t)table.size(), n_cells};
        table.insert(table.end(), ids, ids + pages);
        n_new += nn;
        n_cells += kv;
        t_new += (nn + kTokTile - 1) / kTokTile;
        t_all += (kv + kTokTile - 1) / kTokTile;
        FAILIF(n_new > INT32_MAX || t_all > INT32_MAX, c, MURE_ERR_UNSUPPORTED, "more than 2^31 - 1 new tokens or tiles of cells");
        tile_new[s + 1] = (int32_t)t_new;
        tile_all[s + 1] = (int32_t)t_all;
        if (tree && nn > 0) {
            FAILIF(!parents, c, MURE_ERR_INVALID_ARG, "NULL parents");
            FAILIF(nn > MURE_TREE_MAX, c, MURE_ERR_UNSUPPORTED, "sequence %d: a tree of %lld tokens, and %d are the most", s, (long long)nn,
                   (int)MURE_TREE_MAX);
            const std::string why = add_tree(nodes, bits, parents + seq[s].row0, (int)nn, (int)pos, b.window, b.sinks);
            FAILIF(!why.empty(), c, MURE_ERR_INVALID_ARG, "sequence %d: %s", s, why.c_str());
        }
        if (nn > 0 && pos + nn > kv) {
            if (past_end < 0) past_end = s;
            if (fault.empty())
                fault = "sequence " + std::to_string(s) + ": new tokens end at " + std::to_string(pos + nn) + ", past its " +
                        std::to_string(kv) + " cells";
            continue;
        }
        for (int64_t q = pos; q < pos + nn;) {
            const int64_t stop = std::min(pos + nn, ((q >> page_log2) + 1) << page_log2);
            const int first = (int)(q & (d.page_size - 1));
            written.push_back({ids[q >> page_log2], first, first + (int)(stop - q) - 1});
            q = stop;
        }
    }
    // two sequences may share a page that is written only where they write different cells of it
    std::sort(written.begin(), written.end(),
              [](const Span &x, const Span &y) { return x.page != y.page ? x.page < y.page : x.first < y.first; });
    for (size_t i = 1; i < written.size() && fault.empty(); ++i)
        if (written[i].page == written[i - 1].page && written[i].first <= written[i - 1].last)
            fault = "two new tokens have the cell " + std::to_string(written[i].first) + " of page " +
                    std::to_string(written[i].page);

    // attention: the pieces of the kernels that take this type
    const int group = b.n_heads / d.n_kv_heads;
    const bool wide = d.form == MURE_FORM_E4M3;
    const FewShape fshape = mure::few_shape(d.dtype, d.form, d.head_dim);
    const Shape few_shape{kFewRows, fshape.tile, 16, fshape.blocks, 2, 3.0, 1.0};
    const Shape chunk_shape{kChunkRows, kChunkTile, chunk_box(d.page_size), chunk_blocks(), 4, 4.0, 0.9};
    const Shape tree_shape{kTreeRows, kChunkTile, chunk_box(d.page_size), tree_blocks(), 2, 4.0, 0.9};
    std::vector<Unit> few, chunk, forest;
    std::vector<int32_t> wide_table, wide_pages;
    std::unordered_map<int32_t, int32_t> wide_of;
    std::vector<int> widen;                     // the sequences whose codes are wanted as 16-bit cells
    int64_t most_rows = 0;
    for (const TokSeq &q : seq) most_rows = std::max(most_rows, (int64_t)q.n_new * group);
    for (int s = 0; s < n; ++s) {
        const TokSeq &q = seq[s];
        const int64_t rows = (int64_t)q.n_new * group;
        FAILIF(rows > kMostPos, c, MURE_ERR_UNSUPPORTED, "sequence %d: more than 2^30 rows", s);
        // (a batch of trees on cells as they are goes to one kernel whole: 64 trees of 3 to 40 tokens within a window, of which 18
        // have few rows, 45 us in two launches one after the other, 41 in one; the kernel for few rows is little faster
        // on those even by itself, but on codes twice as fast.  One tree of more than kTreeRows rows takes the others along to the
        // two-tile kernel.  63 small ones alone, one of 134 rows over 2,000 cells alone, all in one plan, in two plans, us: 4 to 30 tokens, 32 heads on 8 of
        // 128 values, 154, 31, 170, 185; single tokens of these 150, 31, 168, 180; 3 to 40 tokens within a window, 15 heads
        // on 5 of 64, 43, 27, 55, 71; but single tokens of 8 heads on 8 of 64 84, 29, 127, 113)
        const int up_to = tree ? few_tree_rows_up_to(wide, d.head_dim) : few_rows_up_to(wide, d.head_dim);
        const bool as_chunk = d.dtype != MURE_F32 && d.head_dim <= kChunkDim && (tree && !wide ? most_rows : rows) > up_to;
        const bool as_tree = as_chunk && tree && !wide && most_rows <= kTreeRows;
        const Shape &sh = as_tree ? tree_shape : as_chunk ? chunk_shape : few_shape;
        FAILIF((int64_t)(few.size() + chunk.size() + forest.size()) + (rows + sh.rows - 1) / sh.rows * d.n_kv_heads > kMostUnits, c,
               MURE_ERR_UNSUPPORTED, "more than 2^24 pieces of work");
        add_units(as_tree ? forest : as_chunk ? chunk : few, q, tree ? nodes.data() + q.row0 : nullptr, d.n_kv_heads, group, b.window, b.sinks, sh);
        if (as_chunk && wide) widen.push_back(s);
    }
    // the pages that any of a sequence's rows reads, with where they are in the table; false from f: enough
    auto read_pages = [&](const TokSeq &q, auto f) {
        const int64_t end = std::min<int64_t>(q.kv, (int64_t)q.pos + q.n_new);
        const int64_t from = b.window > 0 ? std::max(0, q.pos - b.window + 1) : 0;
        for (int64_t i = 0; i << page_log2 < end; ++i) {
            if (((i + 1) << page_log2) <= from && i << page_log2 >= b.sinks) continue;
            if (!f(q.table0 + i, table[q.table0 + i])) return;
        }
    };
    // Trees on codes: their pieces widen the tiles that they read themselves, unless so many read the same ones that
    // widening the pages once costs less (48 trees of 48 tokens over 4,000 cells, as many on the same pages: 1 tree 282 us
    // against 418, 2 282 / 297, 3 282 / 260, 8 282 / 213).
    p->fused = false;
    if (tree && d.head_dim % 16 == 0 && !widen.empty()) {
        int64_t tiles = 0, most = 0, different = 0;
        for (const Unit &u : chunk) tiles += u.tiles;
        const int64_t page_cells = (int64_t)d.page_size * d.n_kv_heads, enough = (2 * tiles * kChunkTile + 5 * page_cells - 1) / (5 * page_cells);
        for (int s : widen) most += ((int64_t)seq[s].kv + d.page_size - 1) >> page_log2;
        IdSet ids(std::min<int64_t>(most, d.n_pages));
        for (int s : widen)
            if (different < enough) read_pages(seq[s], [&](int64_t, int32_t id) { return (different += ids.insert(id)) < enough; });
        p->fused = different >= enough;
    }
    if (!p->fused)
        for (int s : widen) {
            wide_table.resize(table.size(), 0);
            read_pages(seq[s], [&](int64_t at, int32_t id) {
                const auto known = wide_of.emplace(id, (int32_t)wide_pages.size());
                if (known.second) wide_pages.push_back(id);
                wide_table[at] = known.first->second;
                return true;
            });
        }
    const Shares fs = pack(few, few_shape), cs = pack(chunk, chunk_shape), ts = pack(forest, tree_shape);

    Image im;
    const size_t o_seq = im.add(seq), o_table = im.add(table), o_new = im.add(tile_new), o_all = im.add(tile_all);
    const size_t o_few = im.add(fs.items), o_few1 = im.add(fs.first), o_fewc = im.add(std::vector<int32_t>(fs.cut.size(), 0));
    const size_t o_chunk = im.add(cs.items), o_chunk1 = im.add(cs.first), o_cut = im.add(cs.cut);
    const size_t o_tree = im.add(ts.items), o_tree1 = im.add(ts.first), o_treec = im.add(ts.cut);
    const size_t o_wt = im.add(wide_table), o_wp = im.add(wide_pages), o_node = im.add(nodes), o_bits = im.add(bits);
    const size_t few_part = ((size_t)fs.parts * few_part_floats(d.head_dim) * 4 + 255) / 256 * 256;
    reserve(c, p->mem, p->mem_bytes, im.bytes.size());
    const size_t chunk_part = (size_t)cs.parts * chunk_part_floats(d.head_dim) * 4, chunk_again = (cs.items.size() * (kChunkRows / 8) + 255) / 256 * 256;
    const size_t tree_part = (size_t)ts.parts * tree_part_floats(d.head_dim) * 4;
    reserve(c, p->part, p->part_bytes, few_part + chunk_part + chunk_again + tree_part + ts.items.size() * (kTreeRows / 8));
    if (!wide_pages.empty()) {
        const int64_t pool = (int64_t)wide_pages.size() * d.n_kv_heads * d.page_size * d.head_dim * 2;
        reserve(c, p->wide, p->wide_bytes, 2 * (size_t)pool);
        FAILIF(!chunk_map(p->map_k, p->wide, d.dtype, d.n_kv_heads, d.head_dim, d.page_size, (int64_t)wide_pages.size()) ||
                   !chunk_map(p->map_v, static_cast<char *>(p->wide) + pool, d.dtype, d.n_kv_heads, d.head_dim, d.page_size,
                              (int64_t)wide_pages.size()),
               c, MURE_ERR_CUDA, "no tensor map of the widened pages");
    }
    upload(c, p->mem, im.bytes.data(), im.bytes.size());
    char *m = static_cast<char *>(p->mem);
    TokBatch &v = p->b;
    v.seq = reinterpret_cast<TokSeq *>(m + o_seq);
    v.table = reinterpret_cast<int32_t *>(m + o_table);
    v.tile_new = reinterpret_cast<int32_t *>(m + o_new);
    v.tile_all = reinterpret_cast<int32_t *>(m + o_all);
    p->few.items = reinterpret_cast<TokItem *>(m + o_few);
    p->few.first = reinterpret_cast<int32_t *>(m + o_few1);
    p->few.blocks = (int)fs.first.size() - 1;
    p->few.part = static_cast<float *>(p->part);
    p->few.count = reinterpret_cast<int32_t *>(m + o_fewc);
    char *part = static_cast<char *>(p->part) + few_part;
    auto set_chunk = [&](TokChunk &k, const Shares &s, size_t o_items, size_t o_first, size_t o_cut, int rows, int64_t floats) {
        k.w.items = reinterpret_cast<TokItem *>(m + o_items);
        k.w.first = reinterpret_cast<int32_t *>(m + o_first);
        k.w.blocks = (int)s.first.size() - 1;
        k.w.part = reinterpret_cast<float *>(part);
        k.w.again = reinterpret_cast<uint32_t *>(part + (size_t)s.parts * floats * 4);
        k.ml = k.w.part + (int64_t)s.parts * (floats - 2 * rows);
        k.cut = reinterpret_cast<TokItem *>(m + o_cut);
        k.n_cut = (int)s.cut.size();
    };
    set_chunk(p->chunk, cs, o_chunk, o_chunk1, o_cut, kChunkRows, chunk_part_floats(d.head_dim));
    part += chunk_part + chunk_again;
    set_chunk(p->tree, ts, o_tree, o_tree1, o_treec, kTreeRows, tree_part_floats(d.head_dim));
    p->wide_table = reinterpret_cast<int32_t *>(m + o_wt);
    p->wide_pages = reinterpret_cast<int32_t *>(m + o_wp);
    p->n_wide = (int64_t)wide_pages.size();
    v.node = tree ? reinterpret_cast<TokNode *>(m + o_node) : nullptr;
    v.bits = reinterpret_cast<uint32_t *>(m + o_bits);
    v.n_seqs = n;
    v.one_new = t_new == n;
    for (int s = 0; s < n && v.one_new; ++s) v.one_new = tile_new[s + 1] - tile_new[s] == 1;
    v.n_heads = b.n_heads;
    v.group = group;
    v.window = b.window;
    v.sinks = b.sinks;
    v.scale_log2 = scale_log2;
    p->n_new = n_new;
    p->n_cells = n_cells;
    p->tiles_new = t_new;
    p->tiles_all = t_all;
    p->new_past_end = past_end;
    p->append_fault = fault;
    p->seq = std::move(seq);
    p->ready = true;
}

mure_status create_plan(mure_tokens *t, const mure_tokens_batch *batch, bool tree, const int32_t *parents, mure_tokens_plan **out)
{
    if (!t) return MURE_ERR_INVALID_ARG;
    mure_ctx *c = t->ctx;
    return run(c, [&] {
        FAILIF(!out, c, MURE_ERR_INVALID_ARG, "NULL out");
        *out = nullptr;
        CK(c, cudaSetDevice(c->device));
        auto p = std::make_unique<mure_tokens_plan>();
        p->ctx = c;
        p->d = t->d;
        try {
            set_plan(p.get(), batch, tree, parents);
        } catch (...) {
            dfree(c, p->mem);
            dfree(c, p->part);
            dfree(c, p->wide);
            throw;
        }
        *out = p.release();
    });
}

mure_status reset_plan(mure_tokens_plan *p, const mure_tokens_batch *batch, bool tree, const int32_t *parents)
{
    if (!p) return MURE_ERR_INVALID_ARG;
    return run(p->ctx, [&] {
        p->ready = false;
        CK(p->ctx, cudaSetDevice(p->ctx->device));
        set_plan(p, batch, tree, parents);
    });
}

}  // namespace

extern "C" {

mure_status mure_tokens_create(mure_ctx *c, const mure_tokens_desc *desc, mure_tokens **out)
{
    if (!c) return MURE_ERR_INVALID_ARG;
    return run(c, [&] {
        FAILIF(!out, c, MURE_ERR_INVALID_ARG, "NULL out");
        *out = nullptr;
        FAILIF(!desc, c, MURE_ERR_INVALID_ARG, "NULL description");
        const mure_tokens_desc &d = *desc;
        check_geometry(c, d);
        const bool q = d.form == MURE_FORM_E4M3, any = d.k || d.v || d.k_scale || d.v_scale;
        FAILIF(any && (!d.k || !d.v || (q && (!d.k_scale || !d.v_scale))), c, MURE_ERR_INVALID_ARG,
               "some of the pools are NULL");
        FAILIF(!q && (d.k_scale || d.v_scale), c, MURE_ERR_INVALID_ARG, "scales without MURE_FORM_E4M3");
        FAILIF((uintptr_t)d.k % 16 || (uintptr_t)d.v % 16 || (uintptr_t)d.k_scale % 16 || (uintptr_t)d.v_scale % 16, c, MURE_ERR_INVALID_ARG, "pools are not 16-byte aligned");
        CK(c, cudaSetDevice(c->device));
        auto t = std::make_unique<mure_tokens>();
        t->ctx = c;
        t->d = d;
        if (!any) {
            const int64_t rows = d.n_pages * d.n_kv_heads * d.page_size;
            const int64_t pool = (rows * d.head_dim * (q ? 1 : elt_bytes(d.dtype)) + 255) / 256 * 256;
            const int64_t scales = q ? (rows + 255) / 256 * 256 : 0;
            char *m = static_cast<char *>(dalloc(c, 2 * (pool + scales)));
            t->own = m;
            t->d.k = m;
            t->d.v = m + pool;
            t->d.k_scale = q ? reinterpret_cast<uint8_t *>(m + 2 * pool) : nullptr;
            t->d.v_scale = q ? t->d.k_scale + scales : nullptr;
            const cudaError_t e = cudaMemsetAsync(m, 0, 2 * (pool + scales), c->stream);
            if (e != cudaSuccess) dfree(c, m);
            CK(c, e);
        }
        if (d.dtype != MURE_F32 && q && d.head_dim <= kChunkDim && d.head_dim % 16 == 0) {
            const bool ok = chunk_code_map(t->map_k, t->d.k, d.n_kv_heads, d.head_dim, d.page_size, d.n_pages) &&
                            chunk_code_map(t->map_v, t->d.v, d.n_kv_heads, d.head_dim, d.page_size, d.n_pages);
            if (!ok) dfree(c, t->own);
            FAILIF(!ok, c, MURE_ERR_CUDA, "no tensor map of the pools");
        }
        if (d.dtype != MURE_F32 && !q && d.head_dim <= kChunkDim) {
            const bool ok = chunk_map(t->map_k, t->d.k, d.dtype, d.n_kv_heads, d.head_dim, d.page_size, d.n_pages) &&
                            chunk_map(t->map_v, t->d.v, d.dtype, d.n_kv_heads, d.head_dim, d.page_size, d.n_pages);
            if (!ok) dfree(c, t->own);
            FAILIF(!ok, c, MURE_ERR_CUDA, "no tensor map of the pools");
        }
        *out = t.release();
    });
}

void mure_tokens_free(mure_tokens *t)
{
    if (!t) return;
    if (t->own) {
        cudaStreamSynchronize(t->ctx->stream);
        dfree(t->ctx, t->own);
    }
    delete t;
}

mure_status mure_tokens_buffers(const mure_tokens *t, mure_tokens_desc *out)
{
    if (!t || !out) return MURE_ERR_INVALID_ARG;
    *out = t->d;
    return MURE_OK;
}

mure_status mure_tokens_plan_create(mure_tokens *t, const mure_tokens_batch *batch, mure_tokens_plan **out)
{
    return create_plan(t, batch, false, nullptr, out);
}

mure_status mure_tokens_plan_create_tree(mure_tokens *t, const mure_tokens_batch *batch, const int32_t *parents, mure_tokens_plan **out)
{
    return create_plan(t, batch, true, parents, out);
}

mure_status mure_tokens_plan_set(mure_tokens_plan *p, const mure_tokens_batch *batch) { return reset_plan(p, batch, false, nullptr); }

mure_status mure_tokens_plan_set_tree(mure_tokens_plan *p, const mure_tokens_batch *batch, const int32_t *parents)
{
    return reset_plan(p, batch, true, parents);
}

void mure_tokens_plan_free(mure_tokens_plan *p)
{
    if (!p) return;
    dfree(p->ctx, p->mem);
    dfree(p->ctx, p->part);
    dfree(p->ctx, p->wide);
    delete p;
}

mure_status mure_tokens_append(mure_tokens *t, mure_tokens_plan *p, const mure_tokens_rows *k, const mure_tokens_rows *v)
{
    if (!t) return MURE_ERR_INVALID_ARG;
    mure_ctx *c = t->ctx;
    return run(c, [&] {
        check_pair(c, t, p);
        FAILIF(!p->append_fault.empty(), c, MURE_ERR_INVALID_ARG, "%s", p->append_fault.c_str());
        const TokRows kr = check_rows(c, k, t->d, p->n_new, t->d.n_kv_heads, "k");
        const TokRows vr = check_rows(c, v, t->d, p->n_new, t->d.n_kv_heads, "v");
        CK(c, cudaSetDevice(c->device));
        c->launches += launch_tokens_append(pool_of(t), p->b, t->d.dtype, t->d.form, kr, vr, p->tiles_new, c->stream);
        check_launch(c);
    });
}

mure_status mure_tokens_read(mure_tokens *t, mure_tokens_plan *p, int32_t part, const mure_tokens_rows *k,
                             const mure_tokens_rows *v)
{
    if (!t) return MURE_ERR_INVALID_ARG;
    mure_ctx *c = t->ctx;
    return run(c, [&] {
        check_pair(c, t, p);
        FAILIF(part != 0 && part != 1, c, MURE_ERR_INVALID_ARG, "part must be 0 or 1");
        // (the cells of new tokens past the cells held do not exist; shared ones may be read twice)
        FAILIF(part == 1 && p->new_past_end >= 0, c, MURE_ERR_INVALID_ARG, "sequence %d: new tokens end past its cells",
               p->new_past_end);
        const int64_t rows = part ? p->n_new : p->n_cells;
        const TokRows kr = check_rows(c, k, t->d, rows, t->d.n_kv_heads, "k");
        const TokRows vr = check_rows(c, v, t->d, rows, t->d.n_kv_heads, "v");
        check_apart(c, kr, t->d, rows, t->d.n_kv_heads, "k");
        check_apart(c, vr, t->d, rows, t->d.n_kv_heads, "v");
        CK(c, cudaSetDevice(c->device));
        c->launches += launch_tokens_read(pool_of(t), p->b, t->d.dtype, t->d.form, part, kr, vr,
                                          part ? p->tiles_new : p->tiles_all, c->stream);
        check_launch(c);
    });
}

mure_status mure_tokens_attend(mure_tokens *t, mure_tokens_plan *p, const mure_tokens_rows *q, const mure_tokens_rows *out,
                               float *lse)
{
    if (!t) return MURE_ERR_INVALID_ARG;
    mure_ctx *c = t->ctx;
    return run(c, [&] {
        check_pair(c, t, p);
        const TokRows qr = check_rows(c, q, t->d, p->n_new, p->b.n_heads, "q");
        const TokRows orow = check_rows(c, out, t->d, p->n_new, p->b.n_heads, "out");
        check_apart(c, orow, t->d, p->n_new, p->b.n_heads, "out");
        FAILIF((uintptr_t)lse % 4 != 0, c, MURE_ERR_INVALID_ARG, "lse is not aligned");
        CK(c, cudaSetDevice(c->device));
        const mure_tokens_desc &d = t->d;
        c->launches += launch_tokens_few(pool_of(t), p->b, p->few, d.dtype, d.form, qr, orow, lse, c->stream);
        c->launches += launch_tokens_tree(pool_of(t), p->b, p->tree, d.dtype, qr, orow, lse, d.n_pages, t->map_k, t->map_v, c->err_dev,
                                          c->wait_limit, c->stream);
        if (p->chunk.w.blocks > 0) {
            const TokPool codes = pool_of(t);
            TokPool pool = codes;
            TokBatch b = p->b;
            const bool codes_in = d.form == MURE_FORM_E4M3, wide = codes_in && !p->fused;
            if (wide) {
                const int64_t bytes = p->n_wide * d.n_kv_heads * d.page_size * d.head_dim * 2;
                pool.k = p->wide;
                pool.v = static_cast<char *>(p->wide) + bytes;
                b.table = p->wide_table;
                c->launches += launch_tokens_widen(codes, d.dtype, p->wide_pages, p->n_wide, pool.k, pool.v, c->stream);
            }
            c->launches += launch_tokens_chunk(pool, b, p->chunk, d.dtype, qr, orow, lse, wide ? p->n_wide : d.n_pages,
                                               wide ? p->map_k : t->map_k, wide ? p->map_v : t->map_v, codes_in ? &codes : nullptr,
                                               p->b.table, p->fused, c->err_dev, c->wait_limit, c->stream);
        }
        check_launch(c);
    });
}

mure_status mure_synchronize(mure_ctx *c)
{
    if (!c) return MURE_ERR_INVALID_ARG;
    return run(c, [&] {
        CK(c, cudaSetDevice(c->device));
        int dev_err = 0;
        CK(c, cudaMemcpyAsync(&dev_err, c->err_dev, sizeof(int), cudaMemcpyDeviceToHost, c->stream));
        CK(c, cudaStreamSynchronize(c->stream));
        if (dev_err) {
            CK(c, cudaMemsetAsync(c->err_dev, 0, sizeof(int), c->stream));
            FAILIF(true, c, dev_err == MURE_ERR_TIMEOUT ? MURE_ERR_TIMEOUT : MURE_ERR_UNSUPPORTED,
                   "a device-side check failed (code %d)", dev_err);
        }
    });
}

}  // extern "C"
