// Token caches: what the host lays out for a batch and the kernels read (not part of the ABI).
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace mure {

// One sequence of a batch.
struct TokSeq {
    int32_t row0;    // its first new token among the batch's packed ones
    int32_t n_new;
    int32_t pos;     // position of the first new token
    int32_t kv;      // cells held
    int64_t table0;  // its first page in the table
    int64_t cell0;   // cells of the sequences before it
};

// A cache's pools: cell (page, head h, slot) starts at ((page * hk + h) << page_log2 | slot) * d.
struct TokPool {
    void *k = nullptr, *v = nullptr;
    uint8_t *ks = nullptr, *vs = nullptr;   // E4M3: a scale byte per row
    int hk = 0, d = 0, page_log2 = 0;
};

// A new token of a tree: its cells before the sequence's new ones are seen by its position, as in any batch; of the new
// ones' those whose bit is set (itself and its ancestors, as far as a window holds them).
struct TokNode {
    int32_t depth;   // its position is the sequence's first new one's and this
    int32_t first;   // the cell of the sequence's first new token
    int32_t words;   // 32-bit words of bits
    uint32_t at;     // the first one
};

// A batch on the device.
struct TokBatch {
    const TokSeq *seq = nullptr;
    const int32_t *table = nullptr;          // the sequences' pages, one after the other
    const int32_t *tile_new = nullptr;       // [n_seqs + 1] tiles of kTokTile new tokens before a sequence's
    const int32_t *tile_all = nullptr;       // [n_seqs + 1] the same for its cells
    int n_seqs = 0;
    int one_new = 0;                         // every sequence has one tile of new tokens
    int n_heads = 0, group = 0;              // query heads; query heads per cached one
    int window = 0, sinks = 0;
    float scale_log2 = 0.f;                  // factor of the scores, times log2(e)
    const TokNode *node = nullptr;           // trees: a new token each (null: new tokens follow one another)
    const uint32_t *bits = nullptr;
};

constexpr int kTokTile = 16;

// Rows of activations (mure_tokens_rows); vec: every row starts on a 16-byte boundary.
struct TokRows {
    char *p = nullptr;
    int64_t ts = 0, hs = 0;
    int vec = 0;
};

// A piece of an attention call's work: rows r0 .. r0 + rows of one sequence and cached head (row r is
// new token r / group, query head h * group + r % group) over the tiles t0 .. t1 - 1 of the cells
// that any of them may attend to: first those of a0 .. a1 - 1 (the sinks, where they lie
// apart), then those of b0 .. b1 - 1, tiles from b0 rounded down to the kernel's alignment.
struct TokItem {
    int32_t h, r0, rows;
    int32_t pos, row0;                // of the sequence's first new token
    int32_t a1, b0, b1;               // (a0 is 0)
    int32_t t0, t1;
    int32_t part, part0, parts;       // parts > 1: partial result `part` of part0 .. part0 + parts - 1
    int32_t unit;                     // parts > 1: the counter of the rows' finished parts
    int64_t table0;
};

// The pieces, block by block, and room for partial results.
struct TokWork {
    const TokItem *items = nullptr;
    const int32_t *first = nullptr;   // [blocks + 1] a block's first item
    int blocks = 0;
    float *part = nullptr;            // [parts][rows of a piece][padded d + 2]: sums, maximum, sum of powers
    int32_t *count = nullptr;         // [units], zero between calls
    uint32_t *again = nullptr;        // chunks: [items][kChunkRows / 32] a bit per row that is done again
};

// Rows of a piece and cells of a tile of the kernel for few rows.
constexpr int kFewRows = 16;
constexpr int kMostParts = 512;       // of a unit
struct FewShape {
    int tile, blocks;                 // cells of a tile; blocks that run at a time
};
FewShape few_shape(int dtype, int form, int d);
int few_part_floats(int d);
int launch_tokens_few(const TokPool &pool, const TokBatch &b, const TokWork &w, int dtype, int form, TokRows q, TokRows out,
                      float *lse, cudaStream_t s);

// Pieces of the kernel for chunks: up to 256 rows over tiles of 128 cells.
constexpr int kChunkRows = 256, kChunkTile = 128, kChunkDim = 128;
struct TokChunk {
    TokWork w;
    float *ml = nullptr;              // partial results' maxima and sums
    const TokItem *cut = nullptr;     // [n_cut] the first part of every cut unit
    int n_cut = 0;
};
int chunk_blocks();
int chunk_box(int page_size);         // cells of a box its copies take (and its tiles' alignment)
int64_t chunk_part_floats(int d);
bool chunk_map(CUtensorMap &map, void *pool, int dtype, int hk, int d, int page_size, int64_t n_pages);
// The map of a pool of codes, d a multiple of 16: with it (fused) a tree's pieces widen the codes themselves.
bool chunk_code_map(CUtensorMap &map, void *pool, int hk, int d, int page_size, int64_t n_pages);
int launch_tokens_chunk(const TokPool &pool, const TokBatch &b, const TokChunk &c, int dtype, TokRows q, TokRows out, float *lse,
                        int64_t n_pages, const CUtensorMap &map_k, const CUtensorMap &map_v, const TokPool *codes,
                        const int32_t *code_table, bool fused, int *err, int64_t spin, cudaStream_t s);
// The parts of c's cut units, `of` rows each, joined (early: their kernel lets dependent launches begin).
int launch_tokens_join(const TokChunk &c, int of, const TokBatch &b, int dtype, int d, TokRows out, float *lse, bool early, cudaStream_t s);

// Pieces of the kernel for trees: up to 128 rows over tiles of 128 cells, two blocks on a multiprocessor.
constexpr int kTreeRows = 128;
int tree_blocks();
int64_t tree_part_floats(int d);
int launch_tokens_tree(const TokPool &pool, const TokBatch &b, const TokChunk &c, int dtype, TokRows q, TokRows out, float *lse,
                       int64_t n_pages, const CUtensorMap &map_k, const CUtensorMap &map_v, int *err, int64_t spin, cudaStream_t s);

// E4M3 pages pages[0 .. n_list) as pages 0 .. n_list - 1 of 16-bit pools k and v, which launch_tokens_chunk takes
// together with where they come from (`codes`, `code_table`).  A value that f16 does not reach becomes a NaN:
// the rows that meet it are done from the codes.
int launch_tokens_widen(const TokPool &pool, int dtype, const int32_t *pages, int64_t n_list, void *k, void *v, cudaStream_t s);

// Norm and rotation of the new tokens' queries and keys.
struct TokRotary {
    const uint64_t *turn = nullptr;      // [rot / 2] a pair's turns per position, times 2^64, modulo 2^64
    const float *weight = nullptr;       // [2][d] of the queries' norm and the keys'
    const uint8_t *axis = nullptr;       // [rot / 2] the pair's axis of positions
    int rot = 0, adjacent = 0;
    int norm_q = 0, norm_k = 0;
    float eps = 0.f;
    const int32_t *positions = nullptr;  // [axes][position_stride] (null: the batch's, along every axis)
    int64_t position_stride = 0;
};
// cells: k and v go into their cells (form as given); else k's rows to k_out, and v is not used.
int launch_tokens_rotate(const TokPool &pool, const TokBatch &b, const TokRotary &r, int dtype, int form, bool cells, int q_heads,
                         int k_heads, TokRows q, TokRows k, TokRows v, TokRows q_out, TokRows k_out, int64_t tokens, int64_t tiles,
                         cudaStream_t s);

// Pages pages[2 i] of one cache to pages[2 i + 1] of another of its geometry (host array, n pairs).
int launch_tokens_copy_pages(const TokPool &from, const TokPool &to, int elt, bool scales, const int32_t *pages, int64_t n, cudaStream_t s);
// New tokens' cells moved up: of sequence seq[i] (host arrays), the cells of the new tokens index[first[i] ..
// end[i] - 1], ascending, to those of its new tokens to[i], to[i] + 1, ...
int launch_tokens_keep(const TokPool &pool, const TokBatch &b, int elt, bool scales, const int32_t *seq, const int32_t *first,
                       const int32_t *end, const int32_t *to, const int32_t *index, int64_t n, cudaStream_t s);

int launch_tokens_append(const TokPool &pool, const TokBatch &b, int dtype, int form, TokRows k, TokRows v, int64_t tiles,
                         cudaStream_t s);
int launch_tokens_read(const TokPool &pool, const TokBatch &b, int dtype, int form, int part, TokRows k, TokRows v,
                       int64_t tiles, cudaStream_t s);

}  // namespace mure
