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
int launch_tokens_chunk(const TokPool &pool, const TokBatch &b, const TokChunk &c, int dtype, TokRows q, TokRows out, float *lse,
                        int64_t n_pages, const CUtensorMap &map_k, const CUtensorMap &map_v, const TokPool *codes,
                        const int32_t *code_table, int *err, int64_t spin, cudaStream_t s);
// E4M3 pages pages[0 .. n_list) as pages 0 .. n_list - 1 of 16-bit pools k and v, which launch_tokens_chunk takes
// together with where they come from (`codes`, `code_table`).  A value that f16 does not reach becomes a NaN:
// the rows that meet it are done from the codes.
int launch_tokens_widen(const TokPool &pool, int dtype, const int32_t *pages, int64_t n_list, void *k, void *v, cudaStream_t s);

int launch_tokens_append(const TokPool &pool, const TokBatch &b, int dtype, int form, TokRows k, TokRows v, int64_t tiles,
                         cudaStream_t s);
int launch_tokens_read(const TokPool &pool, const TokBatch &b, int dtype, int form, int part, TokRows k, TokRows v,
                       int64_t tiles, cudaStream_t s);

}  // namespace mure
