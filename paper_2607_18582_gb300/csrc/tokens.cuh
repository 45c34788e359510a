// Token caches: what the host lays out for a batch and the kernels read (not part of the ABI).
#pragma once

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
    const int32_t *tile_new = nullptr;       // [n_seqs + 1] tiles of kTokTileNew new tokens before a sequence's
    const int32_t *tile_all = nullptr;       // [n_seqs + 1] the same for kTokTileAll cells
    int n_seqs = 0;
    int n_heads = 0, group = 0;              // query heads; query heads per cached one
    int window = 0, sinks = 0;
    float scale_log2 = 0.f;                  // factor of the scores, times log2(e)
};

constexpr int kTokTileNew = 16, kTokTileAll = 64;

// Rows of activations (mure_tokens_rows); vec: every row starts on a 16-byte boundary.
struct TokRows {
    char *p = nullptr;
    int64_t ts = 0, hs = 0;
    int vec = 0;
};

int launch_tokens_append(const TokPool &pool, const TokBatch &b, int dtype, int form, TokRows k, TokRows v, int64_t tiles,
                         cudaStream_t s);
int launch_tokens_read(const TokPool &pool, const TokBatch &b, int dtype, int form, int part, TokRows k, TokRows v,
                       int64_t tiles, cudaStream_t s);
int launch_tokens_attend_rows(const TokPool &pool, const TokBatch &b, int dtype, int form, int64_t n_tokens, TokRows q,
                              TokRows out, float *lse, cudaStream_t s);

}  // namespace mure
