// Internal declarations of the drafting and eviction operators: tree and weighted attention over the pages, the choice of
// the tokens to keep, and their move to the front.
#pragma once
#include <stdint.h>

#include <vector>

#include "ppd_internal.h"

namespace ppd {

constexpr int kTreeCols = 32;        // query columns of a tree tile: one matrix-instruction block
constexpr int kTreeWaves = 4;        // waves of a tree tile's workgroup, each with every fourth slab of the keys
constexpr int kTreeThreads = 64 * kTreeWaves;
constexpr int kSlab = 32;            // keys a wave works at a time: two pages
constexpr int kTreeStep = kSlab * kTreeWaves;  // split boundaries are multiples of it
constexpr int kMaxTreeChunk = 8192;  // keys per tree tile at most (its page ids are staged in LDS)
constexpr int kMaxTreeBlockChunk = 16384;  // the same of a row block
constexpr int32_t kMaxTreeTokens = INT32_MAX - kMaxTreeBlockChunk;  // of a sequence: rounded up to whole tiles its keys are numbered in 32 bits
constexpr int kMaxMaskWords = 16;    // 64-bit words of a row's tree mask at most
constexpr int kKeptScores = 19200;  // scores that a tree tile holds in LDS: two workgroups' fill a unit
constexpr int kWeighKeys = 256;      // keys of a workgroup that adds up attention weights
constexpr int kSelectBatch = 512;    // sequences per launch of the select kernel (their lengths are kernel arguments)
constexpr int kSelectChunk = 16384;  // weights that a workgroup of the select kernels holds in registers
constexpr int kSelectBins = 2048;    // of the chunks' histograms
constexpr int kSelectRowWords = 4;   // of a row's counts, in front of its chunks'
constexpr int kCompactBatch = 256;   // the same for the move (two lists)

// A tile of tree attention: all `ncols` query columns of one sequence and KV head (row-major over the G heads of the group), at most
// kTreeCols, against keys [kv_begin, kv_end).
struct TreeItem {
    int32_t seq, kvh;
    int32_t grow0;             // the sequence's first row in q, out and the masks
    int32_t ncols;
    int32_t L, kv_total;
    int32_t kv_begin, kv_end;
    int64_t part_off;          // floats, of this tile's partial; -1 where the tile has all keys and writes `out`
    int64_t score_off;         // floats, where the scores of the sequence and head go; -1: they are not kept
};

// Columns whose key range was split over nsplit tiles with consecutive partials ([ncols][D] sums, then [ncols] (m, l) pairs).
struct TreeGroup {
    int32_t kvh;
    int32_t grow0;             // of the sequence
    int32_t col0, ncols;
    int32_t nsplit, unused;
    int64_t part_off, part_stride;
};

// Keys [kv_begin, min(kv_begin + kWeighKeys, kv_total)) of one sequence and KV head, whose weights are added up over all its columns.
struct WeighItem {
    int32_t seq, kvh, grow0, cols;
    int32_t L, kv_total, kv_begin;
    int32_t group;             // of kept scores, where the range was split; or -1
    int64_t score_off;         // floats: scores [slab][column][32 keys], or -1: they are computed again
};

// Keys of kept scores: whole slabs, whose every key is written.
constexpr int32_t score_keys(int32_t kv_total) { return (kv_total + kSlab - 1) / kSlab * kSlab; }

struct TreePlan {
    std::vector<TreeItem> items;           // tiles of sequences with at most kTreeCols query columns
    std::vector<ppd_work_item> blocks;     // row blocks of the others
    std::vector<TreeGroup> groups;
    std::vector<WeighItem> weighs, score_weighs;  // from K, from kept scores
    int64_t partial_floats = 0, score_floats = 0;
    int32_t rows = 0, join_cols = 0;
};

// Builds the tile list of a tree or weighted attention call, whose lengths the caller has checked; false if it has more than kMaxTiles tiles.
bool build_tree_plan(const ppd_shape& s, const int32_t* L, const int32_t* n, int32_t B, bool weighted, int kv_elem_bytes, int num_cus, TreePlan* plan);

struct TreeParams {
    const uint16_t* q;
    uint16_t* out;
    const void* pool;
    const int32_t* page_tables;
    const uint64_t* mask;      // [rows][mask_words], or NULL: row j sees the new tokens up to itself
    const TreeItem* items;
    const TreeGroup* groups;
    const WeighItem *weighs, *score_weighs;
    float* partials;
    float* scores;
    float* stats;              // weighted attention: per row and query head the softmax reference and one over the sum
    float* weights;            // [B][Hkv][weight_stride]
    int64_t weight_stride;
    uint32_t* err_flags;
    int64_t num_pages;
    int64_t page_stride;       // elements
    int32_t mask_words;
    int32_t max_pages;
    int32_t Hq, Hkv, G;
    int32_t n_items, n_groups, n_weighs, n_score_weighs;
    int32_t join_cols;         // most columns of a group
    float scale_log2e;         // softmax scale * log2(e), times the K scale of FP8 pages
    float v_scale;
};

// Arguments of the row-block kernel: those of the mixed kernel, and what a tree adds.
struct TreeBlockParams : KParams {
    const uint64_t* mask;
    float* stats;
    int32_t mask_words;
};

struct SelectParams {
    const float* weights;
    int32_t* keep;
    int64_t weight_stride, keep_stride;
    int32_t Hkv, budget, sinks, recent;
    int32_t B;
    // rows longer than kSelectChunk: chunks of the longest (0: none is longer), every chunk's histogram, every row's candidates (key and
    // chunk) and counts
    int32_t max_chunks;
    uint32_t *hist, *candidates;
    int32_t* counts;
    int32_t length[kSelectBatch];
};

struct CompactParams {
    void* pool;
    const int32_t* page_tables;
    const int32_t* keep;
    float* weights;            // or NULL
    uint32_t* err_flags;
    int64_t keep_layer, keep_seq, keep_head;  // element strides of the lists
    int64_t weight_layer, weight_stride;
    int64_t pool_layer;        // elements
    int64_t num_pages, page_stride;
    int32_t max_pages, Hkv, B;
    int32_t step;              // positions of a head that a workgroup takes at a time: 16, 32, 64 or 128
    int32_t first[kCompactBatch], count[kCompactBatch];
};

// Launchers; stream is a hipStream_t, the result a hipError_t.
int launch_tree(const TreeParams& p, int head_dim, bool fp8_pages, void* stream);
int launch_tree_blocks(const TreeBlockParams& p, int head_dim, bool fp8_pages, void* stream);
int launch_tree_join(const TreeParams& p, int head_dim, void* stream);
int launch_weigh(const TreeParams& p, int head_dim, bool fp8_pages, void* stream);
int launch_select(const SelectParams& p, int longest, void* stream);
int launch_compact(const CompactParams& p, int head_dim, bool fp8_pages, int layers, void* stream);

}  // namespace ppd
