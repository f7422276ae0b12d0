// Internal declarations of attention over shared prefixes.
#pragma once
#include <stdint.h>

#include <vector>

#include "ppd_ops.h"

namespace ppd {

constexpr int kSharedStep = kTileTokens;  // sharing is used in steps of this many tokens: the key ranges of row blocks begin at multiples of it
constexpr int kMaxNested = 16;            // shared ranges one behind the other, at most, that a sequence is part of
constexpr int kPrefixCols = 128;          // query columns of a prefix tile at most: 32 for each of its four waves
constexpr int kMaxPrefixChunk = kMaxTreeChunk;  // keys of one at most (its page ids are staged in LDS)

// A tile: `ncols` query columns (row-major over the G heads of a group) of consecutive rows against keys [kv_begin, kv_end), which are read
// by the page table of sequence `seq`.  Row j sees the keys up to L + j (a shared range: all, its L is its end).
struct PrefixItem {
    int32_t seq, kvh;
    int32_t grow0, ncols;
    int32_t L, kv_total;
    int32_t kv_begin, kv_end;
    int64_t part_off;          // floats, of this tile's partial; -1 where the tile has all keys of its rows and writes `out`
};

// Waves of a tile that have the same columns, each with every waves-th slab of the keys.
constexpr int prefix_key_waves(int ncols) { return ncols <= 32 ? 4 : ncols <= 64 ? 2 : 1; }

// Partials of some columns: `nsplit` of ncols * D floats, the sums, then [ncols] (m, l) pairs, one behind the other, and behind these the next
// KV head's.  The sums are [ncols][D], or, of a tile whose waves have columns of their own, [4 columns][D / 4][column][4], fewer in the last.
struct JoinSource {
    int64_t part_off;
    int32_t ncols, col0;       // col0: where the unit's first column is among them
    int32_t nsplit, by_rows;
};

// Rows whose columns have the same sources: those from the unit's number times `source_stride` on, so that unit and sources are asked for at
// once.
struct JoinUnit {
    int32_t grow0, nrows;
    int32_t nsources, unused;
};

// Neighbouring sequences that are planned together, and run before the next ones: where its lists begin in the plan's, and how long they are.
struct PrefixPart {
    int64_t item0, block0, unit0, source0;
    int32_t n_items, n_blocks, n_units;
    int32_t join_cols, source_stride;
};

struct PrefixPlan {
    std::vector<PrefixItem> items;
    std::vector<ppd_work_item> blocks;     // row blocks: columns beyond kPrefixCols
    std::vector<JoinUnit> units;
    std::vector<JoinSource> sources;
    std::vector<PrefixPart> parts;         // of build_prefix_parts
    int64_t partial_floats = 0;            // of the part that has most
    int32_t join_cols = 0;                 // most columns of a unit
    int32_t source_stride = 0;             // most sources of one
    int64_t keys_read = 0, keys_alone = 0; // keys per KV head that tiles are over, and without sharing
};

// Builds the tile list of a prefix attention call, whose arguments the caller has checked (shared[i] of sequence i > 0: tokens it has in
// common with the one before, at most what either has cached); false if it has more than kMaxTiles tiles.
bool build_prefix_plan(const ppd_shape& s, const int32_t* shared, const int32_t* L, const int32_t* n, int32_t B, int kv_elem_bytes, int num_cus, PrefixPlan* plan);

// The same of a batch whose partials may not take more than `most_floats`: sequences that need more are halved until they do not, or there is one
// left (which then takes what it takes).  The parts run one after the other in the same workspace.
constexpr int64_t kMostPartialFloats = int64_t(1) << 28;
constexpr int64_t kFewestPartialFloats = int64_t(1) << 22;  // as little as is tried where memory is short
bool build_prefix_parts(const ppd_shape& s, const int32_t* shared, const int32_t* L, const int32_t* n, int32_t B, int kv_elem_bytes, int num_cus, int64_t most_floats,
                        PrefixPlan* plan);

struct PrefixParams {
    const uint16_t* q;
    uint16_t* out;
    const void* pool;
    const int32_t* page_tables;
    const PrefixItem* items;
    const JoinUnit* units;
    const JoinSource* sources;
    float* partials;
    uint32_t* err_flags;
    int64_t num_pages;
    int64_t page_stride;       // elements
    int32_t max_pages;
    int32_t Hq, Hkv, G, invG;  // invG = 65536 / G + 1: col / G == (col * invG) >> 16
    int32_t n_items, n_units;
    int32_t join_cols, source_stride;
    float scale_log2e;         // softmax scale * log2(e), times the K scale of FP8 pages
    float v_scale;
};

// Launchers; stream is a hipStream_t, the result a hipError_t.
int launch_prefix(const PrefixParams& p, int head_dim, bool fp8_pages, void* stream);
int launch_prefix_join(const PrefixParams& p, int head_dim, void* stream);

}  // namespace ppd
