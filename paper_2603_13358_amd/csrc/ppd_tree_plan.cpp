// Tile list of tree and weighted attention: which columns of which sequence meet which keys in which workgroup.
#include <algorithm>
#include <functional>

#include "ppd_ops.h"

namespace ppd {

namespace {

// What a kind of tile costs, in keys' time: `start_keys` is its start and end, `join_keys` the launch that joins partials and
// `column_keys` a column of a partial, written and read again.  `slots` tiles are resident.
struct TileKind {
    int32_t max_chunk, step;
    double start_keys, join_keys, column_keys;
    int32_t slots;
};

// A sequence's key range: `tiles` tiles of `cols` query columns each have it, for every KV head.
struct KeyRange {
    int32_t keys, tiles, cols;
};

// Rounded up; the sum may pass 32 bits.
int32_t ceil_div(int64_t a, int64_t b) { return (int32_t)((a + b - 1) / b); }

}  // namespace

double last_tile_end(std::vector<double>& tiles, int32_t slots) {
    std::sort(tiles.begin(), tiles.end(), std::greater<double>());
    std::vector<double> ends;  // heap, the earliest on top
    for (double t : tiles) {
        if ((int32_t)ends.size() < slots) {
            ends.push_back(t);
            if ((int32_t)ends.size() == slots) std::make_heap(ends.begin(), ends.end(), std::greater<double>());
            continue;
        }
        std::pop_heap(ends.begin(), ends.end(), std::greater<double>());
        ends.back() += t;
        std::push_heap(ends.begin(), ends.end(), std::greater<double>());
    }
    return *std::max_element(ends.begin(), ends.end());
}

namespace {

// Keys per tile, about: every sequence's range is cut evenly into as many tiles as this needs.  Fewer tiles start less often and leave
// fewer partials, more fill the slots more evenly.  Up to four rounds the tiles are laid out to see how long they take; many short
// ones last about their even share and half of the longest.
int32_t choose_chunk(const TileKind& kind, const std::vector<KeyRange>& ranges, int32_t heads) {
    int32_t longest = 1;
    for (const auto& r : ranges) longest = std::max(longest, r.keys);
    const int32_t slots = std::max(1, kind.slots / heads);
    int32_t chunk = kind.max_chunk;
    double best = -1;
    std::vector<double> tiles;
    for (double c = std::min<double>(kind.max_chunk, longest); c >= kind.step; c *= 0.84) {
        double count = 0, sum = 0, most = 0, joined = 0;
        for (const auto& r : ranges) {
            const double pieces = (double)ceil_div(r.keys, (int64_t)c);
            const double cost = r.keys / pieces + kind.start_keys;
            count += pieces * r.tiles;
            sum += pieces * r.tiles * cost;
            most = std::max(most, cost);
            if (pieces > 1) joined += pieces * r.tiles * r.cols;
        }
        if (count * heads > kMaxTiles) break;
        double est = count <= slots ? most : sum / slots + 0.5 * most;
        if (count > slots && count <= 4.0 * slots) {
            tiles.clear();
            for (const auto& r : ranges) {
                const int64_t pieces = ceil_div(r.keys, (int64_t)c);
                tiles.insert(tiles.end(), (size_t)(pieces * r.tiles), (double)r.keys / pieces + kind.start_keys);
            }
            est = last_tile_end(tiles, slots);
        }
        if (joined > 0) est += kind.join_keys + kind.column_keys * joined * heads;
        if (best < 0 || est < best) {
            best = est;
            chunk = (int32_t)c;
        }
        if (count > 16.0 * slots) break;
    }
    return chunk;
}

}  // namespace

bool build_tree_plan(const ppd_shape& s, const int32_t* L, const int32_t* n, int32_t B, bool weighted, int kv_elem_bytes, int num_cus, TreePlan* plan) {
    const int G = s.num_q_heads / s.num_kv_heads, Hkv = s.num_kv_heads, D = s.head_dim;
    plan->items.clear();
    plan->blocks.clear();
    plan->groups.clear();
    plan->weighs.clear();
    plan->score_weighs.clear();
    plan->score_floats = 0;
    plan->partial_floats = 0;
    plan->join_cols = 0;
    // Measured on weighted and tree calls of 1, 6, 24 and 64 sequences (4 and 24 columns; D = 128 on bf16 and FP8 pages, D = 64): starts of 64 or
    // 128 keys take up to 17 % longer (64 trees, D = 64: 24.4 -> 28.7 us), 512 and 1024 the same but for 24 trees at D = 128, which gain (63 ->
    // 55.5 us, FP8 43 -> 35), as they do with columns of 0.02; joins of 64 to 2048 keys make no difference.
    const TileKind narrow = {kMaxTreeChunk, kTreeStep, 256, 256, 0, 2 * num_cus};
    // Measured over batches of 4, 6 and 32 sequences cut into 512 to 8192 keys (D = 128): a row block takes 6.6 us and 1.2 us per 64
    // keys, a split launch 9.5 us more and 0.2 us per 1000 columns of partials.  On FP8 pages and at D = 64, where a step takes another
    // time, the same numbers serve: over 2, 6 and 32 sequences, 5 and 8 query heads to a KV head, starts of 200 to 500 keys and joins
    // of 250 to 1000 are within 2 %; a start of 700 costs 5-8 % on FP8 pages, twice the column 4-12 % at D = 128 (and gains up to 7 % for
    // two sequences at D = 64), half of it up to 9 % at D = 64.
    const TileKind wide = {kMaxTreeBlockChunk, kTileTokens, 350, 500, 0.0114, num_cus};
    const int block_rows = kMfmaCols / G;
    // Scores are kept where writing and reading them (8 bytes a column and key) moves no more than reading K again.  Kept against computed
    // again, us, decodes of 1, 8 and 64 sequences of 4K, 8K-16K and 1K-8K keys, 8 KV heads:
    //   D = 128, bf16   8 columns 13.4 72 175 / 19 94 222    16: 14.3 81 198 / 20 94 226    32 (the last kept): 16.4 100 250 / 21 97 236
    //   D = 128, FP8    8 columns 13.5 43 101 / 19 62 134    16 (the last kept): 14.3 54 123 / 20 62 136    32: 16.4 74 177 / 21 65 141
    //   D = 64, bf16    8 columns 11.3 43 97 / 16 54 123     16 (the last kept): 11.9 54 118 / 17 54 124    32: 13.3 67 158 / 18 56 127
    //   D = 64, FP8     8 columns (the last kept): 11.8 30 64 / 17 40 82     16: 12.3 42 87 / 17 40 83
    // One sequence gains by them at any width, batches up to half of the rule's edge at least; at the edge on bf16 pages of D = 128 batches
    // lose 3-6 %.
    auto keeps_scores = [&](int32_t rows) { return weighted && (int64_t)rows * G <= kTreeCols && (int64_t)rows * G * 8 <= (int64_t)D * kv_elem_bytes; };
    auto max_piece = [&](int32_t rows) {
        if ((int64_t)rows * G > kTreeCols) return wide.max_chunk;
        return keeps_scores(rows) ? std::min(narrow.max_chunk, kKeptScores / (rows * G) / narrow.step * narrow.step) : narrow.max_chunk;
    };
    double fewest = 0;
    std::vector<KeyRange> narrow_ranges, wide_ranges;
    for (int i = 0; i < B; ++i) {
        const bool is_wide = (int64_t)n[i] * G > kTreeCols;
        const int32_t blocks = is_wide ? ceil_div(n[i], block_rows) : 1;
        (is_wide ? wide_ranges : narrow_ranges).push_back({L[i] + n[i], blocks, is_wide ? ceil_div(n[i], blocks) * G : n[i] * G});
        fewest += (double)blocks * Hkv * (((double)L[i] + n[i]) / std::min(kMaxTreeChunk, max_piece(n[i])) + 1);
    }
    if (fewest > kMaxTiles) return false;
    const int32_t narrow_chunk = narrow_ranges.empty() ? 0 : choose_chunk(narrow, narrow_ranges, Hkv);
    const int32_t wide_chunk = wide_ranges.empty() ? 0 : choose_chunk(wide, wide_ranges, Hkv);
    int32_t grow0 = 0;
    for (int i = 0; i < B; ++i) {
        const int32_t total = L[i] + n[i];
        const bool is_wide = (int64_t)n[i] * G > kTreeCols;
        const TileKind& kind = is_wide ? wide : narrow;
        const bool keep_scores = keeps_scores(n[i]);
        const int32_t most = max_piece(n[i]);
        const int32_t chunk = std::min(most, is_wide ? wide_chunk : narrow_chunk);
        const int32_t pieces = ceil_div(total, chunk);
        const int32_t piece = std::min(most, ceil_div(ceil_div(total, pieces), kind.step) * kind.step);
        const int32_t nsplit = ceil_div(total, piece);
        const int32_t blocks = is_wide ? ceil_div(n[i], block_rows) : 1, rows = ceil_div(n[i], blocks);
        for (int h = 0; h < Hkv; ++h) {
            for (int32_t row0 = 0; row0 < n[i]; row0 += rows) {
                const int32_t nrows = std::min(rows, n[i] - row0), cols = nrows * G;
                const int64_t stride = (int64_t)cols * (D + 2);
                if (nsplit > 1) {
                    plan->groups.push_back({h, grow0, row0 * G, cols, nsplit, 0, plan->partial_floats, stride});
                    plan->join_cols = std::max(plan->join_cols, cols);
                }
                for (int32_t p = 0; p < nsplit; ++p) {
                    const int32_t begin = p * piece, end = std::min(total, (p + 1) * piece);
                    const int64_t part = nsplit > 1 ? plan->partial_floats + p * stride : -1;
                    if (is_wide) {
                        ppd_work_item it{};
                        it.kind = 1;
                        it.seq = i;
                        it.kvh = h;
                        it.row0 = row0;
                        it.nrows = nrows;
                        it.grow0 = grow0 + row0;
                        it.L = L[i];
                        it.kv_total = total;
                        it.kv_begin = begin;
                        it.kv_end = end;
                        it.group = nsplit > 1 ? (int32_t)plan->groups.size() - 1 : -1;
                        it.part_off = part;
                        plan->blocks.push_back(it);
                    } else {
                        plan->items.push_back({i, h, grow0, cols, L[i], total, begin, end, part, keep_scores ? plan->score_floats : -1});
                    }
                }
                if (nsplit > 1) plan->partial_floats += stride * nsplit;
            }
            if (weighted) {
                std::vector<WeighItem>& list = keep_scores ? plan->score_weighs : plan->weighs;
                for (int32_t t = 0; t < total; t += kWeighKeys) list.push_back({i, h, grow0, n[i] * G, L[i], total, t, keep_scores && nsplit > 1 ? (int32_t)plan->groups.size() - 1 : -1, keep_scores ? plan->score_floats : -1});
                if (keep_scores) plan->score_floats += (int64_t)n[i] * G * score_keys(total);
            }
        }
        grow0 += n[i];
    }
    plan->rows = grow0;
    auto longest_first = [](const auto& a, const auto& b) { return a.kv_end - a.kv_begin > b.kv_end - b.kv_begin; };
    std::stable_sort(plan->items.begin(), plan->items.end(), longest_first);
    std::stable_sort(plan->blocks.begin(), plan->blocks.end(), longest_first);
    return true;
}

}  // namespace ppd
