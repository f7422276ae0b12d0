// Tile list of attention over shared prefixes: which rows meet which keys in which workgroup, and whose partials make a row's result.
#include <algorithm>
#include <cmath>
#include <tuple>

#include "ppd_prefix.h"

namespace ppd {

namespace {

// A range of keys and the sequences [lo, hi] that have it, in the same pages: a shared one, or a sequence's own end with its new tokens.
struct Segment {
    int32_t lo, hi;
    int32_t begin, end;
    bool own;
};

int32_t ceil_div(int64_t a, int64_t b) { return (int32_t)((a + b - 1) / b); }

// What a tile takes, ns: its start and end, and a key while memory keeps up.  Measured over whole launches at D = 128 (start and end 3.6-4.2
// us and 1.2 us for four slabs of few columns, 5-6 us and 0.98 us a slab of 128 columns on bf16 pages, 1.09 on FP8; row blocks 6.6 us and 1.2 us
// for 64 keys, of launches that leave units idle: where every unit has one they are slower, and the 680 blocks of 18 next turns, which add up to
// 104 us over 256 units at this price, take 164-171); D = 64 by its share of the work.
struct TileTime { double start, key; };
TileTime tile_time(int ncols, int head_dim, int kv_elem_bytes) {
    const int waves = prefix_key_waves(ncols);
    const double half = head_dim == 64 ? 0.7 : 1.0;
    if (waves == 4) return {3600, 10 * half};
    if (waves == 2) return {6000, 20 * half};
    return {5500, (kv_elem_bytes == 1 ? 34 : 31) * half};
}
constexpr TileTime kRowBlockTime = {6600, 19};
// Over 19 batches (2 to 256 sequences, 300 to 60000 shared tokens) starts of 9 and 13 us for 128 columns, partials at 2.5 TB/s and reading added
// to the tiles' time in part gave the same on average within 1 %; keys' times and starts that knew no bound by memory 2 % more.
constexpr double kBytesPerNs = 6000, kPartialBytesPerNs = 4000, kJoinNs = 5000;

// Work that tiles are made of: `tiles` column ranges of `cols` columns each go over `keys` keys, for every KV head.
struct Range {
    int64_t keys;
    int32_t tiles, cols, max_keys;
    TileTime time;
    bool partial;  // its columns are joined with others', also where it is not cut
};

int32_t pieces_of(const Range& r, double slice) { return std::max(ceil_div(r.keys, r.max_keys), (int32_t)std::ceil(r.keys * r.time.key / slice)); }

// The time of keys, ns, at which ranges are cut, and *time of the launch: fewer tiles start less often and leave fewer partials, more fill the
// slots more evenly; and K and V have to be read, if only once for the column ranges side by side.
double reading_time(double keys, int32_t heads, int head_dim, int kv_elem_bytes) { return keys * 2 * head_dim * kv_elem_bytes * heads / kBytesPerNs + 4000; }

double choose_slice(const std::vector<Range>& ranges, int32_t heads, int32_t slots, int head_dim, int kv_elem_bytes, double* time) {
    double longest = 0, keys = 0, best = -1, slice = 0;
    for (const Range& r : ranges) {
        longest = std::max(longest, r.keys * r.time.key);
        keys += (double)r.keys;
    }
    const double reading = reading_time(keys, heads, head_dim, kv_elem_bytes);
    const int32_t share = std::max(1, slots / heads);
    std::vector<double> tiles;
    for (double c = longest + 1; c >= 1000; c *= 0.84) {
        double count = 0, sum = 0, most = 0, joined = 0;
        for (const Range& r : ranges) {
            const double pieces = pieces_of(r, c), cost = r.keys * r.time.key / pieces + r.time.start;
            count += pieces * r.tiles;
            sum += pieces * r.tiles * cost;
            most = std::max(most, cost);
            if (pieces > 1 || r.partial) joined += pieces * r.tiles * r.cols * heads;
        }
        if (count * heads > kMaxTiles) break;
        const double moved = joined * (head_dim + 2) * 4 / kPartialBytesPerNs;  // written, and read by the join
        const double behind = moved + (joined > 0 ? kJoinNs + moved : 0), least = std::max(std::max(most, sum / share), reading) + behind;
        if (best >= 0 && least >= best) {
            if (count > 16.0 * share) break;
            continue;
        }
        double est = count <= share ? most : sum / share + 0.5 * most;
        if (count > share && count <= 4.0 * share) {
            tiles.clear();
            for (const Range& r : ranges) {
                const int64_t pieces = pieces_of(r, c);
                tiles.insert(tiles.end(), (size_t)(pieces * r.tiles), r.keys * r.time.key / pieces + r.time.start);
            }
            est = last_tile_end(tiles, share);
        }
        est = std::max(est, reading) + behind;
        if (best < 0 || est < best) {
            best = est;
            slice = c;
        }
        if (count > 16.0 * share) break;
    }
    *time = std::max(0.0, best);
    return slice > 0 ? slice : longest + 1;
}

// A tile's keys in throughput, relative to those of few columns.
double key_cost(int64_t cols) {
    const int64_t full = cols / kPrefixCols, rest = cols % kPrefixCols;
    auto one = [](int64_t c) { return prefix_key_waves((int)c) == 4 ? 1.0 : prefix_key_waves((int)c) == 2 ? 0.85 : 1.65; };
    return full * one(kPrefixCols) + (rest ? one(rest) : 0);
}

// The shared ranges of sequences [lo, hi] from key `start` on, and their own ends.  common[i] is what sequence i has in common with the one
// before; the least of them is in common to all, and where it occurs they fall apart into runs.
class Segments {
public:
    Segments(const std::vector<int32_t>& common, const int32_t* L, const int32_t* n, const std::vector<int32_t>& row0, int G)
        : common_(common), L_(L), n_(n), row0_(row0), G_(G) {}
    std::vector<Segment> list;

    // A shared range has to save more than it costs: the tiles of the runs that have fewer columns, and their reading the keys each for
    // itself (half a key's time), against a partial's columns more to be written and read (3.7 keys' time each, 1040 bytes) and a tile's start.
    // Ranges that are shared nest at most kMaxNested deep.  Runs that are not worth it may fall apart as often as there are lengths in common,
    // so what is left to do is kept in a list (the first run last) and not on the stack.
    void add(int32_t first, int32_t last) {
        struct Run { int32_t lo, hi, start, level; };
        std::vector<Run> todo{{first, last, 0, 0}};
        while (!todo.empty()) {
            const int32_t lo = todo.back().lo, hi = todo.back().hi;
            int32_t start = todo.back().start, level = todo.back().level;
            todo.pop_back();
            if (lo == hi || level == kMaxNested) {
                for (int32_t i = lo; i <= hi; ++i) list.push_back({i, i, start, L_[i] + n_[i], true});
                continue;
            }
            const int32_t least = *std::min_element(common_.begin() + lo + 1, common_.begin() + hi + 1);
            double apart = -0.5;
            for (int32_t from = lo; from <= hi;) {
                const int32_t to = run_end(from, hi, least);
                apart += key_cost(columns(from, to)) + 0.5;
                from = to + 1;
            }
            const int64_t cols = columns(lo, hi);
            if ((least - start) * (apart - key_cost(cols)) > 3.7 * cols + 200) {
                list.push_back({lo, hi, start, least, false});
                start = least;
                ++level;
            }
            const size_t at = todo.size();
            for (int32_t from = lo; from <= hi;) {
                const int32_t to = run_end(from, hi, least);
                todo.push_back({from, to, start, level});
                from = to + 1;
            }
            std::reverse(todo.begin() + at, todo.end());
        }
    }

private:
    int32_t run_end(int32_t from, int32_t hi, int32_t least) const {
        while (from < hi && common_[from + 1] > least) ++from;
        return from;
    }
    int64_t columns(int32_t lo, int32_t hi) const { return (int64_t)(row0_[hi + 1] - row0_[lo]) * G_; }

    const std::vector<int32_t>& common_;
    const int32_t *L_, *n_;
    const std::vector<int32_t>& row0_;
    int G_;
};

// The longest tiles first, and those of the same keys (the column ranges of one segment, head and piece) one after the other on one XCD:
// workgroups go round the XCDs, each of which has an L2 of its own.
template <class Item, class Time>
void order_for_xcds(std::vector<Item>& items, Time time) {
    struct Key {
        int64_t time;
        int32_t seq, kvh, begin, total;
        uint32_t index;
        bool same_keys(const Key& o) const { return seq == o.seq && kvh == o.kvh && begin == o.begin && total == o.total && time == o.time; }
        bool operator<(const Key& o) const {
            if (time != o.time) return time > o.time;
            return std::tie(seq, kvh, begin, total, index) < std::tie(o.seq, o.kvh, o.begin, o.total, o.index);
        }
    };
    std::vector<Key> keys(items.size());
    for (size_t i = 0; i < items.size(); ++i) keys[i] = {time(items[i]), items[i].seq, items[i].kvh, items[i].kv_begin, items[i].kv_total, (uint32_t)i};
    std::sort(keys.begin(), keys.end());
    std::vector<uint32_t> lists[kXcds];
    for (size_t i = 0; i < keys.size();) {
        size_t to = i + 1;
        while (to < keys.size() && keys[i].same_keys(keys[to])) ++to;
        auto* const least = std::min_element(lists, lists + kXcds, [](const auto& a, const auto& b) { return a.size() < b.size(); });
        for (; i < to; ++i) least->push_back(keys[i].index);
    }
    std::vector<Item> ordered;
    ordered.reserve(items.size());
    size_t longest = 0;
    for (const auto& l : lists) longest = std::max(longest, l.size());
    for (size_t k = 0; k < longest; ++k)
        for (const auto& l : lists)
            if (k < l.size()) ordered.push_back(items[l[k]]);
    items.swap(ordered);
}

}  // namespace

bool build_prefix_plan(const ppd_shape& s, const int32_t* shared, const int32_t* L, const int32_t* n, int32_t B, int kv_elem_bytes, int num_cus, PrefixPlan* plan) {
    const int G = s.num_q_heads / s.num_kv_heads, Hkv = s.num_kv_heads, D = s.head_dim;
    *plan = PrefixPlan();
    std::vector<int32_t> common(B, 0), row0(B + 1, 0);
    for (int i = 0; i < B; ++i) {
        row0[i + 1] = row0[i] + n[i];
        if (i > 0) common[i] = shared[i] / kSharedStep * kSharedStep;
        plan->keys_alone += (int64_t)L[i] + n[i];
    }
    auto rows_of = [&](const Segment& g) { return row0[g.hi + 1] - row0[g.lo]; };
    // How a segment is cut: `tiles` column ranges of `rows` rows each.
    struct Cut { bool is_wide; int32_t tiles, rows, key_waves; TileTime time; };
    // A list of segments, how it is cut and its time.  Row blocks are a launch of their own: where a sequence has more columns than a tile
    // takes there is one, and it takes all segments of more than 32 columns.
    struct Choice {
        std::vector<Segment> segments;
        bool any_wide = false, possible = true;
        double narrow_slice = 0, wide_slice = 0, time = 0;
    };
    auto cut_of = [&](const Choice& x, const Segment& g) {
        const int32_t rows = rows_of(g);
        Cut c;
        c.is_wide = x.any_wide && (int64_t)rows * G > kTreeCols;
        const int32_t most = (c.is_wide ? kMfmaCols : kPrefixCols) / G;
        c.tiles = ceil_div(rows, most);
        c.rows = ceil_div(rows, c.tiles);
        c.key_waves = prefix_key_waves(std::min<int32_t>(c.rows * G, kPrefixCols));
        c.time = c.is_wide ? kRowBlockTime : tile_time(c.rows * G, D, kv_elem_bytes);
        return c;
    };
    auto weigh = [&](Choice& x) {
        for (const Segment& g : x.segments) x.any_wide |= g.own && (int64_t)rows_of(g) * G > kPrefixCols;
        double fewest = 0;
        std::vector<Range> narrow, wide;
        for (const Segment& g : x.segments) {
            const Cut c = cut_of(x, g);
            const int32_t max_keys = c.is_wide ? kMaxTreeBlockChunk : kMaxPrefixChunk;
            std::vector<Range>& list = c.is_wide ? wide : narrow;
            if (!g.own || c.tiles == 1) {
                list.push_back({g.end - g.begin, c.tiles, c.rows * G, max_keys, c.time, !g.own || g.begin > 0});
            } else {  // a tile's last row sees no keys behind itself
                for (int32_t r = 0; r < rows_of(g); r += c.rows)
                    list.push_back({std::min(g.end, L[g.lo] + r + c.rows) - g.begin, 1, c.rows * G, max_keys, c.time, g.begin > 0});
            }
            fewest += (double)c.tiles * Hkv * ((double)(g.end - g.begin) / max_keys + 1);
        }
        x.possible = fewest <= kMaxTiles;
        if (!x.possible) return;
        double narrow_time = 0, wide_time = 0;
        if (!narrow.empty()) x.narrow_slice = choose_slice(narrow, Hkv, 2 * num_cus, D, kv_elem_bytes, &narrow_time);
        if (!wide.empty()) x.wide_slice = choose_slice(wide, Hkv, num_cus, D, kv_elem_bytes, &wide_time);
        x.time = narrow_time + wide_time;
    };
    Choice choice;
    {
        Segments segments(common, L, n, row0, G);
        for (int32_t from = 0; from < B;) {  // what shares nothing stands alone
            int32_t to = from;
            while (to + 1 < B && common[to + 1] > 0) ++to;
            segments.add(from, to);
            from = to + 1;
        }
        choice.segments.swap(segments.list);
    }
    weigh(choice);
    // (Keys that have to be read anyway, once for each sequence, may already say that it takes longer.)
    if (choice.segments.size() > (size_t)B && (!choice.possible || reading_time((double)plan->keys_alone, Hkv, D, kv_elem_bytes) < choice.time)) {
        // Nothing shared, and where no range is cut either no join: small batches (three sequences of 231 keys, 200 of them shared, 8.3 -> 5.3 us).
        Choice apart;
        for (int32_t i = 0; i < B; ++i) apart.segments.push_back({i, i, 0, L[i] + n[i], true});
        weigh(apart);
        if (apart.possible && (!choice.possible || apart.time < choice.time)) choice = std::move(apart);
    }
    if (!choice.possible) return false;

    // Sources of the rows, in the order of the segments: a sequence's shared ranges come before its own end.
    std::vector<std::vector<JoinSource>> unit_sources;
    struct PlacedTile { int32_t cols, nsplit; int64_t part_off; };  // a column range's; part_off -1: it writes the result
    struct Placed { int32_t row0, tile_rows; bool is_wide; std::vector<PlacedTile> tiles; };
    std::vector<Placed> path;  // the shared ranges around the segment at hand, and itself
    std::vector<const Segment*> around;
    for (const Segment& g : choice.segments) {
        while (!around.empty() && around.back()->hi < g.lo) {
            around.pop_back();
            path.pop_back();
        }
        const Cut c = cut_of(choice, g);
        const int32_t total_rows = rows_of(g);
        const int32_t step = c.is_wide ? kTileTokens : kSlab * c.key_waves, most = c.is_wide ? kMaxTreeBlockChunk : kMaxPrefixChunk;
        path.push_back({row0[g.lo], c.rows, c.is_wide, {}});
        for (int32_t r = 0; r < total_rows; r += c.rows) {
            const int32_t nrows = std::min(c.rows, total_rows - r), cols = nrows * G;
            // its last row sees no keys behind itself
            const int32_t last = g.own ? std::min(g.end, L[g.lo] + r + nrows) : g.end, keys = last - g.begin;
            const int32_t pieces = pieces_of({keys, 0, 0, most, c.time, false}, c.is_wide ? choice.wide_slice : choice.narrow_slice);
            const int32_t piece = std::min(most, ceil_div(ceil_div(keys, pieces), step) * step);
            const int32_t nsplit = ceil_div(keys, piece);
            const bool direct = g.own && around.empty() && nsplit == 1;
            const int32_t cached = g.own ? L[g.lo] + r : g.end;  // the new tokens before the tile's rows are seen by all of them
            const int64_t stride = (int64_t)cols * (D + 2);
            path.back().tiles.push_back({cols, nsplit, direct ? -1 : plan->partial_floats});
            plan->keys_read += keys;
            for (int h = 0; h < Hkv; ++h)
                for (int32_t p = 0; p < nsplit; ++p) {
                    const int32_t begin = g.begin + p * piece, end = std::min(last, begin + piece);
                    const int64_t part = direct ? -1 : plan->partial_floats + ((int64_t)h * nsplit + p) * stride;
                    if (c.is_wide) {
                        ppd_work_item it{};
                        it.kind = 1;
                        it.seq = g.lo;
                        it.kvh = h;
                        it.nrows = nrows;
                        it.grow0 = row0[g.lo] + r;
                        it.L = cached;
                        it.kv_total = g.end;
                        it.kv_begin = begin;
                        it.kv_end = end;
                        it.group = -1;
                        it.part_off = part;
                        plan->blocks.push_back(it);
                    } else {
                        plan->items.push_back({g.lo, h, row0[g.lo] + r, cols, cached, g.end, begin, end, part});
                    }
                }
            if (!direct) plan->partial_floats += stride * nsplit * Hkv;
            if (plan->items.size() + plan->blocks.size() > (size_t)kMaxTiles) return false;
        }
        if (!g.own) {
            around.push_back(&g);
            continue;
        }
        // The sequence's rows, cut where a tile of any of its ranges ends.
        for (int32_t r = row0[g.lo]; r < row0[g.lo + 1];) {
            int32_t end = row0[g.lo + 1];
            for (const Placed& x : path) end = std::min(end, x.row0 + ((r - x.row0) / x.tile_rows + 1) * x.tile_rows);
            if (path.back().tiles[(r - path.back().row0) / c.rows].part_off >= 0) {
                plan->units.push_back({r, end - r, (int32_t)path.size(), 0});
                unit_sources.emplace_back();
                plan->source_stride = std::max(plan->source_stride, (int32_t)path.size());
                plan->join_cols = std::max(plan->join_cols, (end - r) * G);
                for (const Placed& x : path) {
                    const int32_t tile = (r - x.row0) / x.tile_rows;
                    const PlacedTile& t = x.tiles[tile];
                    unit_sources.back().push_back({t.part_off, t.cols, (r - x.row0 - tile * x.tile_rows) * G, t.nsplit, x.is_wide || prefix_key_waves(t.cols) > 1});
                }
            }
            r = end;
        }
        path.pop_back();
    }
    plan->sources.reserve(unit_sources.size() * plan->source_stride);
    for (auto& of_unit : unit_sources) {
        of_unit.resize(plan->source_stride, JoinSource{});
        plan->sources.insert(plan->sources.end(), of_unit.begin(), of_unit.end());
    }
    order_for_xcds(plan->items, [&](const PrefixItem& x) { 
        const TileTime t = tile_time(x.ncols, D, kv_elem_bytes);
        return (int64_t)((x.kv_end - x.kv_begin) * t.key + t.start);
    });
    order_for_xcds(plan->blocks, [](const ppd_work_item& x) { return (int64_t)(x.kv_end - x.kv_begin); });
    return true;
}

// A part reads its shared ranges once more, and its launches start and drain once more.  500 turns of 16 rows behind 30016 tokens (64 query heads,
// D = 128; 1.3 GB of partials) 7.78 ms at once and 7.72 in two parts, 2000 of 4 rows 8.04 and 7.95, 120 of 200 rows (2.4 GB) 20.74 and 20.77.
bool build_prefix_parts(const ppd_shape& s, const int32_t* shared, const int32_t* L, const int32_t* n, int32_t B, int kv_elem_bytes, int num_cus, int64_t most_floats,
                        PrefixPlan* plan) {
    std::vector<int32_t> row0(B + 1, 0);
    for (int32_t i = 0; i < B; ++i) row0[i + 1] = row0[i] + n[i];
    struct Span { int32_t lo, hi; };
    std::vector<Span> todo{{0, B}};  // the first one last
    PrefixPlan all, part;
    std::vector<int32_t> common;
    while (!todo.empty()) {
        const Span x = todo.back();
        todo.pop_back();
        common.assign(shared + x.lo, shared + x.hi);
        common[0] = 0;  // with a sequence of another part
        if (!build_prefix_plan(s, common.data(), L + x.lo, n + x.lo, x.hi - x.lo, kv_elem_bytes, num_cus, &part)) return false;
        if (part.partial_floats > most_floats && x.hi - x.lo > 1) {
            const int32_t half = row0[x.lo] + (row0[x.hi] - row0[x.lo]) / 2;
            const int32_t at = (int32_t)(std::lower_bound(row0.begin() + x.lo + 1, row0.begin() + x.hi - 1, half) - row0.begin());
            todo.push_back({at, x.hi});
            todo.push_back({x.lo, at});
            continue;
        }
        all.parts.push_back({(int64_t)all.items.size(), (int64_t)all.blocks.size(), (int64_t)all.units.size(), (int64_t)all.sources.size(), (int32_t)part.items.size(),
                             (int32_t)part.blocks.size(), (int32_t)part.units.size(), part.join_cols, part.source_stride});
        for (PrefixItem& t : part.items) t.seq += x.lo, t.grow0 += row0[x.lo];
        for (ppd_work_item& t : part.blocks) t.seq += x.lo, t.grow0 += row0[x.lo];
        for (JoinUnit& u : part.units) u.grow0 += row0[x.lo];
        auto append = [](auto& to, auto& from) {
            if (to.empty()) to.swap(from);
            else to.insert(to.end(), from.begin(), from.end());
        };
        append(all.items, part.items);
        append(all.blocks, part.blocks);
        append(all.units, part.units);
        append(all.sources, part.sources);
        all.partial_floats = std::max(all.partial_floats, part.partial_floats);
        all.join_cols = std::max(all.join_cols, part.join_cols);
        all.source_stride = std::max(all.source_stride, part.source_stride);
        all.keys_read += part.keys_read;
        all.keys_alone += part.keys_alone;
    }
    *plan = std::move(all);
    return true;
}

}  // namespace ppd
