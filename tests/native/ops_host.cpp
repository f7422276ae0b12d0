// Host-only checks of the drafting and eviction entry points (built and run by tests/test_ops_host.py): their host code as it is,
// compiled against the stand-in runtime of host_runtime/, whose launches are recorded instead of run.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>
#include <limits>
#include <map>
#include <random>
#include <set>
#include <vector>

#include "../../paper_2603_13358_amd/csrc/ppd_api.hip"
#include "../../paper_2603_13358_amd/csrc/ppd_ops_api.hip"

std::function<void()> sim_bind(const void* f, void** args) {
    if (f != reinterpret_cast<const void*>(&ppd_upload_kernel)) std::abort();
    auto host = *static_cast<const uint4**>(args[0]);
    auto dev = *static_cast<uint4**>(args[1]);
    auto granules = *static_cast<int64_t*>(args[2]);
    auto counters = *static_cast<uint32_t**>(args[3]);
    auto read = *static_cast<uint32_t**>(args[4]);
    auto serial = *static_cast<uint32_t*>(args[5]);
    return [=] { ppd_upload_kernel(host, dev, granules, counters, read, serial); };
}

static std::vector<ppd::TreeParams> g_tree, g_weigh;
static std::vector<ppd::TreeBlockParams> g_blocks;
static std::vector<ppd::SelectParams> g_select;
static std::vector<ppd::CompactParams> g_compact;

namespace ppd {
int prepare_mixed_kernels() { return 0; }
int launch_mixed(const KParams&, int, int, void*, bool) { return 0; }
int launch_narrow(const KParams&, int, int, void*, bool) { return 0; }
int launch_mfma_only(const KParams&, int, int, void*) { return 0; }
int launch_stream_only(const KParams&, int, int, void*) { return 0; }
int launch_merge(const MergeParams&, void*) { return 0; }
int launch_kv_append(const uint16_t*, const uint16_t*, void*, const int64_t*, int64_t, int, int, int64_t, int, int64_t, uint32_t*,
                     void*, bool, float, float) { return 0; }
int launch_tree(const TreeParams& p, int, bool, void*) { g_tree.push_back(p); return 0; }
int launch_tree_blocks(const TreeBlockParams& p, int, bool, void*) { g_blocks.push_back(p); return 0; }
int launch_tree_join(const TreeParams&, int, void*) { return 0; }
int launch_weigh(const TreeParams& p, int, bool, void*) { g_weigh.push_back(p); return 0; }
int launch_select(const SelectParams& p, int, void*) { g_select.push_back(p); return 0; }
int launch_compact(const CompactParams& p, int, bool, int, void*) { g_compact.push_back(p); return 0; }
}  // namespace ppd

#define CHECK(x)                                                      \
    do {                                                              \
        if (!(x)) {                                                   \
            std::printf("%s:%d: not so: %s\n", __FILE__, __LINE__, #x); \
            std::fflush(stdout);                                      \
            std::_Exit(1);                                            \
        }                                                             \
    } while (0)

// calls of the wide kind here have row blocks, so every call launches them once
static size_t attentions() { return g_blocks.size(); }

alignas(16) static char device[64];
static const int32_t* const tables = reinterpret_cast<const int32_t*>(device);
static const uint64_t* const masks = reinterpret_cast<const uint64_t*>(device);
static float* const floats = reinterpret_cast<float*>(device);
static int32_t* const ints = reinterpret_cast<int32_t*>(device);

static ppd_ctx* make(int hq, int hkv, int dim) {
    const ppd_shape s = {hq, hkv, dim, 16, 4096};
    ppd_ctx* ctx = nullptr;
    CHECK(ppd_create(&s, 0, &ctx) == PPD_OK);
    return ctx;
}

// Every refusal comes before anything is enqueued.
static void refusals() {
    ppd_ctx* ctx = make(32, 8, 128);
    const int32_t L[2] = {100, 0}, n[2] = {5, 64};
    const float nan = std::numeric_limits<float>::quiet_NaN();
    auto tree = [&](const void* q, const void* pool, const int32_t* pt, int max_pages, const uint64_t* mask, int words, const int32_t* l, const int32_t* m, int B, float scale, void* out) {
        return ppd_tree_attention(ctx, q, pool, pt, max_pages, mask, words, l, m, B, scale, out, nullptr);
    };
    CHECK(tree(device, device, tables, 7, masks, 1, L, n, 2, 1.f, device) == PPD_OK);
    CHECK(attentions() == 1);
    CHECK(tree(device, device, tables, 7, masks, 1, L, n, 0, 1.f, device) == PPD_OK);
    CHECK(ppd_tree_attention(nullptr, device, device, tables, 7, masks, 1, L, n, 2, 1.f, device, nullptr) == PPD_ERR_NULL);
    CHECK(tree(nullptr, device, tables, 7, masks, 1, L, n, 2, 1.f, device) == PPD_ERR_NULL);
    CHECK(tree(device, nullptr, tables, 7, masks, 1, L, n, 2, 1.f, device) == PPD_ERR_NULL);
    CHECK(tree(device, device, nullptr, 7, masks, 1, L, n, 2, 1.f, device) == PPD_ERR_NULL);
    CHECK(tree(device, device, tables, 7, nullptr, 1, L, n, 2, 1.f, device) == PPD_ERR_NULL);
    CHECK(tree(device, device, tables, 7, masks, 1, nullptr, n, 2, 1.f, device) == PPD_ERR_NULL);
    CHECK(tree(device, device, tables, 7, masks, 1, L, nullptr, 2, 1.f, device) == PPD_ERR_NULL);
    CHECK(tree(device, device, tables, 7, masks, 1, L, n, 2, 1.f, nullptr) == PPD_ERR_NULL);
    CHECK(tree(device, device, tables, 7, masks, 1, L, n, -1, 1.f, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device, tables, 7, masks, 0, L, n, 2, 1.f, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device, tables, 7, masks, 17, L, n, 2, 1.f, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device, tables, 7, masks, 1, L, n, 2, -1.f, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device, tables, 7, masks, 1, L, n, 2, nan, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device, tables, 7, masks, 1, L, n, 2, INFINITY, device) == PPD_ERR_RANGE);
    CHECK(tree(device + 2, device, tables, 7, masks, 1, L, n, 2, 1.f, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device + 8, tables, 7, masks, 1, L, n, 2, 1.f, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device, tables, 7, masks, 1, L, n, 2, 1.f, device + 4) == PPD_ERR_RANGE);
    CHECK(tree(device, device, reinterpret_cast<const int32_t*>(device + 2), 7, masks, 1, L, n, 2, 1.f, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device, tables, 7, reinterpret_cast<const uint64_t*>(device + 4), 1, L, n, 2, 1.f, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device, tables, 6, masks, 1, L, n, 2, 1.f, device) == PPD_ERR_PAGETABLE);
    const int32_t none[2] = {5, 0}, more[2] = {5, 65}, below[2] = {-1, 0}, far[2] = {INT32_MAX - 2, 0};
    CHECK(tree(device, device, tables, 7, masks, 1, L, none, 2, 1.f, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device, tables, 7, masks, 1, L, more, 2, 1.f, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device, tables, 7, masks, 2, L, more, 2, 1.f, device) == PPD_OK);
    CHECK(tree(device, device, tables, 7, masks, 1, below, n, 2, 1.f, device) == PPD_ERR_RANGE);
    CHECK(tree(device, device, tables, INT32_MAX, masks, 1, far, n, 2, 1.f, device) == PPD_ERR_RANGE);
    CHECK(std::string(ppd_last_error(ctx)).size() > 0 && attentions() == 2);

    auto weighted = [&](float* w, int64_t stride) { return ppd_weighted_attention(ctx, device, device, tables, 7, L, n, 2, 1.f, device, w, stride, nullptr); };
    CHECK(weighted(floats, 105) == PPD_OK && g_weigh.size() == 1);
    CHECK(weighted(nullptr, 105) == PPD_ERR_NULL);
    CHECK(weighted(floats, 104) == PPD_ERR_RANGE);
    CHECK(weighted(reinterpret_cast<float*>(device + 2), 105) == PPD_ERR_RANGE);

    const int32_t len[2] = {10, 0}, longer[2] = {10, 21}, negative[2] = {-1, 3};
    auto select = [&](const float* w, const int32_t* l, int B, int budget, int sinks, int recent, int32_t* keep, int64_t ks) {
        return ppd_kv_select(ctx, w, 20, l, B, budget, sinks, recent, keep, ks, nullptr);
    };
    CHECK(select(floats, len, 2, 8, 1, 7, ints, 8) == PPD_OK && g_select.size() == 1);
    CHECK(select(floats, len, 0, 8, 1, 7, ints, 8) == PPD_OK && g_select.size() == 1);
    CHECK(select(nullptr, len, 2, 8, 1, 2, ints, 8) == PPD_ERR_NULL);
    CHECK(select(floats, nullptr, 2, 8, 1, 2, ints, 8) == PPD_ERR_NULL);
    CHECK(select(floats, len, 2, 8, 1, 2, nullptr, 8) == PPD_ERR_NULL);
    CHECK(select(floats, len, -1, 8, 1, 2, ints, 8) == PPD_ERR_RANGE);
    CHECK(select(floats, len, 2, 0, 0, 0, ints, 8) == PPD_ERR_RANGE);
    CHECK(select(floats, len, 2, 8, -1, 2, ints, 8) == PPD_ERR_RANGE);
    CHECK(select(floats, len, 2, 8, 1, -2, ints, 8) == PPD_ERR_RANGE);
    CHECK(select(floats, len, 2, 8, 2, 7, ints, 8) == PPD_ERR_RANGE);
    CHECK(select(floats, len, 2, INT32_MAX, INT32_MAX, 1, ints, 8) == PPD_ERR_RANGE);
    CHECK(select(floats, len, 2, 8, 1, 2, ints, 7) == PPD_ERR_RANGE);
    CHECK(select(floats, longer, 2, 8, 1, 2, ints, 8) == PPD_ERR_RANGE);
    CHECK(select(floats, negative, 2, 8, 1, 2, ints, 8) == PPD_ERR_RANGE);
    CHECK(select(reinterpret_cast<float*>(device + 1), len, 2, 8, 1, 2, ints, 8) == PPD_ERR_RANGE);
    CHECK(select(floats, len, 2, 8, 1, 2, reinterpret_cast<int32_t*>(device + 2), 8) == PPD_ERR_RANGE);
    CHECK(ppd_kv_select(nullptr, floats, 20, len, 2, 8, 1, 2, ints, 8, nullptr) == PPD_ERR_NULL && g_select.size() == 1);

    const int32_t first[2] = {0, 7}, count[2] = {8, 0}, zero[2] = {0, 0};
    const int64_t pool = 2LL * 8 * 16 * 128 * 4096;
    struct Compact {
        void* pages = device;
        int64_t layer = 0;
        int layers = 1;
        const int32_t* pt = tables;
        int max_pages = 2;
        const int32_t* keep = ints;
        int64_t kl = 0, ks = 8, kh = 0;
        const int32_t *first, *count;
        int B = 2;
        float* w = nullptr;
        int64_t stride = 0;
    };
    Compact good;
    good.first = first;
    good.count = count;
    auto compact = [&](const Compact& c) {
        return ppd_kv_compact(ctx, c.pages, c.layer, c.layers, c.pt, c.max_pages, c.keep, c.kl, c.ks, c.kh, c.first, c.count, c.B, c.w, c.stride, nullptr);
    };
    auto with = [&](auto change) {
        Compact c = good;
        change(c);
        return compact(c);
    };
    CHECK(compact(good) == PPD_OK && g_compact.size() == 1);
    CHECK(with([](Compact& c) { c.B = 0; }) == PPD_OK && with([](Compact& c) { c.layers = 0; }) == PPD_OK && with([&](Compact& c) { c.count = zero; }) == PPD_OK);
    CHECK(g_compact.size() == 1);
    CHECK(with([](Compact& c) { c.pages = nullptr; }) == PPD_ERR_NULL);
    CHECK(with([](Compact& c) { c.pt = nullptr; }) == PPD_ERR_NULL);
    CHECK(with([](Compact& c) { c.keep = nullptr; }) == PPD_ERR_NULL);
    CHECK(with([](Compact& c) { c.first = nullptr; }) == PPD_ERR_NULL);
    CHECK(with([](Compact& c) { c.count = nullptr; }) == PPD_ERR_NULL);
    CHECK(with([](Compact& c) { c.B = -1; }) == PPD_ERR_RANGE);
    CHECK(with([](Compact& c) { c.layers = -1; }) == PPD_ERR_RANGE);
    CHECK(with([](Compact& c) { c.layers = 65536; }) == PPD_ERR_RANGE);
    CHECK(with([&](Compact& c) { c.layers = 2, c.layer = pool - 8; }) == PPD_ERR_RANGE);
    CHECK(with([&](Compact& c) { c.layers = 2, c.layer = pool + 4; }) == PPD_ERR_RANGE);
    CHECK(with([&](Compact& c) { c.layers = 2, c.layer = pool + 8; }) == PPD_OK);
    CHECK(with([](Compact& c) { c.pages = device + 8; }) == PPD_ERR_RANGE);
    CHECK(with([](Compact& c) { c.keep = reinterpret_cast<int32_t*>(device + 2); }) == PPD_ERR_RANGE);
    CHECK(with([](Compact& c) { c.w = reinterpret_cast<float*>(device + 2), c.stride = 100; }) == PPD_ERR_RANGE);
    CHECK(with([](Compact& c) { c.w = floats, c.stride = 7; }) == PPD_ERR_RANGE);
    CHECK(with([](Compact& c) { c.w = floats, c.stride = 8; }) == PPD_OK);
    CHECK(with([](Compact& c) { c.max_pages = 0; }) == PPD_ERR_PAGETABLE);
    CHECK(with([](Compact& c) { c.ks = 7; }) == PPD_ERR_RANGE);
    CHECK(with([](Compact& c) { c.kl = -8; }) == PPD_ERR_RANGE);
    CHECK(with([&](Compact& c) { c.first = negative; }) == PPD_ERR_RANGE);
    CHECK(with([&](Compact& c) { c.count = negative; }) == PPD_ERR_RANGE);
    CHECK(g_compact.size() == 3);
    CHECK(ppd_set_kv_format(ctx, PPD_KV_FP8_E4M3, 1.f, 1.f) == PPD_OK);
    CHECK(with([&](Compact& c) { c.layers = 2, c.layer = pool + 8; }) == PPD_ERR_RANGE);
    ppd_destroy(ctx);
}

// Whatever the lengths: every query column meets every key exactly once, what is split is joined, partials do not overlap, no tile
// has more page ids than its LDS, and every key is weighed once.
static void plans() {
    std::mt19937 rng(3);
    int split = 0, whole = 0, blocks = 0;
    size_t with_scores = 0, without = 0;
    for (int trial = 0; trial < 200; ++trial) {
        const int hkv = 1 + rng() % 8, G = 1 + rng() % 8, dim = rng() % 2 ? 128 : 64;
        const ppd_shape s = {hkv * G, hkv, dim, 16, 1 << 20};
        std::vector<int32_t> L((size_t)(1 + rng() % 20)), n(L.size());
        for (auto& x : L) x = (int32_t)(rng() % (1u << (1 + rng() % 17)));
        for (auto& x : n) x = 1 + (int32_t)(rng() % (1u << (rng() % 9)));
        const bool weighted = rng() % 2;
        const int eb = 1 + rng() % 2;
        ppd::TreePlan p;
        CHECK(ppd::build_tree_plan(s, L.data(), n.data(), (int)L.size(), weighted, eb, 256, &p));
        std::vector<int> grow0(L.size() + 1, 0);
        for (size_t i = 0; i < L.size(); ++i) grow0[i + 1] = grow0[i] + n[i];
        CHECK(p.rows == grow0.back());
        std::map<std::tuple<int, int, int>, std::map<int, int>> ranges;  // (sequence, head, first column) -> begin -> end
        std::map<std::tuple<int, int, int>, int> widths;
        std::set<int64_t> offsets;
        auto tile = [&](int seq, int kvh, int col0, int ncols, int Li, int kv_total, int begin, int end, int64_t part_off) {
            CHECK(seq >= 0 && seq < (int)L.size() && kvh >= 0 && kvh < hkv);
            CHECK(Li == L[seq] && kv_total == L[seq] + n[seq]);
            CHECK(ncols >= 1 && col0 >= 0 && col0 + ncols <= n[seq] * G);
            CHECK(begin >= 0 && begin < end && end <= kv_total);
            CHECK(ranges[std::make_tuple(seq, kvh, col0)].emplace(begin, end).second);
            widths[std::make_tuple(seq, kvh, col0)] = ncols;
            if (part_off >= 0) {
                CHECK(part_off + (int64_t)ncols * (dim + 2) <= p.partial_floats && offsets.insert(part_off).second && part_off % 2 == 0);
                ++split;
            } else {
                CHECK(begin == 0 && end == kv_total);
                ++whole;
            }
        };
        for (const auto& it : p.items) {
            tile(it.seq, it.kvh, 0, it.ncols, it.L, it.kv_total, it.kv_begin, it.kv_end, it.part_off);
            CHECK(it.grow0 == grow0[it.seq] && it.ncols <= ppd::kTreeCols && it.ncols == n[it.seq] * G && it.kv_begin % ppd::kSlab == 0);
            CHECK((it.kv_end - it.kv_begin + ppd::kSlab - 1) / ppd::kSlab * 2 <= ppd::kMaxTreeChunk / 16);
        }
        for (const auto& it : p.blocks) {
            tile(it.seq, it.kvh, it.row0 * G, it.nrows * G, it.L, it.kv_total, it.kv_begin, it.kv_end, it.part_off);
            CHECK(it.grow0 == grow0[it.seq] + it.row0 && it.nrows * G <= ppd::kMfmaCols && it.kv_begin % ppd::kTileTokens == 0);
            // the last id's place in LDS is the flag's
            CHECK((it.kv_end - it.kv_begin + ppd::kTileTokens - 1) / ppd::kTileTokens * 4 < ppd::kMaxMfmaChunk / 16 - 1);
            ++blocks;
        }
        int64_t columns = 0;
        for (const auto& r : ranges) {
            int at = 0;
            for (const auto& [b, e] : r.second) {
                CHECK(b == at);
                at = e;
            }
            CHECK(at == L[std::get<0>(r.first)] + n[std::get<0>(r.first)]);
            columns += widths[r.first];
        }
        CHECK(columns == (int64_t)p.rows * G * hkv);
        for (const auto& g : p.groups) CHECK(g.ncols <= p.join_cols);
        std::set<int64_t> joined;
        for (const auto& g : p.groups)
            for (int j = 0; j < g.nsplit; ++j) CHECK(offsets.count(g.part_off + j * g.part_stride) && joined.insert(g.part_off + j * g.part_stride).second);
        CHECK(joined.size() == offsets.size());
        int64_t weighed = 0;
        std::set<std::tuple<int, int, int>> once;
        std::vector<ppd::WeighItem> all = p.weighs;
        all.insert(all.end(), p.score_weighs.begin(), p.score_weighs.end());
        std::map<std::pair<int, int>, int64_t> kept;  // where the scores of a sequence and head go
        for (const auto& it : p.items)
            if (it.score_off >= 0) CHECK(weighted && ppd::score_keys(it.kv_end - it.kv_begin) * it.ncols <= ppd::kKeptScores && kept.emplace(std::make_pair(it.seq, it.kvh), it.score_off).first->second == it.score_off);
        std::map<int64_t, int64_t> areas;
        for (const auto& k : kept) CHECK(areas.emplace(k.second, k.second + (int64_t)n[k.first.first] * G * ppd::score_keys(L[k.first.first] + n[k.first.first])).second);
        int64_t area_end = 0;
        for (const auto& a : areas) {
            CHECK(a.first == area_end && a.first % 4 == 0);
            area_end = a.second;
        }
        CHECK(area_end == p.score_floats);
        for (const auto& w : p.weighs) CHECK(w.score_off < 0);
        for (const auto& w : p.score_weighs) CHECK(kept.at(std::make_pair(w.seq, w.kvh)) == w.score_off);
        for (const auto& w : p.score_weighs) {
            if (w.group >= 0) CHECK(p.groups.at(w.group).kvh == w.kvh && p.groups[w.group].grow0 == w.grow0 && p.groups[w.group].ncols == w.cols && p.groups[w.group].col0 == 0);
            else CHECK(ranges.at(std::make_tuple(w.seq, w.kvh, 0)).size() == 1);
        }
        with_scores += p.score_weighs.size();
        without += p.weighs.size();
        for (const auto& w : all) {
            CHECK(w.kv_begin % ppd::kWeighKeys == 0 && w.kv_begin < w.kv_total && w.kv_total == L[w.seq] + n[w.seq] && w.cols == n[w.seq] * G && w.grow0 == grow0[w.seq]);
            CHECK(once.insert(std::make_tuple(w.seq, w.kvh, w.kv_begin)).second);
            weighed += std::min(ppd::kWeighKeys, w.kv_total - w.kv_begin);
        }
        int64_t keys = 0;
        for (size_t i = 0; i < L.size(); ++i) keys += (int64_t)hkv * (L[i] + n[i]);
        CHECK(weighed == (weighted ? keys : 0));
    }
    CHECK(with_scores > 1000 && without > 1000 && split > 1000 && whole > 1000 && blocks > 1000 && blocks < split + whole - 1000);
    // a batch beyond what one launch takes is refused, not built
    const ppd_shape s = {8192, 1024, 128, 16, 1 << 16};
    std::vector<int32_t> L(4096, 100), n(4096, 64);
    ppd::TreePlan p;
    CHECK(!ppd::build_tree_plan(s, L.data(), n.data(), 4096, true, 2, 256, &p));
}

// Long batches go out in launches of what the kernel arguments hold, each with its own part of every array.
static void batches() {
    ppd_ctx* ctx = make(32, 8, 128);
    const int B = 1300;
    std::vector<int32_t> len(B), first(B), count(B);
    for (int i = 0; i < B; ++i) len[i] = i % 50, first[i] = i % 7, count[i] = i % 9;
    CHECK(ppd_kv_select(ctx, floats, 50, len.data(), B, 20, 2, 3, ints, 20, nullptr) == PPD_OK);
    CHECK(g_select.size() == 3);
    int at = 0;
    for (const auto& p : g_select) {
        CHECK(p.B <= ppd::kSelectBatch && p.weights == floats + (int64_t)at * 8 * 50 && p.keep == ints + (int64_t)at * 8 * 20);
        for (int i = 0; i < p.B; ++i) CHECK(p.length[i] == len[at + i]);
        at += p.B;
    }
    CHECK(at == B);
    CHECK(ppd_kv_compact(ctx, device, 0, 1, tables, 3, ints, 0, 80, 10, first.data(), count.data(), B, floats, 50, nullptr) == PPD_OK);
    CHECK(g_compact.size() == 6);
    at = 0;
    for (const auto& p : g_compact) {
        CHECK(p.B <= ppd::kCompactBatch && p.keep == ints + (int64_t)at * 80 && p.page_tables == tables + at * 3 && p.weights == floats + (int64_t)at * 8 * 50);
        CHECK(p.weight_layer == (int64_t)B * 8 * 50);
        for (int i = 0; i < p.B; ++i) CHECK(p.first[i] == first[at + i] && p.count[i] == count[at + i]);
        at += p.B;
    }
    CHECK(at == B);
    ppd_destroy(ctx);
}

// The plan is uploaded when the lengths change and not otherwise; another stream waits for the one before; under capture nothing is
// planned; a failed launch leaves nothing behind that counts.
static void streams() {
    ppd_ctx* ctx = make(32, 8, 128);
    int32_t L[2] = {1000, 40}, n[2] = {5, 9};
    hipStream_t a, b;
    hipStreamCreateWithFlags(&a, 0);
    hipStreamCreateWithFlags(&b, 0);
    auto tree = [&](hipStream_t s) { return ppd_tree_attention(ctx, device, device, tables, 80, masks, 1, L, n, 2, 1.f, device, s); };
    auto weighted = [&](hipStream_t s) { return ppd_weighted_attention(ctx, device, device, tables, 64, L, n, 2, 1.f, device, floats, 1005, s); };
    sim.capturing = true;
    CHECK(tree(a) == PPD_ERR_RANGE && attentions() == 0);
    sim.capturing = false;
    CHECK(tree(a) == PPD_OK && a->waiting() == 1);
    CHECK(tree(a) == PPD_OK && a->waiting() == 1);  // the plan is there
    sim.capturing = true;
    CHECK(tree(a) == PPD_OK && a->waiting() == 1);
    sim.capturing = false;
    CHECK(tree(b) == PPD_OK && a->waiting() == 0 && b->waiting() == 0);
    CHECK(weighted(b) == PPD_OK && b->waiting() == 1);  // another list: the keys to weigh
    CHECK(g_weigh.size() == 1 && g_weigh[0].n_weighs + g_weigh[0].n_score_weighs == 8 * (4 + 1));
    b->run();
    const ppd::TreeParams& p = g_weigh[0];
    CHECK(p.n_items > 0 && g_blocks.back().n_items > 0);
    for (int i = 0; i < p.n_items; ++i) CHECK(p.items[i].L == L[p.items[i].seq]);
    for (int i = 0; i < g_blocks.back().n_items; ++i) CHECK(g_blocks.back().items[i].L == L[g_blocks.back().items[i].seq]);
    for (int i = 0; i < p.n_weighs; ++i) CHECK(p.weighs[i].L == L[p.weighs[i].seq]);
    for (int i = 0; i < p.n_score_weighs; ++i) CHECK(p.score_weighs[i].L == L[p.score_weighs[i].seq]);
    L[0] = 1001;
    sim.launch_status = hipErrorLaunchFailure;
    CHECK(tree(b) == PPD_ERR_HIP);
    sim.launch_status = hipSuccess;
    const size_t before = attentions();
    CHECK(tree(b) == PPD_OK && b->waiting() == 1 && attentions() == before + 1);
    // mixed attention on another stream waits as well: both share the words that count an upload's workgroups
    CHECK(ppd_mixed_attention(ctx, device, device, tables, 64, L, n, 2, 1.f, device, a) == PPD_OK && b->waiting() == 0);
    a->run();
    for (int i = 0; i < 20; ++i) {  // lengths that change from step to step, the device running behind
        L[0] += 1;
        CHECK(tree(a) == PPD_OK);
        if (a->waiting() >= 4) a->run(1);
    }
    a->run();
    ppd_destroy(ctx);
    delete a;
    delete b;
}

int main(int, char** argv) {
    const std::string what = argv[1];
    if (what == "refusals") refusals();
    else if (what == "plans") plans();
    else if (what == "batches") batches();
    else if (what == "streams") streams();
    else return 2;
    std::printf("ok\n");
    return 0;
}
