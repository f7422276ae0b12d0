// Host-only checks of what the drafting and eviction calls leave behind for the calls and graphs after them (built and run by
// tests/test_ops_repeat.py), with the recorded launches of ops_host.cpp and allocations that fail while a stream is captured, as
// the runtime's do.
#include <hip/hip_runtime.h>

static int g_captured_allocations = 0;
static size_t g_largest = SIZE_MAX;  // of an allocation; larger ones fail
template <class T>
static hipError_t allocate_unless_captured(T** p, size_t n) {
    if (sim.capturing) {
        ++g_captured_allocations;
        return sim.pending = hipErrorInvalidValue;
    }
    if (n > g_largest) return sim.pending = hipErrorInvalidValue;
    *p = static_cast<T*>(std::malloc(n));
    return hipSuccess;
}
#define hipMalloc(p, n) allocate_unless_captured((p), (n))
#define hipHostMalloc(p, n, flags) allocate_unless_captured((p), (n))
#define main ops_host_main
#include "ops_host.cpp"
#undef main

// A context's first call of each kind under capture is refused before anything is allocated, and the next eager one succeeds.
static void first_call_under_capture() {
    const int32_t L[2] = {1000, 40}, n[2] = {5, 9}, rows[2] = {40000, 100};
    auto call = [&](ppd_ctx* ctx, int kind) {
        if (kind == 0) return ppd_tree_attention(ctx, device, device, tables, 80, masks, 1, L, n, 2, 1.f, device, nullptr);
        if (kind == 1) return ppd_weighted_attention(ctx, device, device, tables, 80, L, n, 2, 1.f, device, floats, 1005, nullptr);
        return ppd_kv_select(ctx, floats, 40000, rows, 2, 50, 2, 3, ints, 50, nullptr);
    };
    for (int kind = 0; kind < 3; ++kind) {
        ppd_ctx* ctx = make(32, 8, 128);
        sim.capturing = true;
        CHECK(call(ctx, kind) == PPD_ERR_RANGE && std::string(ppd_last_error(ctx)).find("capture") != std::string::npos);
        CHECK(g_captured_allocations == 0 && attentions() == 0 && g_tree.empty() && g_weigh.empty() && g_select.empty());
        sim.capturing = false;
        CHECK(call(ctx, kind) == PPD_OK);
        const size_t launches = g_tree.size() + g_blocks.size() + g_weigh.size() + g_select.size();
        sim.capturing = true;
        CHECK(call(ctx, kind) == PPD_OK && g_tree.size() + g_blocks.size() + g_weigh.size() + g_select.size() > launches);
        sim.capturing = false;
        CHECK(g_captured_allocations == 0);
        ppd_destroy(ctx);
        g_tree.clear(), g_blocks.clear(), g_weigh.clear(), g_select.clear();
    }
    // rows longer than those of the eager call before need more
    ppd_ctx* ctx = make(32, 8, 128);
    const int32_t longer[2] = {400000, 100};
    CHECK(call(ctx, 2) == PPD_OK);
    sim.capturing = true;
    CHECK(ppd_kv_select(ctx, floats, 400000, longer, 2, 50, 2, 3, ints, 50, nullptr) == PPD_ERR_RANGE && g_captured_allocations == 0);
    CHECK(call(ctx, 2) == PPD_OK);
    sim.capturing = false;
    ppd_destroy(ctx);
}

// Tree and weighted attention, on pages of either format, keep a plan each: calls of one leave the others' plans as they are, also with
// the same lengths, so that a graph of one can be replayed after calls of the other and one graph can hold both.
static void kinds() {
    ppd_ctx* ctx = make(32, 8, 128);
    const int32_t L[3] = {3000, 40, 9000}, n[3] = {5, 9, 1}, other[3] = {3000, 41, 9000};
    hipStream_t s;
    hipStreamCreateWithFlags(&s, 0);
    auto tree = [&](const int32_t* l) { return ppd_tree_attention(ctx, device, device, tables, 600, masks, 1, l, n, 3, 1.f, device, s); };
    auto weighted = [&](const int32_t* l) { return ppd_weighted_attention(ctx, device, device, tables, 600, l, n, 3, 1.f, device, floats, 9001, s); };
    struct Plan {  // what a graph reads, and what was there when it was captured
        ppd::TreeParams p;
        std::vector<ppd::TreeItem> items;
        std::vector<ppd::TreeGroup> groups;
        std::vector<ppd::WeighItem> weighs;
        bool intact() const {
            return std::memcmp(items.data(), p.items, items.size() * sizeof items[0]) == 0 && std::memcmp(groups.data(), p.groups, groups.size() * sizeof groups[0]) == 0 &&
                   std::memcmp(weighs.data(), p.score_weighs, weighs.size() * sizeof weighs[0]) == 0;
        }
    };
    auto last = [&] {
        const ppd::TreeParams p = g_tree.back();
        return Plan{p, {p.items, p.items + p.n_items}, {p.groups, p.groups + p.n_groups}, {p.score_weighs, p.score_weighs + p.n_score_weighs}};
    };
    auto captured = [&](auto call) {
        sim.capturing = true;
        const ppd_status st = call(L);
        sim.capturing = false;
        return st == PPD_OK && s->waiting() == 0;
    };
    CHECK(weighted(L) == PPD_OK && s->waiting() == 1);
    s->run();
    const Plan w = last();
    CHECK(w.items.size() > 0 && w.groups.size() > 0 && w.weighs.size() > 0);
    CHECK(tree(L) == PPD_OK && s->waiting() == 1);
    s->run();
    const Plan t = last();
    CHECK(t.p.items != w.p.items && w.intact());
    CHECK(captured(weighted) && captured(tree) && captured(weighted));
    CHECK(tree(other) == PPD_OK && s->waiting() == 1);
    s->run();
    CHECK(w.intact() && captured(weighted));
    CHECK(ppd_set_kv_format(ctx, PPD_KV_FP8_E4M3, 1.f, 1.f) == PPD_OK);
    CHECK(weighted(L) == PPD_OK && s->waiting() == 1);
    s->run();
    CHECK(w.intact() && captured(weighted));
    CHECK(ppd_set_kv_format(ctx, PPD_KV_BF16, 1.f, 1.f) == PPD_OK);
    CHECK(captured(weighted) && g_tree.back().items == w.p.items);
    // a workspace that could not grow is gone for all of them
    const int32_t far[3] = {300000, 40, 300000};
    g_largest = 1 << 20;
    CHECK(ppd_tree_attention(ctx, device, device, tables, 20000, masks, 1, far, n, 3, 1.f, device, s) == PPD_ERR_WORKSPACE);
    g_largest = SIZE_MAX;
    CHECK(weighted(L) == PPD_OK && s->waiting() == 1 && g_tree.back().partials != nullptr);
    s->run();
    ppd_destroy(ctx);
    delete s;
}

// The longest sequences whose key numbers, rounded up to whole tiles, still fit 32 bits are planned whole; longer ones are refused.
static void longest() {
    const ppd_shape s = {8, 1, 64, 16, 1 << 20};
    for (const int32_t rows : {1, 4, 5, 32}) {
        const int32_t total = ppd::kMaxTreeTokens, L = total - rows;
        ppd::TreePlan p;
        CHECK(ppd::build_tree_plan(s, &L, &rows, 1, false, 1, 256, &p));
        CHECK(p.items.empty() == (rows > 4) && p.blocks.empty() == (rows <= 4));
        std::map<int32_t, int32_t> range;  // begin -> end
        for (const auto& it : p.items) CHECK(range.emplace(it.kv_begin, it.kv_end).second);
        for (const auto& it : p.blocks) CHECK(range.emplace(it.kv_begin, it.kv_end).second);
        int32_t at = 0;
        for (const auto& [b, e] : range) {
            CHECK(b == at && e > b);
            at = e;
        }
        CHECK(at == total && p.groups.size() == 1 && p.groups[0].nsplit == (int)range.size());
    }
    ppd_ctx* ctx = nullptr;
    CHECK(ppd_create(&s, 0, &ctx) == PPD_OK);
    for (const int32_t rows : {1, 4, 5, 32}) {
        for (const int32_t more : {1, 4096, 8192, 12000, 16384 - 8}) {
            if (more > INT32_MAX - ppd::kMaxTreeTokens) continue;
            const int32_t L = ppd::kMaxTreeTokens - rows + more;
            CHECK(ppd_tree_attention(ctx, device, device, tables, INT32_MAX, masks, 1, &L, &rows, 1, 1.f, device, nullptr) == PPD_ERR_RANGE);
            CHECK(ppd_weighted_attention(ctx, device, device, tables, INT32_MAX, &L, &rows, 1, 1.f, device, floats, INT32_MAX, nullptr) == PPD_ERR_RANGE);
        }
    }
    CHECK(g_tree.empty() && g_blocks.empty());
    ppd_destroy(ctx);
}

// Ranges that are split and several row blocks of a sequence at once: every block's groups name its own columns, so that the join
// leaves the references of all rows.  (The lengths are those of the GPU's test of it.)
static void split_blocks() {
    struct { int32_t hq, hkv, dim, eb; std::vector<int32_t> L, n; } cases[] = {
        {8, 1, 128, 2, {9000}, {70}}, {10, 2, 64, 1, {5000, 3}, {130, 60}}, {2, 1, 64, 2, {3000, 200, 2500}, {300, 1, 290}}};
    for (const auto& c : cases) {
        const ppd_shape s = {c.hq, c.hkv, c.dim, 16, 1 << 16};
        const int G = c.hq / c.hkv;
        ppd::TreePlan p;
        CHECK(ppd::build_tree_plan(s, c.L.data(), c.n.data(), (int)c.L.size(), true, c.eb, 256, &p));
        std::set<std::pair<int, int>> rows;  // (row, KV head) of split ranges of row blocks
        bool behind_the_first = false;
        for (const auto& g : p.groups) {
            if (g.ncols <= ppd::kTreeCols && g.col0 == 0) continue;
            behind_the_first |= g.col0 > 0 && g.nsplit > 1;
            CHECK(g.col0 % G == 0 && g.ncols % G == 0);
            for (int col = g.col0; col < g.col0 + g.ncols; col += G) CHECK(rows.emplace(g.grow0 + col / G, g.kvh).second);
        }
        CHECK(behind_the_first && p.weighs.size() > 0);
        int split = 0;
        for (size_t i = 0, at = 0; i < c.L.size(); at += c.n[i++])
            if (rows.count({(int)at, 0}))
                for (int j = 0; j < c.n[i]; ++j)
                    for (int h = 0; h < c.hkv; ++h) CHECK(rows.count({(int)at + j, h}) && ++split);
        CHECK(split == (int)rows.size());
    }
}

int main(int, char** argv) {
    const std::string what = argv[1];
    if (what == "first_call_under_capture") first_call_under_capture();
    else if (what == "kinds") kinds();
    else if (what == "longest") longest();
    else if (what == "split_blocks") split_blocks();
    else return 2;
    std::printf("ok\n");
    return 0;
}
