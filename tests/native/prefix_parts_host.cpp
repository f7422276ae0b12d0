// Host-only checks of prefix attention over batches whose partials do not fit the workspace at once (built and run by tests/test_partials_host.py): the
// host code as it is, with a device that has so much memory as the test says.
#define main prefix_host_main
#include <hip/hip_runtime.h>

static size_t g_memory = SIZE_MAX;  // bytes of one allocation at most
template <class T>
static hipError_t limited_malloc(T** p, size_t n) {
    if (n > g_memory) return sim.pending = hipErrorInvalidValue;
    return hipMalloc(p, n);
}
#define hipMalloc limited_malloc
#include "prefix_host.cpp"
#undef main

struct Lengths {
    std::vector<int32_t> shared, L, n;
    Lengths(int B, int common, int own, int fresh) : shared(B, common), L(B), n(B, fresh) {
        shared[0] = 0;
        for (int i = 0; i < B; ++i) L[i] = common + own + 3 * (i % 50);
    }
    int B() const { return (int)L.size(); }
};

// Every part is the plan of its sequences, and its partials fit unless it is one sequence; returns how many there are.
static size_t check_parts(const ppd_shape& s, const Lengths& x, int64_t most, ppd::PrefixPlan& plan) {
    CHECK(ppd::build_prefix_parts(s, x.shared.data(), x.L.data(), x.n.data(), x.B(), 2, 256, most, &plan));
    int64_t item = 0, block = 0, unit = 0, source = 0, largest = 0;
    int32_t lo = 0, row0 = 0;
    for (const ppd::PrefixPart& part : plan.parts) {
        CHECK(part.item0 == item && part.block0 == block && part.unit0 == unit && part.source0 == source);
        item += part.n_items, block += part.n_blocks, unit += part.n_units, source += (int64_t)part.n_units * part.source_stride;
        CHECK(item <= (int64_t)plan.items.size() && block <= (int64_t)plan.blocks.size() && unit <= (int64_t)plan.units.size() && source <= (int64_t)plan.sources.size());
        int32_t hi = lo;  // behind the last sequence that has a tile in it
        for (int64_t i = part.item0; i < item; ++i) hi = std::max(hi, plan.items[i].seq + 1);
        for (int64_t i = part.block0; i < block; ++i) hi = std::max(hi, plan.blocks[i].seq + 1);
        CHECK(hi > lo);
        Lengths sub(1, 0, 0, 0);
        sub.shared.assign(x.shared.begin() + lo, x.shared.begin() + hi);
        sub.L.assign(x.L.begin() + lo, x.L.begin() + hi);
        sub.n.assign(x.n.begin() + lo, x.n.begin() + hi);
        sub.shared[0] = 0;
        ppd::PrefixPlan one;
        check_plan(s, sub.shared, sub.L, sub.n, one);
        CHECK(one.partial_floats <= most || hi - lo == 1);
        CHECK(part.n_items == (int)one.items.size() && part.n_blocks == (int)one.blocks.size() && part.n_units == (int)one.units.size());
        CHECK(part.join_cols == one.join_cols && part.source_stride == one.source_stride);
        largest = std::max(largest, one.partial_floats);
        for (size_t i = 0; i < one.items.size(); ++i) {
            ppd::PrefixItem t = plan.items[part.item0 + i];
            t.seq -= lo, t.grow0 -= row0;
            CHECK(std::memcmp(&t, &one.items[i], sizeof t) == 0);
        }
        for (size_t i = 0; i < one.blocks.size(); ++i) {
            ppd_work_item t = plan.blocks[part.block0 + i];
            t.seq -= lo, t.grow0 -= row0;
            CHECK(std::memcmp(&t, &one.blocks[i], sizeof t) == 0);
        }
        for (size_t i = 0; i < one.units.size(); ++i) {
            ppd::JoinUnit t = plan.units[part.unit0 + i];
            t.grow0 -= row0;
            CHECK(std::memcmp(&t, &one.units[i], sizeof t) == 0);
        }
        for (size_t i = 0; i < one.sources.size(); ++i) CHECK(std::memcmp(&plan.sources[part.source0 + i], &one.sources[i], sizeof(ppd::JoinSource)) == 0);
        for (int32_t rows : sub.n) row0 += rows;
        lo = hi;
    }
    CHECK(lo == x.B() && plan.partial_floats == largest);
    CHECK(item == (int64_t)plan.items.size() && block == (int64_t)plan.blocks.size() && unit == (int64_t)plan.units.size() && source == (int64_t)plan.sources.size());
    return plan.parts.size();
}

static const ppd_shape kWide = {64, 8, 128, 16, 4096};

// What a batch asks for stays below the bound, however much its rows share and with whom.
static void bound() {
    ppd::PrefixPlan plan;
    for (int fresh : {16, 100, 200}) {
        const Lengths x(fresh == 16 ? 500 : 120, 30016, 200, fresh);
        PrefixState* t = nullptr;
        ppd_ctx* ctx = make(64, 8, 128);
        const size_t tiles = g_tiles.size() + g_blocks.size();
        CHECK(ppd_prefix_attention(ctx, device, device, tables, 4096, x.shared.data(), x.L.data(), x.n.data(), x.B(), 1.f, device, nullptr) == PPD_OK);
        t = static_cast<PrefixState*>(ctx->prefix);
        CHECK(t->d_partials_bytes <= size_t(5) << 28);  // 1 GiB, and the quarter that a buffer grows by on top
        CHECK(g_tiles.size() + g_blocks.size() - tiles == t->plan.parts.size());
        ppd_destroy(ctx);
    }
    std::mt19937 r(9);
    auto in = [&](int lo, int hi) { return (int)(lo + r() % (unsigned)(hi - lo + 1)); };
    size_t parts = 0;
    for (int round = 0; round < 60; ++round) {
        const int G = in(1, 8), Hkv = in(1, 3), B = in(1, 40);
        Lengths x(B, 0, 0, 1);
        const int prompt = in(0, 6000);
        for (int i = 0; i < B; ++i) {
            x.L[i] = prompt + in(0, 3000), x.n[i] = in(0, 2) ? in(1, 4) : in(1, 90);
            if (i > 0) x.shared[i] = in(0, 3) ? in(0, std::min(x.L[i], x.L[i - 1])) : std::min(x.L[i], x.L[i - 1]);
        }
        parts += check_parts({G * Hkv, Hkv, in(0, 1) ? 64 : 128, 16, 4096}, x, 1 << in(8, 18), plan);
    }
    CHECK(parts > 200);
    CHECK(check_parts(kWide, Lengths(64, 8000, 60, 1), ppd::kMostPartialFloats, plan) == 1);
}

// Where an allocation fails the batch runs in more parts, and only what no part can do without fails.
static void memory() {
    ppd_ctx* ctx = make(64, 8, 128);
    const Lengths x(64, 30016, 200, 8);
    auto call = [&](const Lengths& y) { return ppd_prefix_attention(ctx, device, device, tables, 4096, y.shared.data(), y.L.data(), y.n.data(), y.B(), 1.f, device, nullptr); };
    CHECK(call(x) == PPD_OK);
    const PrefixState* t = static_cast<PrefixState*>(ctx->prefix);
    CHECK(t->plan.parts.size() == 1 && t->d_partials_bytes > (24u << 20));
    ppd_destroy(ctx);
    ctx = make(64, 8, 128);
    g_memory = 24u << 20;
    const size_t tiles = g_tiles.size(), joins = g_joins.size();
    CHECK(call(x) == PPD_OK && std::string(ppd_last_error(ctx)).empty());
    t = static_cast<PrefixState*>(ctx->prefix);
    CHECK(t->plan.parts.size() > 1 && t->d_partials_bytes <= g_memory && g_tiles.size() - tiles == t->plan.parts.size() && g_joins.size() - joins == t->plan.parts.size());
    for (size_t i = 0; i < t->plan.parts.size(); ++i) {
        const ppd::PrefixParams& p = g_tiles[tiles + i];
        const ppd::PrefixPart& part = t->plan.parts[i];
        const char* d_plan = static_cast<const char*>(t->d_plan);
        const PlanLayout at(t->plan);
        CHECK(p.items == reinterpret_cast<const ppd::PrefixItem*>(d_plan) + part.item0 && p.n_items == part.n_items);
        CHECK(p.units == reinterpret_cast<const ppd::JoinUnit*>(d_plan + at.units) + part.unit0 && p.n_units == part.n_units);
        CHECK(p.sources == reinterpret_cast<const ppd::JoinSource*>(d_plan + at.sources) + part.source0 && p.source_stride == part.source_stride && p.join_cols == part.join_cols);
    }
    CHECK(call(x) == PPD_OK && g_tiles.size() - tiles == 2 * t->plan.parts.size());  // the plan is there
    const Lengths y(64, 30016, 230, 8);
    CHECK(call(y) == PPD_OK && t->d_partials_bytes <= g_memory);
    const Lengths z(2, 64000, 0, 100);
    g_memory = 0;
    CHECK(call(z) == PPD_ERR_WORKSPACE && !std::string(ppd_last_error(ctx)).empty());
    g_memory = SIZE_MAX;
    CHECK(call(z) == PPD_OK);
    ppd_destroy(ctx);
}

int main(int argc, char** argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "bound") bound();
    else if (what == "memory") memory();
    else return 2;
    std::printf("ok\n");
    return 0;
}
