// Host-only checks of ppd_prefix_attention (built and run by tests/test_prefix_host.py): its host code as it is, compiled against the
// stand-in runtime of host_runtime/, whose launches are recorded instead of run.
#include <hip/hip_runtime.h>

#include <pthread.h>

#include <cmath>
#include <cstdio>
#include <limits>
#include <random>
#include <string>
#include <vector>

#include "../../paper_2603_13358_amd/csrc/ppd_api.hip"
#include "../../paper_2603_13358_amd/csrc/ppd_prefix_api.hip"

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

static std::vector<ppd::PrefixParams> g_tiles, g_joins;
static std::vector<ppd::TreeBlockParams> g_blocks;

namespace ppd {
int prepare_mixed_kernels() { return 0; }
int launch_mixed(const KParams&, int, int, void*, bool) { return 0; }
int launch_narrow(const KParams&, int, int, void*, bool) { return 0; }
int launch_mfma_only(const KParams&, int, int, void*) { return 0; }
int launch_stream_only(const KParams&, int, int, void*) { return 0; }
int launch_merge(const MergeParams&, void*) { return 0; }
int launch_kv_append(const uint16_t*, const uint16_t*, void*, const int64_t*, int64_t, int, int, int64_t, int, int64_t, uint32_t*,
                     void*, bool, float, float) { return 0; }
int launch_tree_blocks(const TreeBlockParams& p, int, bool, void*) { g_blocks.push_back(p); return 0; }
int launch_prefix(const PrefixParams& p, int, bool, void*) { g_tiles.push_back(p); return 0; }
int launch_prefix_join(const PrefixParams& p, int, void*) { g_joins.push_back(p); return 0; }
}  // namespace ppd

#define CHECK(x)                                                      \
    do {                                                              \
        if (!(x)) {                                                   \
            std::printf("%s:%d: not so: %s\n", __FILE__, __LINE__, #x); \
            std::fflush(stdout);                                      \
            std::_Exit(1);                                            \
        }                                                             \
    } while (0)

alignas(16) static char device[64];
static const int32_t* const tables = reinterpret_cast<const int32_t*>(device);

static ppd_ctx* make(int hq, int hkv, int dim) {
    const ppd_shape s = {hq, hkv, dim, 16, 4096};
    ppd_ctx* ctx = nullptr;
    CHECK(ppd_create(&s, 0, &ctx) == PPD_OK);
    return ctx;
}

// Every refusal comes before anything is enqueued.
static void refusals() {
    ppd_ctx* ctx = make(32, 8, 128);
    const int32_t S[3] = {0, 64, 80}, L[3] = {100, 90, 80}, n[3] = {5, 1, 2};
    const float nan = std::numeric_limits<float>::quiet_NaN();
    auto call = [&](const void* q, const void* pool, const int32_t* pt, int max_pages, const int32_t* s, const int32_t* l, const int32_t* m, int B, float scale, void* out) {
        return ppd_prefix_attention(ctx, q, pool, pt, max_pages, s, l, m, B, scale, out, nullptr);
    };
    CHECK(call(device, device, tables, 7, S, L, n, 3, 1.f, device) == PPD_OK && g_tiles.size() == 1);
    CHECK(call(device, device, tables, 7, S, L, n, 0, 1.f, device) == PPD_OK);
    CHECK(ppd_prefix_attention(nullptr, device, device, tables, 7, S, L, n, 3, 1.f, device, nullptr) == PPD_ERR_NULL);
    CHECK(call(nullptr, device, tables, 7, S, L, n, 3, 1.f, device) == PPD_ERR_NULL && call(device, nullptr, tables, 7, S, L, n, 3, 1.f, device) == PPD_ERR_NULL);
    CHECK(call(device, device, nullptr, 7, S, L, n, 3, 1.f, device) == PPD_ERR_NULL && call(device, device, tables, 7, nullptr, L, n, 3, 1.f, device) == PPD_ERR_NULL);
    CHECK(call(device, device, tables, 7, S, nullptr, n, 3, 1.f, device) == PPD_ERR_NULL && call(device, device, tables, 7, S, L, nullptr, 3, 1.f, device) == PPD_ERR_NULL);
    CHECK(call(device, device, tables, 7, S, L, n, 3, 1.f, nullptr) == PPD_ERR_NULL);
    CHECK(call(device, device, tables, 7, S, L, n, -1, 1.f, device) == PPD_ERR_RANGE);
    for (float scale : {-1.f, nan, INFINITY}) CHECK(call(device, device, tables, 7, S, L, n, 3, scale, device) == PPD_ERR_RANGE);
    CHECK(call(device + 2, device, tables, 7, S, L, n, 3, 1.f, device) == PPD_ERR_RANGE && call(device, device + 8, tables, 7, S, L, n, 3, 1.f, device) == PPD_ERR_RANGE);
    CHECK(call(device, device, tables, 7, S, L, n, 3, 1.f, device + 4) == PPD_ERR_RANGE);
    CHECK(call(device, device, reinterpret_cast<const int32_t*>(device + 2), 7, S, L, n, 3, 1.f, device) == PPD_ERR_RANGE);
    CHECK(call(device, device, tables, 6, S, L, n, 3, 1.f, device) == PPD_ERR_PAGETABLE);
    for (int i = 0; i < 3; ++i) {
        int32_t s[3] = {0, 64, 80}, l[3] = {100, 90, 80}, m[3] = {5, 1, 2};
        m[i] = 0;
        CHECK(call(device, device, tables, 7, S, L, m, 3, 1.f, device) == PPD_ERR_RANGE);
        l[i] = -1;
        CHECK(call(device, device, tables, 7, S, l, n, 3, 1.f, device) == PPD_ERR_RANGE);
        s[i] = -16;
        CHECK(call(device, device, tables, 7, s, L, n, 3, 1.f, device) == PPD_ERR_RANGE);
        s[i] = i == 0 ? 16 : i == 1 ? 91 : 81;  // more than one of the two has
        CHECK(call(device, device, tables, 7, s, L, n, 3, 1.f, device) == PPD_ERR_RANGE);
    }
    const int32_t far[3] = {INT32_MAX - 2, 90, 80}, many[3] = {INT32_MAX / 2, INT32_MAX / 2, INT32_MAX / 2};
    CHECK(call(device, device, tables, INT32_MAX, S, far, n, 3, 1.f, device) == PPD_ERR_RANGE);
    CHECK(call(device, device, tables, INT32_MAX, S, L, many, 3, 1.f, device) == PPD_ERR_RANGE);
    CHECK(g_tiles.size() == 1 && g_blocks.empty());
    CHECK(std::string(ppd_last_error(ctx)).find("rows") != std::string::npos);
    ppd_destroy(ctx);
}

// Every row meets each of its keys in one tile, the partials lie apart from each other, and the join finds them.
static void check_plan(const ppd_shape& s, const std::vector<int32_t>& shared, const std::vector<int32_t>& L, const std::vector<int32_t>& n, ppd::PrefixPlan& plan) {
    const int B = (int)L.size(), G = s.num_q_heads / s.num_kv_heads, Hkv = s.num_kv_heads, D = s.head_dim;
    CHECK(ppd::build_prefix_plan(s, shared.data(), L.data(), n.data(), B, 2, 256, &plan));
    std::vector<int32_t> row0(B + 1, 0), seq;
    for (int i = 0; i < B; ++i) {
        row0[i + 1] = row0[i] + n[i];
        seq.insert(seq.end(), n[i], i);
    }
    // what two sequences have in common
    auto common = [&](int a, int b) {
        int32_t least = INT32_MAX;
        for (int i = std::min(a, b) + 1; i <= std::max(a, b); ++i) least = std::min(least, shared[i]);
        return least;
    };
    struct Tile { int seq, kvh, grow0, ncols, begin, end, L, total; int64_t off; };
    std::vector<Tile> tiles;
    for (const auto& t : plan.items) {
        CHECK(t.ncols >= 1 && t.ncols <= ppd::kPrefixCols && t.ncols % G == 0);
        CHECK(t.kv_end - t.kv_begin <= ppd::kMaxPrefixChunk && t.kv_begin % 32 == 0);
        tiles.push_back({t.seq, t.kvh, t.grow0, t.ncols, t.kv_begin, t.kv_end, t.L, t.kv_total, t.part_off});
    }
    for (const auto& t : plan.blocks) {
        CHECK(t.nrows >= 1 && t.nrows * G <= ppd::kMfmaCols && t.kv_end - t.kv_begin <= ppd::kMaxTreeBlockChunk && t.kv_begin % 64 == 0);
        tiles.push_back({t.seq, t.kvh, t.grow0, t.nrows * G, t.kv_begin, t.kv_end, t.L + t.row0, t.kv_total, t.part_off});
    }
    std::vector<std::pair<int64_t, int64_t>> ranges;
    std::vector<std::vector<std::pair<int32_t, int32_t>>> keys((size_t)row0[B] * Hkv);  // of every row and head
    for (const Tile& t : tiles) {
        CHECK(t.kvh >= 0 && t.kvh < Hkv && t.seq >= 0 && t.seq < B && t.begin < t.end && t.end <= t.total && t.grow0 >= 0 && t.grow0 + t.ncols / G <= row0[B]);
        for (int r = 0; r < t.ncols / G; ++r) {
            const int i = seq[t.grow0 + r];
            keys[(size_t)(t.grow0 + r) * Hkv + t.kvh].push_back({t.begin, t.end});
            const bool own = t.total == L[i] + n[i] && i == t.seq && t.total > L[i];
            if (own) CHECK(t.L + r == L[i] + (t.grow0 + r - row0[i]));
            else CHECK(t.L >= t.total && t.end <= L[i] && t.end <= L[t.seq] && (i == t.seq || t.end <= common(i, t.seq)));
        }
        if (t.off >= 0) ranges.push_back({t.off, t.off + (int64_t)t.ncols * (D + 2)});
    }
    std::sort(ranges.begin(), ranges.end());
    int64_t at = 0;
    for (const auto& r : ranges) {
        CHECK(r.first == at);
        at = r.second;
    }
    CHECK(at == plan.partial_floats);
    for (size_t k = 0; k < keys.size(); ++k) {
        std::sort(keys[k].begin(), keys[k].end());
        int32_t to = 0;
        for (const auto& r : keys[k]) {
            CHECK(r.first == to);
            to = r.second;
        }
        const int row = (int)(k / Hkv), i = seq[row];
        CHECK(to > L[i] + row - row0[i] && to <= L[i] + n[i]);  // itself among them
    }
    // the join: of each row the same partials that its tiles write
    std::vector<int> joined(row0[B], 0);
    std::vector<std::vector<int64_t>> found((size_t)row0[B] * Hkv), want = found;
    for (const auto& u : plan.units) {
        const size_t source0 = (&u - plan.units.data()) * (size_t)plan.source_stride;
        CHECK(u.nrows * G <= plan.join_cols && u.nsources >= 1 && u.nsources <= plan.source_stride && plan.sources.size() == plan.units.size() * plan.source_stride);
        for (int r = u.grow0; r < u.grow0 + u.nrows; ++r) {
            CHECK(r < row0[B] && !joined[r]++);
            for (int h = 0; h < Hkv; ++h)
                for (int x = 0; x < u.nsources; ++x) {
                    const ppd::JoinSource& src = plan.sources[source0 + x];
                    for (int p = 0; p < src.nsplit; ++p)
                        found[(size_t)r * Hkv + h].push_back(src.part_off + ((int64_t)h * src.nsplit + p) * src.ncols * (D + 2) + (int64_t)(src.col0 + (r - u.grow0) * G) * D);
                    CHECK(src.col0 + u.nrows * G <= src.ncols);
                }
        }
    }
    for (const Tile& t : tiles)
        for (int r = 0; r < t.ncols / G; ++r) {
            if (t.off >= 0) want[(size_t)(t.grow0 + r) * Hkv + t.kvh].push_back(t.off + (int64_t)r * G * D);
            else CHECK(!joined[t.grow0 + r]);
        }
    for (size_t k = 0; k < found.size(); ++k) {
        std::sort(found[k].begin(), found[k].end());
        std::sort(want[k].begin(), want[k].end());
        CHECK(found[k] == want[k]);
    }
}

static void plans() {
    std::mt19937 r(5);
    auto in = [&](int lo, int hi) { return (int)(lo + r() % (unsigned)(hi - lo + 1)); };
    int64_t wide = 0, joins = 0, saved = 0;
    for (int round = 0; round < 400; ++round) {
        const int G = in(1, 8), Hkv = in(1, 4);
        const ppd_shape s = {G * Hkv, Hkv, in(0, 1) ? 64 : 128, 16, 1 << 20};
        const int B = in(1, 40), longest = in(0, 2) ? 20000 : 2000, most_new = in(0, 2) ? 3 : 200;
        std::vector<int32_t> shared(B, 0), L(B), n(B);
        for (int i = 0; i < B; ++i) {
            L[i] = in(0, longest);
            n[i] = in(1, most_new);
            if (i == 0) continue;
            const int both = std::min(L[i], L[i - 1]);
            shared[i] = in(0, 3) == 0 ? in(0, both) : std::min(both, shared[i - 1] + (in(0, 2) ? 0 : in(-300, 300)));
            if (in(0, 2)) shared[i] = std::min(both, 640 * in(0, 3));
            shared[i] = std::max(0, shared[i]);
        }
        if (in(0, 1)) {  // one prompt in front of all, and of some more than that
            const int prompt = in(100, longest);
            for (int i = 0; i < B; ++i) {
                L[i] = prompt + in(0, 3000);
                if (i > 0) shared[i] = in(0, 1) ? prompt : in(prompt, std::min(L[i], L[i - 1]));
            }
        }
        ppd::PrefixPlan plan;
        check_plan(s, shared, L, n, plan);
        wide += (int64_t)plan.blocks.size();
        joins += (int64_t)plan.units.size();
        saved += plan.keys_read < plan.keys_alone;
    }
    CHECK(wide > 1000 && joins > 1000 && saved > 100);
    // chains of more levels than are kept, both ways, and a batch too large for one launch
    for (int down = 0; down < 2; ++down) {
        const int B = 3000;
        std::vector<int32_t> shared(B, 0), L(B), n(B, 1);
        for (int i = 0; i < B; ++i) L[i] = 64 * (down ? B - i : i + 1);
        for (int i = 1; i < B; ++i) shared[i] = std::min(L[i], L[i - 1]);
        ppd::PrefixPlan plan;
        CHECK(ppd::build_prefix_plan({8, 1, 64, 16, 1 << 20}, shared.data(), L.data(), n.data(), B, 2, 256, &plan));
        for (const auto& u : plan.units) CHECK(u.nsources <= ppd::kMaxNested + 1);
    }
    {
        const int B = 70000;
        std::vector<int32_t> shared(B, 0), L(B, 100), n(B, 1);
        ppd::PrefixPlan plan;
        CHECK(!ppd::build_prefix_plan({64, 64, 64, 16, 1 << 20}, shared.data(), L.data(), n.data(), B, 2, 256, &plan));
        for (int i = 1; i < B; ++i) shared[i] = 64;
        CHECK(!ppd::build_prefix_plan({64, 64, 64, 16, 1 << 20}, shared.data(), L.data(), n.data(), B, 2, 256, &plan));
    }
    {
        std::vector<int32_t> shared = {0, ppd::kMaxTreeTokens - 9}, L = {ppd::kMaxTreeTokens - 5, ppd::kMaxTreeTokens - 9}, n = {5, 9};
        ppd::PrefixPlan plan;
        check_plan({8, 1, 128, 16, 1 << 20}, shared, L, n, plan);
    }
}

// Every sequence shares 64 tokens more with its neighbour than the one before: as many lengths in common as sequences, few of them worth a
// tile.  Planned by a thread with 256 KB of stack.
static void* staircase_on(void* arg) {
    const int B = *static_cast<int*>(arg);
    std::vector<int32_t> shared(B), L(B), n(B, 1);
    for (int i = 0; i < B; ++i) L[i] = 64 * (i + 1), shared[i] = 64 * i;
    ppd::PrefixPlan plan;
    CHECK(ppd::build_prefix_plan({32, 8, 128, 16, 1 << 20}, shared.data(), L.data(), n.data(), B, 2, 256, &plan));
    CHECK(plan.keys_read < plan.keys_alone && plan.units.size() <= (size_t)B);
    if (B <= 700) check_plan({32, 8, 128, 16, 1 << 20}, shared, L, n, plan);
    return nullptr;
}
static void staircase() {
    for (int B : {700, 8000}) {
        pthread_attr_t attr;
        pthread_t thread;
        CHECK(pthread_attr_init(&attr) == 0 && pthread_attr_setstacksize(&attr, 256 << 10) == 0);
        CHECK(pthread_create(&thread, &attr, staircase_on, &B) == 0 && pthread_join(thread, nullptr) == 0);
        pthread_attr_destroy(&attr);
    }
}

// Which calls plan anew, what a capture refuses, and that staging buffers are waited for.
static void streams() {
    ppd_ctx* ctx = make(8, 2, 64);
    SimStream a, b;
    int32_t S[4] = {0, 64000, 64000, 64000}, L[4] = {64030, 64040, 64050, 64060}, n[4] = {1, 1, 1, 1};
    auto call = [&](SimStream* st) { return ppd_prefix_attention(ctx, device, device, tables, 4100, S, L, n, 4, 1.f, device, st); };
    sim.capturing = true;
    CHECK(call(&a) == PPD_ERR_RANGE && !ctx->prefix && g_tiles.empty());
    sim.capturing = false;
    CHECK(call(&a) == PPD_OK && a.waiting() == 1 && g_tiles.size() == 1 && g_joins.size() == 1);  // the upload
    CHECK(call(&a) == PPD_OK && a.waiting() == 1 && g_tiles.size() == 2);
    sim.capturing = true;
    CHECK(call(&a) == PPD_OK && a.waiting() == 1);
    S[2] = 32000;
    CHECK(call(&a) == PPD_ERR_RANGE && a.waiting() == 1 && g_tiles.size() == 3);
    S[2] = 64000;
    sim.capturing = false;
    CHECK(call(&b) == PPD_OK && a.waiting() == 0);  // another stream: the first one's work has ended
    CHECK(b.waiting() == 0 && g_tiles.size() == 4);
    for (int i = 0; i < 3 * kStagingSlots; ++i) {
        L[0] = 64031 + i;
        if (b.waiting() == kStagingSlots) b.run(1);
        CHECK(call(&b) == PPD_OK);
    }
    b.run();
    a.run();
    const auto* items = reinterpret_cast<const ppd::PrefixItem*>(static_cast<PrefixState*>(ctx->prefix)->d_plan);  // what is on the device is the last plan
    const ppd::PrefixPlan& plan = static_cast<PrefixState*>(ctx->prefix)->plan;
    CHECK(std::memcmp(items, plan.items.data(), plan.items.size() * sizeof(ppd::PrefixItem)) == 0);
    ppd_destroy(ctx);
}

int main(int argc, char** argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "refusals") refusals();
    else if (what == "plans") plans();
    else if (what == "streams") streams();
    else if (what == "staircase") staircase();
    else return 2;
    std::printf("ok\n");
    return 0;
}
