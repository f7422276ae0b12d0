// Host-only checks of the rotation's entry points (built and run by tests/test_positions_host.py): their host code as it is, compiled
// against the stand-in runtime of host_runtime/, whose launches are recorded instead of run.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>
#include <limits>
#include <string>
#include <vector>

#include "../../paper_2603_13358_amd/csrc/ppd_api.hip"
#include "../../paper_2603_13358_amd/csrc/ppd_rope_api.hip"

std::function<void()> sim_bind(const void*, void**) { std::abort(); }

static std::vector<ppd::RopeParams> g_rope;
static std::vector<ppd::RotatedAppendParams> g_append;

namespace ppd {
int prepare_mixed_kernels() { return 0; }
int launch_mixed(const KParams&, int, int, void*, bool) { return 0; }
int launch_narrow(const KParams&, int, int, void*, bool) { return 0; }
int launch_mfma_only(const KParams&, int, int, void*) { return 0; }
int launch_stream_only(const KParams&, int, int, void*) { return 0; }
int launch_merge(const MergeParams&, void*) { return 0; }
int launch_kv_append(const uint16_t*, const uint16_t*, void*, const int64_t*, int64_t, int, int, int64_t, int, int64_t, uint32_t*,
                     void*, bool, float, float) { return 0; }
int launch_rope(const RopeParams& p, int, void*) { g_rope.push_back(p); return 0; }
int launch_rotated_append(const RotatedAppendParams& p, int, bool, void*) { g_append.push_back(p); return 0; }
}  // namespace ppd

#define CHECK(x)                                                      \
    do {                                                              \
        if (!(x)) {                                                   \
            std::printf("%s:%d: not so: %s\n", __FILE__, __LINE__, #x); \
            std::fflush(stdout);                                      \
            std::_Exit(1);                                            \
        }                                                             \
    } while (0)

static const double kNan = std::numeric_limits<double>::quiet_NaN();
static char* at(uint64_t a) { return reinterpret_cast<char*>(a); }
static int64_t* ints(uint64_t a) { return reinterpret_cast<int64_t*>(a); }

static ppd_ctx* make(int hq, int hkv, int dim) {
    const ppd_shape s = {hq, hkv, dim, 16, 64};
    ppd_ctx* ctx = nullptr;
    CHECK(ppd_create(&s, 0, &ctx) == PPD_OK);
    return ctx;
}

static void frequencies() {
    double f[64];
    CHECK(ppd_rope_frequencies(128, 1e4, PPD_ROPE_SCALE_NONE, kNan, kNan, kNan, kNan, f) == PPD_OK);  // what is not used is ignored
    for (int i = 0; i < 64; ++i) CHECK(std::fabs(f[i] / std::exp(-2.0 * i / 128 * std::log(1e4)) - 1) < 1e-14);
    CHECK(ppd_rope_frequencies(64, 1e4, PPD_ROPE_SCALE_LINEAR, 4, 0, 0, 0, f) == PPD_OK && f[0] == 0.25);
    CHECK(ppd_rope_frequencies(64, 1e4, PPD_ROPE_SCALE_BASE, 4, 0, 0, 0, f) == PPD_OK && f[0] == 1.0);
    CHECK(std::fabs(f[31] * 4 / std::exp(-62.0 / 64 * std::log(1e4)) - 1) < 1e-12);  // the slowest pair is stretched by the factor
    CHECK(ppd_rope_frequencies(64, 1e4, PPD_ROPE_SCALE_BY_PARTS, 8, 2048, 1, 32, f) == PPD_OK);
    for (int i = 0; i < 32; ++i) {
        const double plain = std::exp(-2.0 * i / 64 * std::log(1e4)), turns = 2048 * plain / (2 * 3.14159265358979323846);
        const double want = turns >= 32 ? plain : turns <= 1 ? plain / 8 : plain * ((turns - 1) / 31 + (32 - turns) / 31 / 8);
        CHECK(std::fabs(f[i] / want - 1) < 1e-12);
    }
    f[0] = -5;
    CHECK(ppd_rope_frequencies(64, 1e4, 0, 1, 0, 0, 0, nullptr) == PPD_ERR_NULL);
    for (int dim : {-2, 0, 1, 63, 130}) CHECK(ppd_rope_frequencies(dim, 1e4, 0, 1, 0, 0, 0, f) == PPD_ERR_SHAPE);
    for (double base : {0.0, -1.0, kNan, (double)INFINITY}) CHECK(ppd_rope_frequencies(64, base, 0, 1, 0, 0, 0, f) == PPD_ERR_RANGE);
    for (int scaling : {-1, 4}) CHECK(ppd_rope_frequencies(64, 1e4, scaling, 1, 0, 0, 0, f) == PPD_ERR_RANGE);
    for (int scaling : {1, 2, 3})
        for (double factor : {0.0, -1.0, kNan, (double)INFINITY}) CHECK(ppd_rope_frequencies(64, 1e4, scaling, factor, 100, 1, 32, f) == PPD_ERR_RANGE);
    CHECK(ppd_rope_frequencies(2, 1e4, PPD_ROPE_SCALE_BASE, 2, 0, 0, 0, f) == PPD_ERR_SHAPE);
    CHECK(ppd_rope_frequencies(64, 1e4, 3, 2, 0, 1, 32, f) == PPD_ERR_RANGE);
    CHECK(ppd_rope_frequencies(64, 1e4, 3, 2, 100, 32, 32, f) == PPD_ERR_RANGE);
    CHECK(ppd_rope_frequencies(64, 1e4, 3, 2, 100, -1, 32, f) == PPD_ERR_RANGE);
    CHECK(ppd_rope_frequencies(64, 1e4, 3, 2, 100, kNan, 32, f) == PPD_ERR_RANGE);
    CHECK(ppd_rope_frequencies(128, 1e-308, 0, 1, 0, 0, 0, f) == PPD_OK || f[0] == -5);
    CHECK(ppd_rope_frequencies(64, 1e4, 1, 1e-320, 0, 0, 0, f) == PPD_ERR_RANGE);  // 1 / 1e-320 is infinite
    CHECK(std::string(ppd_last_error(nullptr)).find("frequency") != std::string::npos);
}

static void settings() {
    ppd_ctx* ctx = make(8, 2, 64);
    double f[64] = {1, 0.5, -0.25, 0, 6.283185307179586476925286766559};
    CHECK(ppd_set_rope(nullptr, f, 8, 0, 1.f) == PPD_ERR_NULL);
    CHECK(ppd_set_rope(ctx, nullptr, 8, 0, 1.f) == PPD_ERR_NULL);
    for (int dim : {0, 1, 7, 66, -8}) CHECK(ppd_set_rope(ctx, f, dim, 0, 1.f) == PPD_ERR_SHAPE);
    for (int layout : {-1, 2}) CHECK(ppd_set_rope(ctx, f, 8, layout, 1.f) == PPD_ERR_RANGE);
    CHECK(ppd_set_rope(ctx, f, 8, 0, (float)kNan) == PPD_ERR_RANGE && ppd_set_rope(ctx, f, 8, 0, INFINITY) == PPD_ERR_RANGE);
    CHECK(ctx->rotation.rotary_dim == 0);
    CHECK(ppd_set_rope(ctx, f, 10, 1, 2.f) == PPD_OK);
    const ppd::Rotation& r = ctx->rotation;
    CHECK(r.rotary_dim == 10 && r.interleaved == 1 && r.amplitude == 2.f && r.turns[3] == 0);
    CHECK(std::fabs((double)r.turns[0] / 18446744073709551616.0 * 2 * 3.14159265358979323846 - 1) < 1e-15);
    CHECK(r.turns[1] * 2 - r.turns[0] + 1 <= 2 && r.turns[1] + 2 * r.turns[2] + 2 <= 4);  // a half, and minus a quarter, to the last unit
    CHECK((int64_t)r.turns[4] < 4096 && (int64_t)r.turns[4] > -4096);  // a whole turn, as far as 64 bits tell
    f[1] = kNan;
    CHECK(ppd_set_rope(ctx, f, 8, 0, 1.f) == PPD_ERR_RANGE && ctx->rotation.rotary_dim == 10);  // the old one stays
    ppd_destroy(ctx);
}

static void rope() {
    ppd_ctx* ctx = make(8, 2, 64);
    double f[32] = {1};
    const uint64_t X = 1 << 20, O = 1 << 24;
    auto call = [&](const void* x, int64_t xs, int heads, const int64_t* pos, int64_t T, void* out, int64_t os) { return ppd_rope(ctx, x, xs, heads, pos, T, 0, out, os, nullptr); };
    CHECK(call(at(X), 512, 8, ints(64), 3, at(O), 512) == PPD_ERR_RANGE);  // no rotation set
    CHECK(ppd_set_rope(ctx, f, 64, 0, 1.f) == PPD_OK);
    CHECK(ppd_rope(nullptr, at(X), 512, 8, ints(64), 3, 0, at(O), 512, nullptr) == PPD_ERR_NULL);
    CHECK(call(nullptr, 512, 8, ints(64), 3, at(O), 512) == PPD_ERR_NULL);
    CHECK(call(at(X), 512, 8, nullptr, 3, at(O), 512) == PPD_ERR_NULL);
    CHECK(call(at(X), 512, 8, ints(64), 3, nullptr, 512) == PPD_ERR_NULL);
    for (int heads : {0, -1, 4097}) CHECK(call(at(X), 512, heads, ints(64), 3, at(O), 512) == PPD_ERR_RANGE);
    for (int64_t T : {int64_t(-1), int64_t(1) << 31, INT64_MAX}) CHECK(call(at(X), 512, 8, ints(64), T, at(O), 512) == PPD_ERR_RANGE);
    CHECK(call(at(X + 8), 512, 8, ints(64), 3, at(O), 512) == PPD_ERR_RANGE);
    CHECK(call(at(X), 512, 8, ints(64), 3, at(O + 2), 512) == PPD_ERR_RANGE);
    CHECK(call(at(X), 512, 8, ints(68), 3, at(O), 512) == PPD_ERR_RANGE);
    for (int64_t s : {int64_t(504), int64_t(0), int64_t(-512), int64_t(516), INT64_MAX / 8 * 8}) {
        CHECK(call(at(X), s, 8, ints(64), 3, at(O), 512) == PPD_ERR_RANGE);
        CHECK(call(at(X), 512, 8, ints(64), 3, at(O), s) == PPD_ERR_RANGE);
        CHECK(call(at(X), s, 8, ints(64), 1, at(O), s) == PPD_OK);  // of one row no stride counts
    }
    CHECK(g_rope.size() == 5);
    // overlaps: only x itself with its own stride
    CHECK(call(at(X), 512, 8, ints(64), 3, at(X), 512) == PPD_OK && call(at(X), 512, 8, ints(64), 1, at(X), 1024) == PPD_OK);
    CHECK(call(at(X), 512, 8, ints(64), 3, at(X), 520) == PPD_ERR_RANGE);
    CHECK(call(at(X), 512, 8, ints(64), 3, at(X + 1024 * 3 - 16), 512) == PPD_ERR_RANGE);
    CHECK(call(at(X), 512, 8, ints(64), 3, at(X + 1024 * 3), 512) == PPD_OK);
    CHECK(call(at(X), 512, 8, ints(64), 3, at(X - 1024 * 3), 512) == PPD_OK);
    CHECK(call(at(X), 512, 8, ints(64), 0, nullptr, 512) == PPD_OK);
    g_rope.clear();
    CHECK(ppd_rope(ctx, at(X), 600, 7, ints(64), 9, 1, at(O), 448, nullptr) == PPD_OK && g_rope.size() == 1);
    const ppd::RopeParams& p = g_rope[0];
    CHECK(p.x == (uint16_t*)X && p.out == (uint16_t*)O && p.positions == ints(64) && p.T == 9 && p.x_stride == 600 && p.out_stride == 448 && p.heads == 7);
    CHECK(p.sin_sign == -1.f && p.rot.rotary_dim == 64 && p.rot.turns[0] == ctx->rotation.turns[0]);
    ppd_destroy(ctx);
}

static void append() {
    ppd_ctx* ctx = make(8, 2, 64);
    double f[32] = {1};
    struct Args { const void *q, *k, *v; int64_t qs, ks, vs; const int64_t* pos; void* pool; const int64_t* slots; int64_t T; void* out; };
    const Args good = {at(1 << 20), at(1 << 21), at(1 << 22), 512, 128, 128, ints(64), at(1 << 28), ints(128), 5, at(1 << 24)};
    auto call = [&](const Args& a) { return ppd_kv_append_rotated(ctx, a.q, a.qs, a.k, a.ks, a.v, a.vs, a.pos, a.pool, a.slots, a.T, a.out, nullptr); };
    auto with = [&](auto change) { Args a = good; change(a); return call(a); };
    CHECK(call(good) == PPD_ERR_RANGE);
    CHECK(ppd_set_rope(ctx, f, 64, 0, 1.f) == PPD_OK);
    CHECK(call(good) == PPD_OK && g_append.size() == 1);
    CHECK(ppd_kv_append_rotated(nullptr, good.q, 512, good.k, 128, good.v, 128, good.pos, good.pool, good.slots, 5, good.out, nullptr) == PPD_ERR_NULL);
    CHECK(with([](Args& a) { a.q = nullptr; }) == PPD_ERR_NULL && with([](Args& a) { a.out = nullptr; }) == PPD_ERR_NULL);
    CHECK(with([](Args& a) { a.k = nullptr; }) == PPD_ERR_NULL && with([](Args& a) { a.v = nullptr; }) == PPD_ERR_NULL);
    CHECK(with([](Args& a) { a.pos = nullptr; }) == PPD_ERR_NULL && with([](Args& a) { a.pool = nullptr; }) == PPD_ERR_NULL && with([](Args& a) { a.slots = nullptr; }) == PPD_ERR_NULL);
    CHECK(with([](Args& a) { a.q = at((1 << 20) + 8); }) == PPD_ERR_RANGE && with([](Args& a) { a.k = at((1 << 21) + 2); }) == PPD_ERR_RANGE);
    CHECK(with([](Args& a) { a.v = at((1 << 22) + 4); }) == PPD_ERR_RANGE && with([](Args& a) { a.out = at((1 << 24) + 8); }) == PPD_ERR_RANGE);
    CHECK(with([](Args& a) { a.pool = at((1 << 28) + 8); }) == PPD_ERR_RANGE && with([](Args& a) { a.pos = ints(68); }) == PPD_ERR_RANGE && with([](Args& a) { a.slots = ints(132); }) == PPD_ERR_RANGE);
    for (int64_t T : {int64_t(-1), int64_t(1) << 31}) CHECK(with([=](Args& a) { a.T = T; }) == PPD_ERR_RANGE);
    for (int64_t s : {int64_t(120), int64_t(0), int64_t(-128), int64_t(130)}) {
        CHECK(with([=](Args& a) { a.qs = s + 384; }) == PPD_ERR_RANGE && with([=](Args& a) { a.ks = s; }) == PPD_ERR_RANGE && with([=](Args& a) { a.vs = s; }) == PPD_ERR_RANGE);
        CHECK(with([=](Args& a) { a.qs = a.ks = a.vs = s; a.T = 1; }) == PPD_OK);
    }
    CHECK(with([](Args& a) { a.out = (void*)a.q; }) == PPD_OK && with([](Args& a) { a.out = (void*)a.q; a.qs = 520; }) == PPD_ERR_RANGE);
    CHECK(with([](Args& a) { a.out = (void*)a.q; a.qs = 520; a.T = 1; }) == PPD_OK);
    CHECK(with([](Args& a) { a.out = (char*)a.q + 16; }) == PPD_ERR_RANGE && with([](Args& a) { a.out = (void*)a.k; }) == PPD_ERR_RANGE && with([](Args& a) { a.out = (void*)a.v; }) == PPD_ERR_RANGE);
    g_append.clear();
    // parts of a projection's rows; then keys and values alone
    CHECK(with([](Args& a) { a.k = (char*)a.q + 1024; a.v = (char*)a.q + 1280; a.qs = a.ks = a.vs = 768; }) == PPD_OK);
    CHECK(with([](Args& a) { a.q = nullptr; a.out = nullptr; a.qs = -1; }) == PPD_OK);
    CHECK(with([](Args& a) { a = Args(); }) == PPD_OK);  // nothing at all
    CHECK(g_append.size() == 2 && g_append[0].q_stride == 768 && g_append[0].Hq == 8 && g_append[0].Hkv == 2 && g_append[0].num_pages == 64 && !g_append[1].q);
    CHECK(ppd_set_kv_format(ctx, PPD_KV_FP8_E4M3, 0.5f, 0.25f) == PPD_OK && call(good) == PPD_OK && g_append.back().inv_k == 2.f && g_append.back().inv_v == 4.f);
    ppd_destroy(ctx);
}

int main(int argc, char** argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "frequencies") frequencies();
    else if (what == "settings") settings();
    else if (what == "rope") rope();
    else if (what == "append") append();
    else return 2;
    std::printf("ok\n");
    return 0;
}
