// Host-only checks of the attention plans' partials in the workspace (built and run by tests/test_partials_host.py).
#include <cstdio>
#include <cstdlib>
#include <random>
#include <string>
#include <vector>

#include "../../paper_2603_13358_amd/csrc/ppd_prefix.h"

#define CHECK(x)                                                      \
    do {                                                              \
        if (!(x)) {                                                   \
            std::printf("%s:%d: not so: %s\n", __FILE__, __LINE__, #x); \
            std::fflush(stdout);                                      \
            std::_Exit(1);                                            \
        }                                                             \
    } while (0)

// Partials start where the kernels, which move four floats of one at a time, say that they do.
static void alignment() {
    std::mt19937 r(3);
    auto in = [&](int lo, int hi) { return (int)(lo + r() % (unsigned)(hi - lo + 1)); };
    int64_t prefix = 0, tree = 0, mixed = 0, odd = 0;
    auto check = [&](int64_t off, int64_t* count) {
        if (off < 0) return;
        CHECK(off % ppd::kPartialAlign == 0);
        odd += off % 4 != 0;
        ++*count;
    };
    for (int round = 0; round < 60; ++round) {
        const int G = in(1, 8), Hkv = in(1, 3), B = in(1, 70), most_new = in(0, 2) ? 3 : 120, prompt = 64 * in(1, 200);
        const ppd_shape s = {G * Hkv, Hkv, in(0, 1) ? 64 : 128, 16, 1 << 20};
        std::vector<int32_t> shared(B, prompt), L(B), n(B);
        shared[0] = 0;
        for (int i = 0; i < B; ++i) L[i] = prompt + in(0, 2000), n[i] = in(1, most_new);
        ppd::PrefixPlan p;
        CHECK(ppd::build_prefix_plan(s, shared.data(), L.data(), n.data(), B, 2, 256, &p));
        for (const auto& t : p.items) check(t.part_off, &prefix);
        for (const auto& t : p.blocks) check(t.part_off, &prefix);
        ppd::TreePlan t;
        CHECK(ppd::build_tree_plan(s, L.data(), n.data(), B, round % 2, 2, 256, &t));
        for (const auto& x : t.items) check(x.part_off, &tree);
        for (const auto& x : t.blocks) check(x.part_off, &tree);
        for (const auto& x : t.groups) CHECK(x.part_stride % ppd::kPartialAlign == 0);
        ppd::Plan m;
        ppd::PlanOptions options;
        const char* why = nullptr;
        CHECK(ppd::build_plan(s, L.data(), n.data(), B, options, &m, &why) == PPD_OK);
        for (const auto& x : m.items) check(x.part_off, &mixed);
    }
    CHECK(prefix > 1000 && tree > 1000 && mixed > 1000 && odd > 100);  // some are off a multiple of 16 bytes
}

int main(int argc, char** argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "alignment") alignment();
    else return 2;
    std::printf("ok\n");
    return 0;
}
