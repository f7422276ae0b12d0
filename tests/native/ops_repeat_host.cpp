// Host-only checks of what the drafting and eviction calls leave behind for the calls and graphs after them (built and run by
// tests/test_ops_repeat.py), with the recorded launches of ops_host.cpp and allocations that fail while a stream is captured, as
// the runtime's do.
#include <hip/hip_runtime.h>

static int g_captured_allocations = 0;
template <class T>
static hipError_t allocate_unless_captured(T** p, size_t n) {
    if (sim.capturing) {
        ++g_captured_allocations;
        return sim.pending = hipErrorInvalidValue;
    }
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

int main(int, char** argv) {
    const std::string what = argv[1];
    if (what == "first_call_under_capture") first_call_under_capture();
    else return 2;
    std::printf("ok\n");
    return 0;
}
