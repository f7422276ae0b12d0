// Host side of attention over shared prefixes: argument checks, plan and launches behind the C ABI.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>

#include "ppd_context.h"
#include "ppd_prefix.h"

namespace {

// A plan and where it lives on the device; it stays valid while the lengths and what is shared do not change.
struct PrefixState {
    Staging staging[kStagingSlots];
    uint32_t* flags = nullptr;  // pinned: the words the slots' `read` point at
    int next_slot = 0;
    void* d_plan = nullptr;
    size_t d_plan_bytes = 0;
    void* d_partials = nullptr;
    size_t d_partials_bytes = 0;
    std::vector<int32_t> shared, L, n;
    bool on_device = false;
    ppd::PrefixPlan plan;
};

void free_prefix_state(void* p) {
    PrefixState* t = static_cast<PrefixState*>(p);
    if (!t) return;
    for (auto& s : t->staging)
        if (s.host) (void)hipHostFree(s.host);
    if (t->flags) (void)hipHostFree(t->flags);
    if (t->d_plan) (void)hipFree(t->d_plan);
    if (t->d_partials) (void)hipFree(t->d_partials);
    delete t;
}

ppd_status prefix_state(ppd_ctx* ctx, PrefixState** out) {
    if (!ctx->prefix) {
        PrefixState* t = new PrefixState();
        if (hipHostMalloc((void**)&t->flags, kStagingSlots * kStagingFlagStride * sizeof(uint32_t), kStagingFlags) != hipSuccess) {
            (void)hipGetLastError();
            t->flags = nullptr;
            free_prefix_state(t);
            return fail(ctx, PPD_ERR_WORKSPACE, "pinned staging allocation failed");
        }
        for (int i = 0; i < kStagingSlots; ++i) {
            t->staging[i].read = t->flags + i * kStagingFlagStride;
            *t->staging[i].read = 0;
        }
        ctx->prefix = t;
        ctx->free_prefix = free_prefix_state;
    }
    *out = static_cast<PrefixState*>(ctx->prefix);
    return PPD_OK;
}

// The plan's lists one behind the other, each at a multiple of 16 bytes.
struct PlanLayout {
    size_t blocks, units, sources, total;
    explicit PlanLayout(const ppd::PrefixPlan& p) {
        auto after = [](size_t at, size_t bytes) { return (at + bytes + 15) / 16 * 16; };
        blocks = after(0, p.items.size() * sizeof(ppd::PrefixItem));
        units = after(blocks, p.blocks.size() * sizeof(ppd_work_item));
        sources = after(units, p.units.size() * sizeof(ppd::JoinUnit));
        total = after(sources, p.sources.size() * sizeof(ppd::JoinSource));
    }
};

template <class T>
void put(char* to, const std::vector<T>& v) {
    if (!v.empty()) std::memcpy(to, v.data(), v.size() * sizeof(T));
}

// Builds the plan, grows the workspace and enqueues the upload.
ppd_status upload_prefix_plan(ppd_ctx* ctx, PrefixState* t, const int32_t* shared, const int32_t* L, const int32_t* n, int32_t B, hipStream_t hs) {
    t->on_device = false;
    ppd_status st = PPD_OK;
    const std::string error = ctx->error;
    for (int64_t most = ppd::kMostPartialFloats;; most /= 4) {
        if (!ppd::build_prefix_parts(ctx->shape, shared, L, n, B, ctx->fp8_pages ? 1 : 2, ctx->num_cus, most, &t->plan))
            return fail(ctx, PPD_ERR_RANGE, "the batch has more tiles than one launch takes");
        st = grow_device(ctx, &t->d_partials, &t->d_partials_bytes, (size_t)t->plan.partial_floats * sizeof(float), hs);
        // Where memory is short the batch is cut into more parts.
        if (st != PPD_ERR_WORKSPACE || most <= ppd::kFewestPartialFloats) break;
    }
    if (st != PPD_OK) return st;
    ctx->error = error;  // that of the last call that failed
    const ppd::PrefixPlan& plan = t->plan;
    const PlanLayout at(plan);
    Staging* sg = nullptr;
    st = next_staging(ctx, t->staging, &t->next_slot, at.total, &sg);
    if (st == PPD_OK) st = grow_device(ctx, &t->d_plan, &t->d_plan_bytes, at.total, hs);
    if (st != PPD_OK) return st;
    char* host = static_cast<char*>(sg->host);
    std::memset(host, 0, at.total);
    put(host, plan.items);
    put(host + at.blocks, plan.blocks);
    put(host + at.units, plan.units);
    put(host + at.sources, plan.sources);
    st = enqueue_upload(ctx, *sg, t->d_plan, at.total, hs);
    if (st != PPD_OK) return st;
    t->shared.assign(shared, shared + B);
    t->L.assign(L, L + B);
    t->n.assign(n, n + B);
    t->on_device = true;
    return PPD_OK;
}

bool same(const std::vector<int32_t>& have, const int32_t* v, int32_t count) {
    return (int32_t)have.size() == count && std::memcmp(have.data(), v, sizeof(int32_t) * count) == 0;
}

ppd_status prefix_attention_impl(ppd_ctx* ctx, const void* q, const void* kv_pages, const int32_t* page_tables, int32_t max_pages, const int32_t* shared,
                                 const int32_t* L, const int32_t* n, int32_t B, float scale, void* out, void* stream) {
    if (!ctx) return PPD_ERR_NULL;
    if (B < 0) return fail(ctx, PPD_ERR_RANGE, "B < 0");
    if (B == 0) return PPD_OK;
    if (!q || !kv_pages || !page_tables || !shared || !L || !n || !out) return fail(ctx, PPD_ERR_NULL, "q / kv_pages / page_tables / shared / L / n / out is NULL");
    if (!(scale >= 0.f) || !std::isfinite(scale)) return fail(ctx, PPD_ERR_RANGE, "scale must be finite and >= 0");
    if (!aligned16(q) || !aligned16(out) || !aligned16(kv_pages) || (reinterpret_cast<uintptr_t>(page_tables) & 3u))
        return fail(ctx, PPD_ERR_RANGE, "q / out / kv_pages must be 16-byte aligned, page_tables 4-byte aligned");
    int64_t rows = 0;
    for (int i = 0; i < B; ++i) {
        if (n[i] < 1 || L[i] < 0) return fail(ctx, PPD_ERR_RANGE, "n_i must be >= 1 and L_i >= 0");
        const int64_t total = (int64_t)L[i] + n[i];
        if (total > ppd::kMaxTreeTokens) return fail(ctx, PPD_ERR_RANGE, "L_i + n_i is too large");
        if ((rows += n[i]) > ppd::kMaxTreeTokens) return fail(ctx, PPD_ERR_RANGE, "the batch has too many rows");
        const int64_t need = (total + ppd::kPage - 1) / ppd::kPage;
        if (need > max_pages)
            return fail(ctx, PPD_ERR_PAGETABLE, "sequence " + std::to_string(i) + " needs " + std::to_string(need) + " pages, max_pages is " + std::to_string(max_pages));
        if (i == 0 ? shared[0] != 0 : shared[i] < 0 || shared[i] > std::min(L[i], L[i - 1]))
            return fail(ctx, PPD_ERR_RANGE, "shared_" + std::to_string(i) + " is " + std::to_string(shared[i]) + ": it must be in [0, min(L_i, L_{i-1})], and 0 for the first sequence");
    }
    hipStream_t hs = static_cast<hipStream_t>(stream);
    PPD_HIP(ctx, hipSetDevice(ctx->device));
    // As with the other attention calls: a context serves one stream at a time, and under capture nothing can be planned or allocated.
    hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
    PPD_HIP(ctx, hipStreamIsCapturing(hs, &capturing));
    const bool in_capture = capturing != hipStreamCaptureStatusNone;
    const auto refuse_in_capture = [&] {
        return fail(ctx, PPD_ERR_RANGE, "plan changed under capture: run the step once eagerly with these shared, L and n first, then capture it");
    };
    if (in_capture && !ctx->prefix) return refuse_in_capture();
    PrefixState* t = nullptr;
    ppd_status st = prefix_state(ctx, &t);
    if (st == PPD_OK && !in_capture) st = follow_stream(ctx, hs);
    if (st != PPD_OK) return st;
    const bool reuse = t->on_device && same(t->L, L, B) && same(t->n, n, B) && same(t->shared, shared, B);
    if (!reuse) {
        if (in_capture) return refuse_in_capture();
        st = upload_prefix_plan(ctx, t, shared, L, n, B, hs);
        if (st != PPD_OK) return st;
    }
    const ppd::PrefixPlan& plan = t->plan;
    const PlanLayout at(plan);
    const char* d_plan = static_cast<const char*>(t->d_plan);
    ppd::PrefixParams p;
    std::memset(&p, 0, sizeof p);
    p.q = static_cast<const uint16_t*>(q);
    p.out = static_cast<uint16_t*>(out);
    p.pool = kv_pages;
    p.page_tables = page_tables;
    p.partials = static_cast<float*>(t->d_partials);
    p.err_flags = ctx->d_counters + 9;
    p.num_pages = ctx->shape.num_pages;
    p.page_stride = 2LL * ctx->shape.num_kv_heads * ppd::kPage * ctx->shape.head_dim;
    p.max_pages = max_pages;
    p.Hq = ctx->shape.num_q_heads;
    p.Hkv = ctx->shape.num_kv_heads;
    p.G = p.Hq / p.Hkv;
    p.invG = 65536 / p.G + 1;
    // Strictly positive, so that a scale of 0 gives 2^(-inf * c) = 0 for keys that are not seen.
    p.scale_log2e = std::max(1e-30f, (float)((double)scale * (double)ctx->k_scale * 1.4426950408889634));
    p.v_scale = ctx->v_scale;
    const int D = ctx->shape.head_dim;
    for (const ppd::PrefixPart& part : plan.parts) {
        p.items = reinterpret_cast<const ppd::PrefixItem*>(d_plan) + part.item0;
        p.units = reinterpret_cast<const ppd::JoinUnit*>(d_plan + at.units) + part.unit0;
        p.sources = reinterpret_cast<const ppd::JoinSource*>(d_plan + at.sources) + part.source0;
        p.n_items = part.n_items;
        p.n_units = part.n_units;
        p.join_cols = part.join_cols;
        p.source_stride = part.source_stride;
        if (part.n_blocks > 0) {
            ppd::TreeBlockParams b;
            std::memset(&b, 0, sizeof b);
            b.q = p.q;
            b.out = p.out;
            b.pool = static_cast<const uint16_t*>(kv_pages);
            b.page_tables = page_tables;
            b.items = reinterpret_cast<const ppd_work_item*>(d_plan + at.blocks) + part.block0;
            b.partials = p.partials;
            b.counters = ctx->d_counters;
            b.num_pages = p.num_pages;
            b.page_stride = p.page_stride;
            b.n_items = part.n_blocks;
            b.max_pages = max_pages;
            b.Hq = p.Hq;
            b.Hkv = p.Hkv;
            b.G = p.G;
            b.invG = p.invG;
            b.scale_log2e = p.scale_log2e;
            b.v_scale = p.v_scale;
            const int rc = ppd::launch_tree_blocks(b, D, ctx->fp8_pages, stream);
            if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "launch prefix row blocks");
        }
        if (p.n_items > 0) {
            const int rc = ppd::launch_prefix(p, D, ctx->fp8_pages, stream);
            if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "launch prefix attention");
        }
        if (p.n_units > 0) {
            const int rc = ppd::launch_prefix_join(p, D, stream);
            if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "launch join of prefix tiles");
        }
    }
    if (ctx->log_calls)
        std::fprintf(stderr, "ppd: prefix_attention%s B=%d parts=%d tiles=%d row blocks=%d joined units=%d keys=%lld of %lld plan=%s\n", ctx->fp8_pages ? " (FP8 pages)" : "",
                     (int)B, (int)plan.parts.size(), (int)plan.items.size(), (int)plan.blocks.size(), (int)plan.units.size(), (long long)plan.keys_read, (long long)plan.keys_alone, reuse ? "reused" : "built");
    return PPD_OK;
}

}  // namespace

extern "C" {

ppd_status ppd_prefix_attention(ppd_ctx* ctx, const void* q, const void* kv_pages, const int32_t* page_tables, int32_t max_pages, const int32_t* shared,
                                const int32_t* L, const int32_t* n, int32_t B, float scale, void* out, void* stream) {
    return guarded(ctx, [&] { return prefix_attention_impl(ctx, q, kv_pages, page_tables, max_pages, shared, L, n, B, scale, out, stream); });
}

}  // extern "C"
