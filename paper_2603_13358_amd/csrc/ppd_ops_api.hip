// Host side of the drafting and eviction operators: argument checks, plans and launches behind the C ABI.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>

#include "ppd_context.h"
#include "ppd_ops.h"

namespace {

// A plan and where it lives on the device.  As with mixed attention it stays valid while the lengths do not change: the layers of one
// engine step call with the same ones.
struct TreeSlot {
    void* d_plan = nullptr;
    size_t d_plan_bytes = 0;
    std::vector<int32_t> L, n;
    bool on_device = false;
    ppd::TreePlan plan;
};

// Plans and workspace of tree and weighted attention.  Both kinds of call and both page formats have a plan of their own: a graph that
// holds calls of one kind is not touched by the other's, and one graph can hold both.
struct TreeState {
    Staging staging[kStagingSlots];
    uint32_t* flags = nullptr;  // pinned: the words the slots' `read` point at
    int next_slot = 0;
    TreeSlot slots[2][2];  // [weighted][FP8 pages]
    void* d_partials = nullptr;
    size_t d_partials_bytes = 0;
    void* d_stats = nullptr;
    size_t d_stats_bytes = 0;
    void* d_scores = nullptr;
    size_t d_scores_bytes = 0;
    void* d_select = nullptr;
    size_t d_select_bytes = 0;
};

void free_tree_state(void* p) {
    TreeState* t = static_cast<TreeState*>(p);
    if (!t) return;
    for (auto& s : t->staging)
        if (s.host) (void)hipHostFree(s.host);
    if (t->flags) (void)hipHostFree(t->flags);
    for (auto& kind : t->slots)
        for (auto& s : kind)
            if (s.d_plan) (void)hipFree(s.d_plan);
    if (t->d_partials) (void)hipFree(t->d_partials);
    if (t->d_stats) (void)hipFree(t->d_stats);
    if (t->d_scores) (void)hipFree(t->d_scores);
    if (t->d_select) (void)hipFree(t->d_select);
    delete t;
}

ppd_status tree_state(ppd_ctx* ctx, TreeState** out) {
    if (!ctx->tree) {
        TreeState* t = new TreeState();
        if (hipHostMalloc((void**)&t->flags, kStagingSlots * kStagingFlagStride * sizeof(uint32_t), kStagingFlags) != hipSuccess) {
            (void)hipGetLastError();
            t->flags = nullptr;
            free_tree_state(t);
            return fail(ctx, PPD_ERR_WORKSPACE, "pinned staging allocation failed");
        }
        for (int i = 0; i < kStagingSlots; ++i) {
            t->staging[i].read = t->flags + i * kStagingFlagStride;
            *t->staging[i].read = 0;
        }
        ctx->tree = t;
        ctx->free_tree = free_tree_state;
    }
    *out = static_cast<TreeState*>(ctx->tree);
    return PPD_OK;
}

template <class T>
size_t bytes_of(const std::vector<T>& v) { return v.size() * sizeof(T); }

// Builds the plan, grows the workspace and enqueues the upload.
ppd_status upload_tree_plan(ppd_ctx* ctx, TreeState* t, TreeSlot* slot, const int32_t* L, const int32_t* n, int32_t B, bool weighted, hipStream_t hs) {
    slot->on_device = false;
    if (!ppd::build_tree_plan(ctx->shape, L, n, B, weighted, ctx->fp8_pages ? 1 : 2, ctx->num_cus, &slot->plan))
        return fail(ctx, PPD_ERR_RANGE, "the batch has more tiles than one launch takes");
    const ppd::TreePlan& plan = slot->plan;
    const size_t items = bytes_of(plan.items), blocks = bytes_of(plan.blocks), groups = bytes_of(plan.groups);
    const size_t weighs = bytes_of(plan.weighs), score_weighs = bytes_of(plan.score_weighs);
    const size_t total = items + blocks + groups + weighs + score_weighs, upload = (total + 15) / 16 * 16;
    Staging* sg = nullptr;
    ppd_status st = next_staging(ctx, t->staging, &t->next_slot, upload, &sg);
    if (st != PPD_OK) return st;
    st = grow_device(ctx, &slot->d_plan, &slot->d_plan_bytes, upload, hs);
    if (st == PPD_OK) st = grow_device(ctx, &t->d_partials, &t->d_partials_bytes, (size_t)plan.partial_floats * sizeof(float), hs);
    if (st == PPD_OK && weighted) st = grow_device(ctx, &t->d_stats, &t->d_stats_bytes, (size_t)plan.rows * ctx->shape.num_q_heads * 2 * sizeof(float), hs);
    if (st == PPD_OK) st = grow_device(ctx, &t->d_scores, &t->d_scores_bytes, (size_t)plan.score_floats * sizeof(float), hs);
    if (st != PPD_OK) {  // the workspace may be gone: every plan has to ask for its own again
        for (auto& kind : t->slots)
            for (auto& s : kind) s.on_device = false;
        return st;
    }
    char* host = static_cast<char*>(sg->host);
    if (items) std::memcpy(host, plan.items.data(), items);
    if (blocks) std::memcpy(host + items, plan.blocks.data(), blocks);
    if (groups) std::memcpy(host + items + blocks, plan.groups.data(), groups);
    if (weighs) std::memcpy(host + items + blocks + groups, plan.weighs.data(), weighs);
    if (score_weighs) std::memcpy(host + items + blocks + groups + weighs, plan.score_weighs.data(), score_weighs);
    std::memset(host + total, 0, upload - total);
    st = enqueue_upload(ctx, *sg, slot->d_plan, upload, hs);
    if (st != PPD_OK) return st;
    slot->L.assign(L, L + B);
    slot->n.assign(n, n + B);
    slot->on_device = true;
    return PPD_OK;
}

ppd_status tree_attention_impl(ppd_ctx* ctx, const void* q, const void* kv_pages, const int32_t* page_tables, int32_t max_pages,
                               const uint64_t* mask, int32_t mask_words, const int32_t* L, const int32_t* n, int32_t B, float scale,
                               void* out, float* weights, int64_t weight_stride, bool weighted, void* stream) {
    if (!ctx) return PPD_ERR_NULL;
    if (B < 0) return fail(ctx, PPD_ERR_RANGE, "B < 0");
    if (B == 0) return PPD_OK;
    if (!q || !kv_pages || !page_tables || !L || !n || !out || (weighted ? !weights : !mask))
        return fail(ctx, PPD_ERR_NULL, weighted ? "q / kv_pages / page_tables / L / n / out / weights is NULL" : "q / kv_pages / page_tables / tree_mask / L / n / out is NULL");
    if (!(scale >= 0.f) || !std::isfinite(scale)) return fail(ctx, PPD_ERR_RANGE, "scale must be finite and >= 0");
    if (!aligned16(q) || !aligned16(out) || !aligned16(kv_pages) || (reinterpret_cast<uintptr_t>(page_tables) & 3u) ||
        (reinterpret_cast<uintptr_t>(weights) & 3u) || (reinterpret_cast<uintptr_t>(mask) & 7u))
        return fail(ctx, PPD_ERR_RANGE, "q / out / kv_pages must be 16-byte aligned, tree_mask 8-byte, page_tables and weights 4-byte aligned");
    if (!weighted && (mask_words < 1 || mask_words > ppd::kMaxMaskWords)) return fail(ctx, PPD_ERR_RANGE, "mask_words must be in [1, 16]");
    for (int i = 0; i < B; ++i) {
        if (n[i] < 1 || L[i] < 0) return fail(ctx, PPD_ERR_RANGE, "n_i must be >= 1 and L_i >= 0");
        const int64_t total = (int64_t)L[i] + n[i];
        if (total > ppd::kMaxTreeTokens) return fail(ctx, PPD_ERR_RANGE, "L_i + n_i is too large");
        if (!weighted && n[i] > 64 * mask_words)
            return fail(ctx, PPD_ERR_RANGE, "sequence " + std::to_string(i) + " has " + std::to_string(n[i]) + " nodes, a mask of " + std::to_string(mask_words) + " words has fewer bits");
        if (weighted && total > weight_stride)
            return fail(ctx, PPD_ERR_RANGE, "sequence " + std::to_string(i) + " has " + std::to_string(total) + " tokens, weight_stride is " + std::to_string(weight_stride));
        const int64_t need = (total + ppd::kPage - 1) / ppd::kPage;
        if (need > max_pages)
            return fail(ctx, PPD_ERR_PAGETABLE, "sequence " + std::to_string(i) + " needs " + std::to_string(need) + " pages, max_pages is " + std::to_string(max_pages));
    }
    hipStream_t hs = static_cast<hipStream_t>(stream);
    PPD_HIP(ctx, hipSetDevice(ctx->device));
    // As with mixed attention: a context serves one stream at a time, and under capture nothing can be planned or allocated, the state
    // of a context's first call among it.
    hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
    PPD_HIP(ctx, hipStreamIsCapturing(hs, &capturing));
    const bool in_capture = capturing != hipStreamCaptureStatusNone;
    const auto refuse_in_capture = [&] {
        return fail(ctx, PPD_ERR_RANGE, "plan changed under capture: run the step once eagerly with these L, n and options first, then capture it");
    };
    if (in_capture && !ctx->tree) return refuse_in_capture();
    TreeState* t = nullptr;
    ppd_status st = tree_state(ctx, &t);
    if (st == PPD_OK && !in_capture) st = follow_stream(ctx, hs);
    if (st != PPD_OK) return st;
    TreeSlot& slot = t->slots[weighted][ctx->fp8_pages];
    const bool reuse = slot.on_device && (int32_t)slot.L.size() == B && std::memcmp(slot.L.data(), L, sizeof(int32_t) * B) == 0 &&
                       std::memcmp(slot.n.data(), n, sizeof(int32_t) * B) == 0;
    if (!reuse) {
        if (in_capture) return refuse_in_capture();
        st = upload_tree_plan(ctx, t, &slot, L, n, B, weighted, hs);
        if (st != PPD_OK) return st;
    }
    const ppd::TreePlan& plan = slot.plan;
    const char* d_plan = static_cast<const char*>(slot.d_plan);
    ppd::TreeParams p;
    std::memset(&p, 0, sizeof p);
    p.q = static_cast<const uint16_t*>(q);
    p.out = static_cast<uint16_t*>(out);
    p.pool = kv_pages;
    p.page_tables = page_tables;
    p.mask = weighted ? nullptr : mask;
    p.items = reinterpret_cast<const ppd::TreeItem*>(d_plan);
    const char* const d_groups = d_plan + bytes_of(plan.items) + bytes_of(plan.blocks);
    p.groups = reinterpret_cast<const ppd::TreeGroup*>(d_groups);
    p.weighs = reinterpret_cast<const ppd::WeighItem*>(d_groups + bytes_of(plan.groups));
    p.score_weighs = p.weighs + plan.weighs.size();
    p.scores = static_cast<float*>(t->d_scores);
    p.partials = static_cast<float*>(t->d_partials);
    p.stats = weighted ? static_cast<float*>(t->d_stats) : nullptr;
    p.weights = weights;
    p.weight_stride = weight_stride;
    p.err_flags = ctx->d_counters + 9;
    p.num_pages = ctx->shape.num_pages;
    p.page_stride = 2LL * ctx->shape.num_kv_heads * ppd::kPage * ctx->shape.head_dim;
    p.mask_words = mask_words;
    p.max_pages = max_pages;
    p.Hq = ctx->shape.num_q_heads;
    p.Hkv = ctx->shape.num_kv_heads;
    p.G = p.Hq / p.Hkv;
    p.n_items = (int32_t)plan.items.size();
    p.n_groups = (int32_t)plan.groups.size();
    p.n_weighs = (int32_t)plan.weighs.size();
    p.n_score_weighs = (int32_t)plan.score_weighs.size();
    p.join_cols = plan.join_cols;
    // Strictly positive, so that a scale of 0 gives 2^(-inf * c) = 0 for keys that are not seen.
    p.scale_log2e = std::max(1e-30f, (float)((double)scale * (double)ctx->k_scale * 1.4426950408889634));
    p.v_scale = ctx->v_scale;
    const int D = ctx->shape.head_dim;
    int rc = 0;
    if (!plan.blocks.empty()) {
        ppd::TreeBlockParams b;
        std::memset(&b, 0, sizeof b);
        b.q = p.q;
        b.out = p.out;
        b.pool = static_cast<const uint16_t*>(kv_pages);
        b.page_tables = page_tables;
        b.items = reinterpret_cast<const ppd_work_item*>(d_plan + bytes_of(plan.items));
        b.partials = p.partials;
        b.counters = ctx->d_counters;
        b.num_pages = p.num_pages;
        b.page_stride = p.page_stride;
        b.n_items = (int32_t)plan.blocks.size();
        b.max_pages = max_pages;
        b.Hq = p.Hq;
        b.Hkv = p.Hkv;
        b.G = p.G;
        b.invG = 65536 / p.G + 1;
        b.scale_log2e = p.scale_log2e;
        b.v_scale = p.v_scale;
        b.mask = p.mask;
        b.stats = p.stats;
        b.mask_words = mask_words;
        rc = ppd::launch_tree_blocks(b, D, ctx->fp8_pages, stream);
        if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "launch tree row blocks");
    }
    if (p.n_items > 0) {
        rc = ppd::launch_tree(p, D, ctx->fp8_pages, stream);
        if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "launch tree attention");
    }
    if (p.n_groups > 0 || p.n_score_weighs > 0) {
        rc = ppd::launch_tree_join(p, D, stream);
        if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "launch join of tree tiles");
    }
    if (p.n_weighs > 0) {
        rc = ppd::launch_weigh(p, D, ctx->fp8_pages, stream);
        if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "launch weights");
    }
    if (ctx->log_calls)
        std::fprintf(stderr, "ppd: %s_attention%s B=%d tiles=%d row blocks=%d joined groups=%d plan=%s\n", weighted ? "weighted" : "tree", ctx->fp8_pages ? " (FP8 pages)" : "",
                     (int)B, (int)p.n_items, (int)plan.blocks.size(), (int)p.n_groups, reuse ? "reused" : "built");
    return PPD_OK;
}

// Rows of more than one chunk leave histograms and candidates in the workspace between their launches.
ppd_status select_workspace(ppd_ctx* ctx, ppd::SelectParams* p, int32_t longest, hipStream_t hs) {
    p->max_chunks = (longest + ppd::kSelectChunk - 1) / ppd::kSelectChunk;
    const size_t rows = (size_t)p->B * p->Hkv, chunks = rows * p->max_chunks;
    if (chunks > (size_t)INT32_MAX) return fail(ctx, PPD_ERR_RANGE, "more rows of this length than one launch takes");
    const size_t bytes = (chunks * (ppd::kSelectBins + 2 * ppd::kSelectChunk) + rows * (p->max_chunks + ppd::kSelectRowWords)) * sizeof(uint32_t);
    hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
    PPD_HIP(ctx, hipStreamIsCapturing(hs, &capturing));
    if (capturing != hipStreamCaptureStatusNone && (!ctx->tree || bytes > static_cast<TreeState*>(ctx->tree)->d_select_bytes))
        return fail(ctx, PPD_ERR_RANGE, "rows this long need a workspace, which cannot be allocated under capture: run the call once eagerly first");
    TreeState* t = nullptr;
    ppd_status st = tree_state(ctx, &t);
    if (st != PPD_OK) return st;
    if (capturing == hipStreamCaptureStatusNone) {
        st = follow_stream(ctx, hs);
        if (st == PPD_OK) st = grow_device(ctx, &t->d_select, &t->d_select_bytes, bytes, hs);
        if (st != PPD_OK) return st;
    }
    p->hist = static_cast<uint32_t*>(t->d_select);
    p->candidates = p->hist + chunks * ppd::kSelectBins;
    p->counts = reinterpret_cast<int32_t*>(p->candidates + chunks * 2 * ppd::kSelectChunk);
    return PPD_OK;
}

ppd_status select_impl(ppd_ctx* ctx, const float* weights, int64_t weight_stride, const int32_t* length, int32_t B, int32_t budget, int32_t sinks,
                       int32_t recent, int32_t* keep, int64_t keep_stride, void* stream) {
    if (!ctx) return PPD_ERR_NULL;
    if (B < 0) return fail(ctx, PPD_ERR_RANGE, "B < 0");
    if (budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget)
        return fail(ctx, PPD_ERR_RANGE, "budget must be >= 1, sinks and recent >= 0 and together at most the budget");
    if (B == 0) return PPD_OK;
    if (!weights || !length || !keep) return fail(ctx, PPD_ERR_NULL, "weights / length / keep is NULL");
    if ((reinterpret_cast<uintptr_t>(weights) & 3u) || (reinterpret_cast<uintptr_t>(keep) & 3u))
        return fail(ctx, PPD_ERR_RANGE, "weights and keep must be 4-byte aligned");
    for (int i = 0; i < B; ++i) {
        if (length[i] < 0 || length[i] > weight_stride || length[i] > INT32_MAX - 65536) return fail(ctx, PPD_ERR_RANGE, "length_i must be in [0, weight_stride]");
        if (std::min(length[i], budget) > keep_stride) return fail(ctx, PPD_ERR_RANGE, "keep_stride is smaller than the tokens to keep");
    }
    PPD_HIP(ctx, hipSetDevice(ctx->device));
    ppd::SelectParams p;
    std::memset(&p, 0, sizeof p);
    p.weight_stride = weight_stride;
    p.keep_stride = keep_stride;
    p.Hkv = ctx->shape.num_kv_heads;
    p.budget = budget;
    p.sinks = sinks;
    p.recent = recent;
    for (int32_t at = 0; at < B; at += ppd::kSelectBatch) {
        p.B = std::min(B - at, ppd::kSelectBatch);
        p.weights = weights + (int64_t)at * p.Hkv * weight_stride;
        p.keep = keep + (int64_t)at * p.Hkv * keep_stride;
        std::copy(length + at, length + at + p.B, p.length);
        const int32_t longest = *std::max_element(p.length, p.length + p.B);
        p.max_chunks = 0;
        if (longest > ppd::kSelectChunk) {
            ppd_status st = select_workspace(ctx, &p, longest, static_cast<hipStream_t>(stream));
            if (st != PPD_OK) return st;
        }
        const int rc = ppd::launch_select(p, longest, stream);
        if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "launch kv_select");
    }
    if (ctx->log_calls) std::fprintf(stderr, "ppd: kv_select B=%d budget=%d\n", (int)B, (int)budget);
    return PPD_OK;
}

ppd_status compact_impl(ppd_ctx* ctx, void* kv_pages, int64_t layer_stride_elems, int32_t num_layers, const int32_t* page_tables, int32_t max_pages,
                        const int32_t* keep, int64_t keep_layer_stride, int64_t keep_seq_stride, int64_t keep_head_stride, const int32_t* first,
                        const int32_t* count, int32_t B, float* weights, int64_t weight_stride, void* stream) {
    if (!ctx) return PPD_ERR_NULL;
    if (B < 0) return fail(ctx, PPD_ERR_RANGE, "B < 0");
    if (num_layers < 0 || num_layers > 65535) return fail(ctx, PPD_ERR_RANGE, "num_layers must be in [0, 65535]");
    if (B == 0 || num_layers == 0) return PPD_OK;
    if (!kv_pages || !page_tables || !keep || !first || !count) return fail(ctx, PPD_ERR_NULL, "kv_pages / page_tables / keep / first / count is NULL");
    const int Hkv = ctx->shape.num_kv_heads, D = ctx->shape.head_dim;
    const int64_t pool_elems = 2LL * Hkv * ppd::kPage * D * ctx->shape.num_pages;
    if (num_layers > 1 && layer_stride_elems < pool_elems) return fail(ctx, PPD_ERR_RANGE, "layer_stride_elems is smaller than one pool: layers would overlap");
    if (!aligned16(kv_pages) || (num_layers > 1 && layer_stride_elems % (ctx->fp8_pages ? 16 : 8) != 0) || (reinterpret_cast<uintptr_t>(page_tables) & 3u) ||
        (reinterpret_cast<uintptr_t>(keep) & 3u) || (reinterpret_cast<uintptr_t>(weights) & 3u))
        return fail(ctx, PPD_ERR_RANGE, "kv_pages must be 16-byte aligned (layer_stride_elems a multiple of 8, of 16 for FP8 pages), page_tables, keep and weights 4-byte aligned");
    if (keep_layer_stride < 0 || keep_seq_stride < 0 || keep_head_stride < 0) return fail(ctx, PPD_ERR_RANGE, "the strides of keep must be >= 0");
    int64_t most = 0;
    for (int i = 0; i < B; ++i) {
        if (first[i] < 0 || count[i] < 0) return fail(ctx, PPD_ERR_RANGE, "first_i and count_i must be >= 0");
        const int64_t end = (int64_t)first[i] + count[i];
        if (count[i] > 0 && end > (int64_t)max_pages * ppd::kPage)
            return fail(ctx, PPD_ERR_PAGETABLE, "sequence " + std::to_string(i) + ": tokens up to " + std::to_string(end) + " are kept, its pages hold " + std::to_string((int64_t)max_pages * ppd::kPage));
        if (count[i] > 0 && end > INT32_MAX - 65536) return fail(ctx, PPD_ERR_RANGE, "first_i + count_i is too large");
        if (weights && count[i] > 0 && end > weight_stride) return fail(ctx, PPD_ERR_RANGE, "weight_stride is smaller than first_i + count_i");
        most = std::max<int64_t>(most, count[i]);
    }
    for (int64_t s : {keep_layer_stride, keep_seq_stride, keep_head_stride})
        if (s > 0 && s < most) return fail(ctx, PPD_ERR_RANGE, "a stride of keep is smaller than a list: lists would overlap");
    if (most == 0) return PPD_OK;
    PPD_HIP(ctx, hipSetDevice(ctx->device));
    ppd::CompactParams p;
    std::memset(&p, 0, sizeof p);
    p.pool = kv_pages;
    p.err_flags = ctx->d_counters + 9;
    p.keep_layer = keep_layer_stride;
    p.keep_seq = keep_seq_stride;
    p.keep_head = keep_head_stride;
    p.weight_layer = (int64_t)B * Hkv * weight_stride;
    p.weight_stride = weight_stride;
    p.pool_layer = layer_stride_elems;
    p.num_pages = ctx->shape.num_pages;
    p.page_stride = 2LL * Hkv * ppd::kPage * D;
    p.max_pages = max_pages;
    p.Hkv = Hkv;
    for (int32_t at = 0; at < B; at += ppd::kCompactBatch) {
        p.B = std::min(B - at, ppd::kCompactBatch);
        p.page_tables = page_tables + (int64_t)at * max_pages;
        p.keep = keep + (int64_t)at * keep_seq_stride;
        p.weights = weights ? weights + (int64_t)at * Hkv * weight_stride : nullptr;
        std::copy(first + at, first + at + p.B, p.first);
        std::copy(count + at, count + at + p.B, p.count);
        // the fewest positions at a time that take the longest list in one step, or 128
        int64_t span = 0;
        for (int i = 0; i < p.B; ++i) span = std::max<int64_t>(span, p.first[i] % 8 + (int64_t)p.count[i]);
        p.step = 16;
        while (p.step < 128 && p.step < span) p.step *= 2;
        const int rc = ppd::launch_compact(p, D, ctx->fp8_pages, num_layers, stream);
        if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "launch kv_compact");
    }
    if (ctx->log_calls) std::fprintf(stderr, "ppd: kv_compact B=%d layers=%d\n", (int)B, (int)num_layers);
    return PPD_OK;
}

}  // namespace

extern "C" {

ppd_status ppd_tree_attention(ppd_ctx* ctx, const void* q, const void* kv_pages, const int32_t* page_tables, int32_t max_pages,
                              const uint64_t* tree_mask, int32_t mask_words, const int32_t* L, const int32_t* n, int32_t B, float scale,
                              void* out, void* stream) {
    return guarded(ctx, [&] {
        return tree_attention_impl(ctx, q, kv_pages, page_tables, max_pages, tree_mask, mask_words, L, n, B, scale, out, nullptr, 0, false, stream);
    });
}

ppd_status ppd_weighted_attention(ppd_ctx* ctx, const void* q, const void* kv_pages, const int32_t* page_tables, int32_t max_pages,
                                  const int32_t* L, const int32_t* n, int32_t B, float scale, void* out, float* weights,
                                  int64_t weight_stride, void* stream) {
    return guarded(ctx, [&] {
        return tree_attention_impl(ctx, q, kv_pages, page_tables, max_pages, nullptr, 0, L, n, B, scale, out, weights, weight_stride, true, stream);
    });
}

ppd_status ppd_kv_select(ppd_ctx* ctx, const float* weights, int64_t weight_stride, const int32_t* length, int32_t B, int32_t budget,
                         int32_t sinks, int32_t recent, int32_t* keep, int64_t keep_stride, void* stream) {
    return guarded(ctx, [&] { return select_impl(ctx, weights, weight_stride, length, B, budget, sinks, recent, keep, keep_stride, stream); });
}

ppd_status ppd_kv_compact(ppd_ctx* ctx, void* kv_pages, int64_t layer_stride_elems, int32_t num_layers, const int32_t* page_tables,
                          int32_t max_pages, const int32_t* keep, int64_t keep_layer_stride, int64_t keep_seq_stride,
                          int64_t keep_head_stride, const int32_t* first, const int32_t* count, int32_t B, float* weights,
                          int64_t weight_stride, void* stream) {
    return guarded(ctx, [&] {
        return compact_impl(ctx, kv_pages, layer_stride_elems, num_layers, page_tables, max_pages, keep, keep_layer_stride, keep_seq_stride, keep_head_stride,
                            first, count, B, weights, weight_stride, stream);
    });
}

}  // extern "C"
