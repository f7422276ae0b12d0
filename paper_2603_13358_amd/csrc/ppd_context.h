// The context behind a ppd_ctx handle, and what the host API's files share: errors, workspaces, plan staging.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <exception>
#include <new>
#include <string>
#include <thread>
#include <utility>
#include <vector>

#include "ppd_internal.h"

namespace {

constexpr int kStagingSlots = 4;
constexpr int kStagingFlagStride = 16;  // words between the slots' flags: a cache line each
// the upload kernel reads the staged plan in place, and the host reads the flag it writes: mapped, coherent
constexpr unsigned kStagingFlags = hipHostMallocMapped | hipHostMallocCoherent;

// A pinned buffer a plan is staged in on its way to the device.  The upload kernel writes the upload's serial number
// to *read when it has read the buffer.
struct Staging {
    void* host = nullptr;  // pinned, mapped
    size_t bytes = 0;
    uint32_t* read = nullptr;  // written by the device
    uint32_t serial = 0;
};

}  // namespace

struct ppd_ctx {
    ppd_shape shape;
    int device = 0;
    int num_cus = 256;
    ppd::PlanOptions opts;
    std::string error;
    ppd::Plan plan;
    // device workspace
    void* d_items = nullptr;
    size_t d_items_bytes = 0;
    float* d_partials = nullptr;
    size_t d_partials_floats = 0;
    uint32_t* d_counters = nullptr;  // kCounterWords words: error flags, finished-workgroup counts, queue cursors
    Staging staging[kStagingSlots];
    uint32_t* staging_flags = nullptr;  // pinned, behind static_staging: the words the slots' `read` point at
    int next_slot = 0;
    // the plan on the device stays valid while L, n and the planner options do not change (the layers of one
    // engine step call with the same lengths): such calls skip planning and upload
    std::vector<int32_t> plan_L, plan_n;
    ppd::PlanOptions plan_opts;
    bool plan_on_device = false;
    std::vector<int32_t> block_order;
    // where that plan lives: 1 = the context's own workspace, 2 = the library's static scratch array
    int plan_where = 0;
    hipStream_t plan_stream = nullptr;  // the stream the plan was uploaded on and the last call ran on
    bool have_plan_stream = false;
    // the co-resident pair: the stream kernel runs on a stream of the context's own, forked from and joined to the
    // caller's stream with these events
    hipStream_t side_stream = nullptr;
    hipEvent_t ev_fork = nullptr, ev_join = nullptr;
    int launch_mode = 0;  // option "launch_mode"
    bool narrow_kernel = true;  // option "narrow_kernel": launches without row-block tiles run ppd_narrow_kernel
    // element format of the pools (ppd_set_kv_format): FP8 E4M3 codes with one scale per tensor, or bf16
    bool fp8_pages = false;
    float k_scale = 1.f, v_scale = 1.f;
    // debugging aids switched on by environment variables read in ppd_create
    bool log_calls = false;          // PPD_LOG=1: one line per call on stderr
    uint32_t* d_slot_seen = nullptr;  // PPD_DEBUG_SLOTS=1: one bit per pool slot, to find duplicate slots of an append
    Staging static_staging;  // of the entry point that allocates nothing (fixed size, allocated with the context)
    // optional timing of the attention kernels alone (option "timing"): one pair of events per call since the option
    // was set or the times were last collected, up to kMaxTimedLaunches
    bool timing = false;
    std::vector<std::pair<hipEvent_t, hipEvent_t>> ev_pairs;
    size_t ev_used = 0;
    // drafting and eviction (ppd_ops_api.hip): their plan and workspace, made by the first call that needs one
    void* tree = nullptr;
    void (*free_tree)(void*) = nullptr;
    // positions and shared prefixes: the rotation (ppd_set_rope; rotary_dim 0: none yet), and the plan and workspace of prefix attention
    ppd::Rotation rotation = {};
    void* prefix = nullptr;
    void (*free_prefix)(void*) = nullptr;
};

namespace ppd {
inline thread_local std::string g_create_error;  // message of the last failing call that has no context

// PPD_DEBUG_SLOTS=1: looks for duplicate slots among the T slots of an append (error flag bit 2), on `stream`.
void check_duplicate_slots(ppd_ctx* ctx, const int64_t* slot_mapping, int64_t T, hipStream_t stream);
}  // namespace ppd

namespace {

using ppd::g_create_error;

ppd_status fail(ppd_ctx* ctx, ppd_status st, const std::string& msg) {
    if (ctx) ctx->error = msg; else g_create_error = msg;
    return st;
}

ppd_status hip_fail(ppd_ctx* ctx, hipError_t e, const char* what) {
    return fail(ctx, PPD_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

#define PPD_HIP(ctx, call)                                         \
    do {                                                           \
        hipError_t e_ = (call);                                    \
        if (e_ != hipSuccess) return hip_fail((ctx), e_, #call);   \
    } while (0)

// Grows a device buffer (contents are not kept).  Waits for the stream first: the old buffer may be in use.
inline ppd_status grow_device(ppd_ctx* ctx, void** ptr, size_t* have, size_t need, hipStream_t st) {
    if (need <= *have) return PPD_OK;
    PPD_HIP(ctx, hipStreamSynchronize(st));
    if (*ptr) PPD_HIP(ctx, hipFree(*ptr));
    *ptr = nullptr;
    *have = 0;
    size_t want = need + need / 4 + 4096;
    if (hipMalloc(ptr, want) != hipSuccess) {
        (void)hipGetLastError();
        *ptr = nullptr;
        return fail(ctx, PPD_ERR_WORKSPACE, "workspace allocation of " + std::to_string(want) + " bytes failed");
    }
    *have = want;
    return PPD_OK;
}

// The kernels move 16 bytes per lane: tensors and pools must start on a 16-byte boundary.
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Copies a staged plan from pinned host memory to the device and tells the host that the staging buffer has been read.
// Bound by the latency of one read across PCIe (2 us) up to ~50 KB, by its bandwidth beyond (180 KB: ~6 us).  A copy
// command does the same through the copy engine, whose hand-overs with the kernels before and after leave the stream
// idle for ~20 us; a kernel follows and is followed like any other.
// Measured: 13-15 us less per new plan (a decode step of 64 sequences at 1K-8K over two layers 433 -> 418 us, an
// append-prefill of 16 and the decode step after it 816 -> 793 us).
// One workgroup moves 16 KiB (16 B per lane, every read issued at once); the last one to finish (counted in word
// kUploadWord of the counters, which it re-arms) writes the serial number.
constexpr int kUploadThreads = 1024;
__global__ __launch_bounds__(kUploadThreads) void ppd_upload_kernel(const uint4* host, uint4* dev, int64_t granules, uint32_t* counters,
                                                                    uint32_t* read, uint32_t serial) {
    const int64_t i = (int64_t)blockIdx.x * kUploadThreads + threadIdx.x;
    if (i < granules) dev[i] = host[i];
    __syncthreads();  // the workgroup's reads have returned: their values are stored
    if (threadIdx.x == 0) {
        if (gridDim.x > 1) {
            if (atomicAdd(&counters[ppd::kUploadWord], 1u) != gridDim.x - 1) return;
            __hip_atomic_store(&counters[ppd::kUploadWord], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __hip_atomic_store(read, serial, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
    }
}

// Waits until the upload that last used a staging buffer has read it.  That upload alone: a host that runs ahead of the
// device must neither wait for the layers enqueued behind it nor for other streams, and synchronising is not allowed while
// a stream of the process is being captured.  An upload is always launched before its serial number counts here, so the
// flag arrives as soon as the work in front of it on its stream is done.
void wait_staging_read(const Staging& sg) {
    int spins = 0;
    while (__atomic_load_n(sg.read, __ATOMIC_ACQUIRE) != sg.serial) {
        if (spins < 1 << 10) ++spins;
        else std::this_thread::yield();
    }
}

// A context serves one stream at a time: what the call before enqueued on another one has to finish first.
inline ppd_status follow_stream(ppd_ctx* ctx, hipStream_t hs) {
    if (ctx->have_plan_stream && ctx->plan_stream != hs) PPD_HIP(ctx, hipStreamSynchronize(ctx->plan_stream));
    ctx->plan_stream = hs;
    ctx->have_plan_stream = true;
    return PPD_OK;
}

// Nothing may leave a C entry point but a status.
template <class F>
ppd_status guarded(ppd_ctx* ctx, F f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return ctx ? fail(ctx, PPD_ERR_WORKSPACE, "out of host memory") : PPD_ERR_WORKSPACE;
    } catch (const std::exception& e) {
        return ctx ? fail(ctx, PPD_ERR_WORKSPACE, e.what()) : PPD_ERR_WORKSPACE;
    }
}

// The next of a ring of staging buffers, free and with room for `bytes`.
inline ppd_status next_staging(ppd_ctx* ctx, Staging* ring, int* next, size_t bytes, Staging** out) {
    Staging& sg = ring[*next];
    wait_staging_read(sg);
    *next = (*next + 1) % kStagingSlots;
    if (sg.bytes < bytes) {
        if (sg.host) PPD_HIP(ctx, hipHostFree(sg.host));
        sg.host = nullptr;
        sg.bytes = 0;
        const size_t want = bytes + bytes / 4 + 4096;
        if (hipHostMalloc(&sg.host, want, kStagingFlags) != hipSuccess) {
            (void)hipGetLastError();
            sg.host = nullptr;
            return fail(ctx, PPD_ERR_WORKSPACE, "pinned staging allocation failed");
        }
        sg.bytes = want;
    }
    *out = &sg;
    return PPD_OK;
}

// Enqueues the upload of a staged plan of `bytes`, a multiple of 16.
inline ppd_status enqueue_upload(ppd_ctx* ctx, Staging& sg, void* to, size_t bytes, hipStream_t hs) {
    const uint4* src = static_cast<const uint4*>(sg.host);
    uint4* dst = static_cast<uint4*>(to);
    int64_t granules = (int64_t)(bytes / 16);
    uint32_t serial = ++sg.serial;
    void* args[] = {&src, &dst, &granules, &ctx->d_counters, &sg.read, &serial};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(&ppd_upload_kernel),
                                         dim3((unsigned)((granules + kUploadThreads - 1) / kUploadThreads)), dim3(kUploadThreads), args, 0, hs);
    if (e != hipSuccess) {
        sg.serial -= 1;  // nothing was enqueued: the buffer is free
        return hip_fail(ctx, e, "launch plan upload");
    }
    return PPD_OK;
}

}  // namespace
