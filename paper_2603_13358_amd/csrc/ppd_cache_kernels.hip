// gfx950 kernels of cache eviction: the choice of the tokens to keep by their weight, and the move of kept tokens to the front.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ppd_device.h"
#include "ppd_ops.h"

namespace ppd {

namespace {

// Larger for the heavier weight: the bits as an integer of the same order.  Both zeros are equal, NaN is heavier than all else.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return ~0u;
    const uint32_t b = w == 0.f ? 0u : __builtin_bit_cast(uint32_t, w);
    return b >> 31 ? ~b : b | 0x80000000u;
}

}  // namespace

// One workgroup chooses for one sequence and KV head.  The weight of the last chosen token is found digit by digit (four
// histograms of eight bits, the heaviest digit first); every wave then counts the chosen ones of its stretch of positions, and
// after a sum over the waves in front writes them in order.  Tokens of that last weight are taken from the lowest position on.
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
__global__ __launch_bounds__(kSelectThreads) void ppd_select_kernel(const SelectParams P) {
    __shared__ uint32_t hist[256];
    __shared__ uint32_t found[2];
    __shared__ int heavier[kSelectWaves], equal[kSelectWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = blockIdx.y, head = blockIdx.x, len = P.length[b];
    const float* w = P.weights + ((int64_t)b * P.Hkv + head) * P.weight_stride;
    int32_t* keep = P.keep + ((int64_t)b * P.Hkv + head) * P.keep_stride;
    if (len <= P.budget) {
        for (int t = tid; t < len; t += kSelectThreads) keep[t] = t;
        return;
    }
    const int lo = P.sinks, hi = len - P.recent;  // the others: positions [lo, hi)
    const int want = P.budget - P.sinks - P.recent;
    uint32_t prefix = 0, mask = 0;
    int left = want;  // of the tokens whose digits so far are `prefix`
    if (want > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0;
            __syncthreads();
            for (int t = lo + tid; t < hi; t += kSelectThreads) {
                const uint32_t k = weight_key(w[t]);
                if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
            }
            __syncthreads();
            if (wave == 0) {
                // lane l has digits 255 - 4l .. 252 - 4l, heaviest first
                uint32_t n[4], mine = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) mine += n[i] = hist[255 - 4 * lane - i];
                uint32_t upto = mine;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const uint32_t o = __shfl_up(upto, d, 64);
                    if (lane >= d) upto += o;
                }
                uint32_t before = upto - mine;
                if (before < (uint32_t)left && upto >= (uint32_t)left) {
                    int i = 0;
                    while (before + n[i] < (uint32_t)left) before += n[i++];
                    found[0] = 255u - 4 * lane - i;
                    found[1] = before;
                }
            }
            __syncthreads();
            prefix |= found[0] << shift;
            mask |= 255u << shift;
            left -= (int)found[1];
        }
    }
    // chosen: the first and the last ones, keys above `prefix`, and the first `left` ones equal to it
    auto classify = [&](int t, bool* above, bool* same) {
        *above = *same = false;
        if (t >= len) return;
        if (t < lo || t >= hi) {
            *above = true;
        } else if (want > 0) {
            const uint32_t k = weight_key(w[t]);
            *above = k > prefix;
            *same = k == prefix;
        }
    };
    const int stretch = (len + kSelectThreads - 1) / kSelectThreads * 64;
    const int begin = wave * stretch, end = begin + stretch;
    int n_above = 0, n_same = 0;
    for (int t = begin; t < end; t += 64) {
        bool above, same;
        classify(t + lane, &above, &same);
        n_above += __popcll(__ballot(above));
        n_same += __popcll(__ballot(same));
    }
    if (lane == 0) {
        heavier[wave] = n_above;
        equal[wave] = n_same;
    }
    __syncthreads();
    int at = 0, same_before = 0;
    for (int i = 0; i < wave; ++i) {
        at += heavier[i];
        same_before += equal[i];
    }
    at += same_before < left ? same_before : left;
    for (int t = begin; t < end; t += 64) {
        bool above, same;
        classify(t + lane, &above, &same);
        const uint64_t m_same = __ballot(same), below = (1ull << lane) - 1;
        const bool chosen = above || (same && same_before + __popcll(m_same & below) < left);
        same_before += __popcll(m_same);
        const uint64_t m = __ballot(chosen);
        if (chosen) keep[at + __popcll(m & below)] = t + lane;
        at += __popcll(m);
    }
}

int launch_select(const SelectParams& p, void* stream) {
    hipLaunchKernelGGL(ppd_select_kernel, dim3((unsigned)p.Hkv, (unsigned)p.B), dim3(kSelectThreads), 0, static_cast<hipStream_t>(stream), p);
    return (int)hipGetLastError();
}

// Moves token keep[i] of one sequence, KV head and layer to position first + i, in place.  The lists ascend and keep[i] >= first + i, so
// a destination is never read by a later token: a workgroup takes 128 destinations at a time, reads all of them, waits, and
// writes.  The d axis of K and of V is independent, so K, V and slices of d are workgroups of their own; the weights are another.
// Entries that do not ascend or lie outside the sequence's pages raise the sticky flag, and their tokens stay where they are.
constexpr int kCompactThreads = 256, kCompactStep = 128;

template <int HD, bool FP8>
__global__ __launch_bounds__(kCompactThreads) void ppd_compact_kernel(const CompactParams P) {
    typedef std::conditional_t<FP8, uint8_t, uint16_t> Elem;
    typedef std::conditional_t<FP8, u32x2, u32x4> Raw;  // eight elements
    __shared__ int64_t from[kCompactStep], to[kCompactStep];  // element offset of the page block of a token, -1: it stays
    __shared__ int from_tok[kCompactStep];
    const int tid = threadIdx.x;
    const int b = blockIdx.x / P.Hkv, head = blockIdx.x % P.Hkv, layer = blockIdx.z;
    const int first = P.first[b], count = P.count[b];
    const int32_t* keep = P.keep + layer * P.keep_layer + b * P.keep_seq + head * P.keep_head;
    const int32_t* pages = P.page_tables + (int64_t)b * P.max_pages;
    int64_t capacity = (int64_t)P.max_pages * kPage;
    if (P.weights && P.weight_stride < capacity) capacity = P.weight_stride;
    const int part = blockIdx.y;  // K slices, V slices, weights
    const int start = first & ~7, end = first + count;  // steps begin on a granule of V
    Elem* const pool = static_cast<Elem*>(P.pool) + layer * P.pool_layer + (int64_t)head * (kPage * HD);
    float* const weights = P.weights ? P.weights + layer * P.weight_layer + ((int64_t)b * P.Hkv + head) * P.weight_stride : nullptr;
    const bool is_weights = part == 2 * P.slices, is_v = part >= P.slices;
    const int width = HD / P.slices, d0 = (part % P.slices) * width;

    auto source = [&](int pos) {  // of destination `pos`, -1 where there is none
        const int i = pos - first;
        if (i < 0 || pos >= end) return -1;
        const int src = keep[i];
        if (src < pos || src >= capacity || (i > 0 && keep[i - 1] >= src)) {
            atomicOr(P.err_flags, 8u);
            return -1;
        }
        return src;
    };
    auto page_base = [&](int pos) {
        int id = pages[pos >> 4];
        if (id < 0 || id >= P.num_pages) {
            atomicOr(P.err_flags, 2u);
            return (int64_t)-1;
        }
        return id * P.page_stride;
    };

    for (int p0 = start; p0 < end; p0 += kCompactStep) {
        if (is_weights) {
            const int src = tid < kCompactStep ? source(p0 + tid) : -1;
            float v = 0.f;
            if (src >= 0) v = weights[src];
            asm volatile("s_waitcnt vmcnt(0)" : "+v"(v) : : "memory");
            __syncthreads();
            if (src >= 0) weights[p0 + tid] = v;
            continue;
        }
        __syncthreads();  // the lists of the step before are read
        if (tid < kCompactStep) {
            const int src = source(p0 + tid);
            int64_t f = -1, t = -1;
            if (src >= 0) {
                f = page_base(src);
                t = page_base(p0 + tid);
            }
            from[tid] = t < 0 ? -1 : f;
            to[tid] = f < 0 ? -1 : t;
            from_tok[tid] = src & 15;
        }
        __syncthreads();
        if (!is_v) {
            constexpr int PER = kCompactStep * (HD / 8) / kCompactThreads;
            const int units = kCompactStep * (width / 8);
            Raw v[PER];
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int u = tid + j * kCompactThreads, t = u % kCompactStep, g = d0 / 8 + u / kCompactStep;
                v[j] = Raw{};
                if (u < units && from[t] >= 0) v[j] = *reinterpret_cast<const Raw*>(pool + from[t] + (g * kPage + from_tok[t]) * 8);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int u = tid + j * kCompactThreads, t = u % kCompactStep, g = d0 / 8 + u / kCompactStep;
                if (u < units && to[t] >= 0) *reinterpret_cast<Raw*>(pool + to[t] + (g * kPage + ((p0 + t) & 15)) * 8) = v[j];
            }
        } else {
            constexpr int PER = kCompactStep / 8 * HD / kCompactThreads;
            const int units = kCompactStep / 8 * width;
            Elem* const vpool = pool + (int64_t)P.Hkv * (kPage * HD);
            Elem v[PER][8];
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int u = tid + j * kCompactThreads, d = d0 + u % width, g = u / width;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = g * 8 + e;
                    v[j][e] = 0;
                    if (u < units && from[t] >= 0) v[j][e] = vpool[from[t] + (from_tok[t] >> 3) * (HD * 8) + d * 8 + (from_tok[t] & 7)];
                }
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int u = tid + j * kCompactThreads, d = d0 + u % width, g = u / width;
                if (u >= units) continue;
                bool whole = true;
#pragma unroll
                for (int e = 0; e < 8; ++e) whole &= to[g * 8 + e] >= 0;
                const int at = (((p0 + g * 8) & 15) >> 3) * (HD * 8) + d * 8;
                if (whole) {
                    *reinterpret_cast<Raw*>(vpool + to[g * 8] + at) = __builtin_bit_cast(Raw, v[j]);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (to[g * 8 + e] >= 0) vpool[to[g * 8 + e] + at + e] = v[j][e];
                }
            }
        }
    }
}

int launch_compact(const CompactParams& p, int head_dim, bool fp8_pages, int layers, void* stream) {
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)(p.B * p.Hkv), (unsigned)(2 * p.slices + (p.weights ? 1 : 0)), (unsigned)layers);
    if (head_dim == 128 && fp8_pages) hipLaunchKernelGGL((ppd_compact_kernel<128, true>), grid, dim3(kCompactThreads), 0, hs, p);
    else if (head_dim == 128) hipLaunchKernelGGL((ppd_compact_kernel<128, false>), grid, dim3(kCompactThreads), 0, hs, p);
    else if (fp8_pages) hipLaunchKernelGGL((ppd_compact_kernel<64, true>), grid, dim3(kCompactThreads), 0, hs, p);
    else hipLaunchKernelGGL((ppd_compact_kernel<64, false>), grid, dim3(kCompactThreads), 0, hs, p);
    return (int)hipGetLastError();
}

}  // namespace ppd
