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

// ---- the choice ---------------------------------------------------------------------------------------------
// The weight of the last chosen token is found digit by digit, the heaviest first (histograms in LDS over 11, 11 and 10 bits): `prefix` holds
// the digits found so far in the places of `mask`, `left` how many of the tokens with these digits are chosen.  A search ends
// early where they all are.  Tokens of that last weight are taken from the lowest position on.
constexpr int kDigits = 3, kBins = kSelectBins;
__device__ __forceinline__ int digit_shift(int i) { return i == 0 ? 21 : i == 1 ? 10 : 0; }
__device__ __forceinline__ int digit_bins(int i) { return i == 2 ? 1024 : 2048; }

struct Search {
    uint32_t prefix = 0, mask = 0;
    int left = 0;
    __device__ __forceinline__ bool candidate(uint32_t key) const { return (key & mask) == prefix; }
    __device__ __forceinline__ bool above(uint32_t key) const { return (key & mask) > prefix; }
};

template <int NT>
struct SearchLds {
    uint32_t hist[kBins];
    uint32_t wave_sum[NT / 64];
    uint32_t found[3];  // digit, tokens above it, tokens of it
};

// Adds the digits of a wave's lanes to the histogram.  Weights that attention leaves crowd in few bins (and many are zero): the
// first lane's digit is counted for all that share it at once.
__device__ __forceinline__ void count_digit(uint32_t* hist, bool live, uint32_t digit) {
    const uint64_t all = __ballot(live);
    if (!all) return;
    const int first = __builtin_ctzll(all);
    const uint32_t common = __builtin_amdgcn_readlane(digit, first);
    const uint64_t same = __ballot(live && digit == common);
    if ((int)(threadIdx.x & 63) == first) atomicAdd(&hist[common], (uint32_t)__popcll(same));
    if (live && digit != common) atomicAdd(&hist[digit], 1u);
}

// Thread t has the bins kBins - 1 - t * PER .. (heaviest first); the one in which the running count reaches `left` is the digit.  All threads
// call it, with the histogram complete; the histogram may be cleared after it.  Returns whether all tokens of the digit are chosen.
template <int NT>
__device__ __forceinline__ bool take_digit(SearchLds<NT>& lds, Search& s, int i, const uint32_t (&n)[kBins / NT]) {
    constexpr int PER = kBins / NT;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t mine = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) mine += n[j];
    uint32_t upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(upto, d, 64);
        if (lane >= d) upto += o;
    }
    if (lane == 63) lds.wave_sum[wave] = upto;
    __syncthreads();
    uint32_t before = upto - mine;
    for (int w = 0; w < wave; ++w) before += lds.wave_sum[w];
    if (before < (uint32_t)s.left && before + mine >= (uint32_t)s.left) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            if (before < (uint32_t)s.left && before + n[j] >= (uint32_t)s.left) {
                lds.found[0] = kBins - 1 - (tid * PER + j);
                lds.found[1] = before;
                lds.found[2] = n[j];
            }
            before += n[j];
        }
    }
    __syncthreads();
    const int shift = digit_shift(i);
    s.prefix |= lds.found[0] << shift;
    s.mask |= (uint32_t)(digit_bins(i) - 1) << shift;
    s.left -= (int)lds.found[1];
    return (int)lds.found[2] == s.left;
}

template <int NT>
__device__ __forceinline__ bool take_digit_from_lds(SearchLds<NT>& lds, Search& s, int i) {
    constexpr int PER = kBins / NT;
    uint32_t n[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) n[j] = lds.hist[kBins - 1 - (threadIdx.x * PER + j)];
    return take_digit<NT>(lds, s, i, n);
}

template <int NT>
__device__ __forceinline__ void clear_hist(SearchLds<NT>& lds) {
    for (int i = threadIdx.x; i < kBins; i += NT) lds.hist[i] = 0;
    __syncthreads();
}

// A line is 64 neighbouring positions, a lane each.  Writes the chosen ones of a line in order and moves on.
struct Writer {
    int32_t* keep;
    int at, same_before;
    __device__ __forceinline__ void line(const Search& s, int pos, bool always, bool candidate) {
        const int lane = threadIdx.x & 63;
        const uint64_t below = (1ull << lane) - 1, same = __ballot(candidate);
        const bool chosen = always || (candidate && same_before + __popcll(same & below) < s.left);
        same_before += __popcll(same);
        const uint64_t m = __ballot(chosen);
        if (chosen) keep[at + __popcll(m & below)] = pos;
        at += __popcll(m);
    }
};

// One workgroup to a sequence and KV head, whose weights it reads once and holds in registers: wave w has the lines w * lines ..
// (w + 1) * lines - 1, at most VPT of them.
template <int NT, int VPT>
__global__ __launch_bounds__(NT) void ppd_select_kernel(const SelectParams P) {
    constexpr int NW = NT / 64;
    __shared__ SearchLds<NT> lds;
    __shared__ int n_above[NW], n_same[NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = blockIdx.y, head = blockIdx.x, len = P.length[b];
    const float* w = P.weights + ((int64_t)b * P.Hkv + head) * P.weight_stride;
    int32_t* keep = P.keep + ((int64_t)b * P.Hkv + head) * P.keep_stride;
    if (len <= P.budget) {
        for (int t = tid; t < len; t += NT) keep[t] = t;
        return;
    }
    const int lo = P.sinks, hi = len - P.recent;  // the others: positions [lo, hi)
    const int lines = ((len + 63) / 64 + NW - 1) / NW;
    const int p0 = wave * lines * 64 + lane;
    uint32_t key[VPT];
#pragma unroll
    for (int r = 0; r < VPT; ++r) {
        const int pos = p0 + r * 64;
        key[r] = 0;
        if (r < lines && pos >= lo && pos < hi) key[r] = __builtin_bit_cast(uint32_t, w[pos]);
    }
#pragma unroll
    for (int r = 0; r < VPT; ++r) key[r] = weight_key(__builtin_bit_cast(float, key[r]));
    Search s;
    s.left = P.budget - P.sinks - P.recent;
    const bool search = s.left > 0;
    if (search) {
        for (int i = 0; i < kDigits; ++i) {
            clear_hist(lds);
            const int shift = digit_shift(i);
            const uint32_t bins = digit_bins(i) - 1;
#pragma unroll
            for (int r = 0; r < VPT; ++r) {
                const int pos = p0 + r * 64;
                if (r < lines) count_digit(lds.hist, pos >= lo && pos < hi && s.candidate(key[r]), (key[r] >> shift) & bins);
            }
            __syncthreads();
            if (take_digit_from_lds<NT>(lds, s, i)) break;
        }
    }
    int above = 0, same = 0;
#pragma unroll
    for (int r = 0; r < VPT; ++r) {
        const int pos = p0 + r * 64;
        if (r < lines) {
            const bool other = pos >= lo && pos < hi;
            above += __popcll(__ballot(pos < len && (!other || (search && s.above(key[r])))));
            same += __popcll(__ballot(other && search && s.candidate(key[r])));
        }
    }
    if (lane == 0) {
        n_above[wave] = above;
        n_same[wave] = same;
    }
    __syncthreads();
    Writer out{keep, 0, 0};
    for (int i = 0; i < wave; ++i) {
        out.at += n_above[i];
        out.same_before += n_same[i];
    }
    out.at += out.same_before < s.left ? out.same_before : s.left;
#pragma unroll
    for (int r = 0; r < VPT; ++r) {
        const int pos = p0 + r * 64;
        if (r < lines) {
            const bool other = pos >= lo && pos < hi;
            out.line(s, pos, pos < len && (!other || (search && s.above(key[r]))), other && search && s.candidate(key[r]));
        }
    }
}

// Longer rows are cut into chunks of kSelectChunk positions, a workgroup each, in three launches: the first leaves every chunk's
// histogram of the first digit; the second finds that digit from all of the row's, and leaves every chunk's candidates (the
// tokens that have it) and how many are above them; the third finds the rest from the candidates of all chunks, which every
// chunk's workgroup reads for itself, and writes its chunk.
constexpr int kChunkThreads = 1024, kChunkLines = kSelectChunk / kChunkThreads;
static_assert(kChunkLines * kChunkThreads == kSelectChunk, "whole lines");

struct ChunkRow {  // what a chunk's workgroup knows of its row
    int row, chunk, len, lo, hi, chunks;
    const float* w;
};
__device__ __forceinline__ ChunkRow chunk_row(const SelectParams& P) {
    ChunkRow c;
    c.row = blockIdx.x / P.max_chunks;
    c.chunk = blockIdx.x % P.max_chunks;
    c.len = P.length[c.row / P.Hkv];
    c.lo = P.sinks;
    c.hi = c.len - P.recent;
    c.chunks = (c.len + kSelectChunk - 1) / kSelectChunk;
    c.w = P.weights + (int64_t)c.row * P.weight_stride;
    return c;
}
// Keys of this thread's lines of the chunk, and which of them are others (neither first nor last ones).
__device__ __forceinline__ void chunk_keys(const ChunkRow& c, uint32_t (&key)[kChunkLines], bool (&other)[kChunkLines], int (&pos)[kChunkLines]) {
    const int p0 = c.chunk * kSelectChunk + (int)(threadIdx.x >> 6) * (kChunkLines * 64) + (int)(threadIdx.x & 63);
#pragma unroll
    for (int r = 0; r < kChunkLines; ++r) {
        pos[r] = p0 + r * 64;
        other[r] = pos[r] >= c.lo && pos[r] < c.hi;
        key[r] = other[r] ? __builtin_bit_cast(uint32_t, c.w[pos[r]]) : 0;
    }
#pragma unroll
    for (int r = 0; r < kChunkLines; ++r) key[r] = weight_key(__builtin_bit_cast(float, key[r]));
}
// The first digit, from the histograms of the row's chunks.
__device__ __forceinline__ bool first_digit(const SelectParams& P, const ChunkRow& c, SearchLds<kChunkThreads>& lds, Search& s) {
    constexpr int PER = kBins / kChunkThreads;
    uint32_t n[PER] = {};
    const uint32_t* h = P.hist + (int64_t)c.row * P.max_chunks * kBins + kBins - 1 - threadIdx.x * PER;
    for (int k = 0; k < c.chunks; ++k)
#pragma unroll
        for (int j = 0; j < PER; ++j) n[j] += h[(int64_t)k * kBins - j];
    return take_digit<kChunkThreads>(lds, s, 0, n);
}

__global__ __launch_bounds__(kChunkThreads) void ppd_select_digits_kernel(const SelectParams P) {
    __shared__ SearchLds<kChunkThreads> lds;
    const ChunkRow c = chunk_row(P);
    if (c.chunk >= c.chunks || c.len <= P.budget || P.budget == P.sinks + P.recent) return;
    uint32_t key[kChunkLines];
    bool other[kChunkLines];
    int pos[kChunkLines];
    chunk_keys(c, key, other, pos);
    clear_hist(lds);
#pragma unroll
    for (int r = 0; r < kChunkLines; ++r) count_digit(lds.hist, other[r], key[r] >> digit_shift(0));
    __syncthreads();
    uint32_t* h = P.hist + ((int64_t)c.row * P.max_chunks + c.chunk) * kBins;
    for (int i = threadIdx.x; i < kBins; i += kChunkThreads) h[i] = lds.hist[i];
}

__global__ __launch_bounds__(kChunkThreads) void ppd_select_candidates_kernel(const SelectParams P) {
    constexpr int NW = kChunkThreads / 64;
    __shared__ SearchLds<kChunkThreads> lds;
    __shared__ int n_above[NW], n_same[NW];
    const ChunkRow c = chunk_row(P);
    if (c.chunk >= c.chunks || c.len <= P.budget) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Search s;
    s.left = P.budget - P.sinks - P.recent;
    const bool search = s.left > 0;
    uint32_t key[kChunkLines];
    bool other[kChunkLines];
    int pos[kChunkLines];
    chunk_keys(c, key, other, pos);
    if (search) first_digit(P, c, lds, s);
    int above = 0, same = 0;
#pragma unroll
    for (int r = 0; r < kChunkLines; ++r) {
        above += __popcll(__ballot(pos[r] < c.len && (!other[r] || (search && s.above(key[r])))));
        same += __popcll(__ballot(other[r] && search && s.candidate(key[r])));
    }
    if (lane == 0) {
        n_above[wave] = above;
        n_same[wave] = same;
    }
    __syncthreads();
    int at = 0;
    for (int i = 0; i < wave; ++i) at += n_same[i];
    const int64_t mine = (int64_t)c.row * P.max_chunks + c.chunk;
    uint32_t* list = P.candidates + mine * kSelectChunk;
#pragma unroll
    for (int r = 0; r < kChunkLines; ++r) {
        const bool cand = other[r] && search && s.candidate(key[r]);
        const uint64_t m = __ballot(cand);
        if (cand) list[at + __popcll(m & ((1ull << lane) - 1))] = key[r];
        at += __popcll(m);
    }
    if (threadIdx.x == 0) {
        int total_above = 0, total_same = 0;
        for (int i = 0; i < NW; ++i) {
            total_above += n_above[i];
            total_same += n_same[i];
        }
        P.counts[mine * 2] = total_above;
        P.counts[mine * 2 + 1] = total_same;
    }
}

__global__ __launch_bounds__(kChunkThreads) void ppd_select_finish_kernel(const SelectParams P) {
    constexpr int NW = kChunkThreads / 64;
    __shared__ SearchLds<kChunkThreads> lds;
    __shared__ int n_above[NW], n_same[NW], before[2];
    const ChunkRow c = chunk_row(P);
    if (c.chunk >= c.chunks) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t* keep = P.keep + (int64_t)c.row * P.keep_stride;
    if (c.len <= P.budget) {
        for (int t = c.chunk * kSelectChunk + tid; t < c.len && t < (c.chunk + 1) * kSelectChunk; t += kChunkThreads) keep[t] = t;
        return;
    }
    Search s;
    s.left = P.budget - P.sinks - P.recent;
    const bool search = s.left > 0;
    uint32_t key[kChunkLines];
    bool other[kChunkLines];
    int pos[kChunkLines];
    chunk_keys(c, key, other, pos);
    const int64_t first = (int64_t)c.row * P.max_chunks;
    bool all = !search || first_digit(P, c, lds, s);
    auto each_candidate = [&](int chunks, auto f) {  // f(live, key) for the candidates of the first `chunks` chunks, by whole waves
        for (int k = 0; k < chunks; ++k) {
            const int n = P.counts[(first + k) * 2 + 1];
            const uint32_t* list = P.candidates + (first + k) * kSelectChunk;
            for (int i = wave * 64; i < n; i += kChunkThreads) f(i + lane < n, i + lane < n ? list[i + lane] : 0u);
        }
    };
    for (int i = 1; i < kDigits && !all; ++i) {
        clear_hist(lds);
        const int shift = digit_shift(i);
        const uint32_t bins = digit_bins(i) - 1;
        each_candidate(c.chunks, [&](bool live, uint32_t k) { count_digit(lds.hist, live && s.candidate(k), (k >> shift) & bins); });
        __syncthreads();
        all = take_digit_from_lds<kChunkThreads>(lds, s, i);
    }
    // how many are chosen for certain, and how many have the last weight, in the chunks in front: counted above the first digit there, the
    // rest among their candidates
    if (tid < 2) before[tid] = 0;
    __syncthreads();
    {
        int above = 0, same = 0;
        if (search)
            each_candidate(c.chunk, [&](bool live, uint32_t k) {
                above += __popcll(__ballot(live && s.above(k)));
                same += __popcll(__ballot(live && s.candidate(k)));
            });
        if (tid < c.chunk) atomicAdd(&before[0], P.counts[(first + tid) * 2]);
        for (int k = tid + kChunkThreads; k < c.chunk; k += kChunkThreads) atomicAdd(&before[0], P.counts[(first + k) * 2]);
        if (lane == 0 && above) atomicAdd(&before[0], above);
        if (lane == 0 && same) atomicAdd(&before[1], same);
    }
    int above = 0, same = 0;
#pragma unroll
    for (int r = 0; r < kChunkLines; ++r) {
        above += __popcll(__ballot(pos[r] < c.len && (!other[r] || (search && s.above(key[r])))));
        same += __popcll(__ballot(other[r] && search && s.candidate(key[r])));
    }
    if (lane == 0) {
        n_above[wave] = above;
        n_same[wave] = same;
    }
    __syncthreads();
    Writer out{keep, before[0], before[1]};
    for (int i = 0; i < wave; ++i) {
        out.at += n_above[i];
        out.same_before += n_same[i];
    }
    out.at += out.same_before < s.left ? out.same_before : s.left;
#pragma unroll
    for (int r = 0; r < kChunkLines; ++r)
        out.line(s, pos[r], pos[r] < c.len && (!other[r] || (search && s.above(key[r]))), other[r] && search && s.candidate(key[r]));
}

int launch_select(const SelectParams& p, int longest, void* stream) {
    hipStream_t hs = static_cast<hipStream_t>(stream);
    if (p.max_chunks > 0) {
        const dim3 grid((unsigned)(p.B * p.Hkv * p.max_chunks));
        hipLaunchKernelGGL(ppd_select_digits_kernel, grid, dim3(kChunkThreads), 0, hs, p);
        hipLaunchKernelGGL(ppd_select_candidates_kernel, grid, dim3(kChunkThreads), 0, hs, p);
        hipLaunchKernelGGL(ppd_select_finish_kernel, grid, dim3(kChunkThreads), 0, hs, p);
        return (int)hipGetLastError();
    }
    const dim3 grid((unsigned)p.Hkv, (unsigned)p.B);
    if (longest <= 256 * 8) hipLaunchKernelGGL((ppd_select_kernel<256, 8>), grid, dim3(256), 0, hs, p);
    else if (longest <= 1024 * 8) hipLaunchKernelGGL((ppd_select_kernel<1024, 8>), grid, dim3(1024), 0, hs, p);
    else hipLaunchKernelGGL((ppd_select_kernel<1024, kSelectChunk / 1024>), grid, dim3(1024), 0, hs, p);
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
