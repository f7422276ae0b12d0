// gfx950 kernels of cache eviction: the choice of the tokens to keep by their weight, and the move of kept tokens to the front.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ppd_device.h"
#include "ppd_ops.h"

namespace ppd {

namespace {

// A weight's bits as an integer of the same order: larger for the heavier one.  Both zeros are equal, NaN is heavier than all else.
// The lightest, negative infinity, is 0x007fffff; kNoKey is below all and kHeldKey above.
constexpr uint32_t kNoKey = 0, kHeldKey = ~0u, kNanKey = ~0u - 1;
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return kNanKey;
    const uint32_t b = w == 0.f ? 0u : __builtin_bit_cast(uint32_t, w);
    return b >> 31 ? ~b : b | 0x80000000u;
}

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // from the lane 1, 2, 4, 8 to the left within 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 to the next 16 lanes
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to the upper half
    return x;
}

__device__ __forceinline__ int lanes_below(uint64_t m) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0)); }

}  // namespace

// ---- the choice ---------------------------------------------------------------------------------------------
// The first and the last tokens get the heaviest key, so that the choice is the `budget` heaviest of all, the lower position first
// where keys are equal.  The key of the last chosen token is found from a histogram over its upper 11 bits, in LDS, which leaves few
// candidates, and from their ranks among one another (or two more histograms, where they are many).  `prefix` holds the bits found
// so far in the places of `mask`, `left` how many of the tokens with these bits are chosen.
// Bound by instructions and barriers, not by the weights: a workgroup's steps behind one another take about 4 us.
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
    static constexpr int kList = 64;  // candidates that are ranked, at most
    uint32_t hist[kBins];
    __attribute__((aligned(16))) uint32_t list[kList];
    uint32_t wave_sum[NT / 64];
    uint32_t listed;
    uint32_t found[3];  // digit, tokens above it, tokens of it
};

// Sum of the values of the waves in front.
template <int NT>
__device__ __forceinline__ uint32_t sum_before(const uint32_t (&v)[NT / 64], int wave) {
    static_assert(NT <= 1024, "the waves' values fit a row of 16 lanes");
    const int lane = threadIdx.x & 63;
    uint32_t x = lane < NT / 64 && lane < wave ? v[lane & (NT / 64 - 1)] : 0u;
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    return __builtin_amdgcn_readlane(x, 15);
}

// Thread t has the bins kBins - 1 - t * PER .. (heaviest first); the one in which the running count reaches `left` is the digit.  All threads
// call it, with the histogram complete.  Returns how many tokens have the digit.
template <int NT>
__device__ __forceinline__ int take_digit(SearchLds<NT>& lds, Search& s, int i, const uint32_t (&n)[kBins / NT]) {
    constexpr int PER = kBins / NT;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t mine = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) mine += n[j];
    const uint32_t upto = wave_scan(mine);
    if (lane == 63) lds.wave_sum[wave] = upto;
    __syncthreads();
    uint32_t before = upto - mine + sum_before<NT>(lds.wave_sum, wave);
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
    return (int)lds.found[2];
}

template <int NT>
__device__ __forceinline__ int take_digit_from_lds(SearchLds<NT>& lds, Search& s, int i) {
    constexpr int PER = kBins / NT;
    uint32_t n[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) n[j] = lds.hist[kBins - 1 - (threadIdx.x * PER + j)];
    return take_digit<NT>(lds, s, i, n);
}

template <int NT>
__device__ __forceinline__ void clear_hist(SearchLds<NT>& lds) {
    for (int i = threadIdx.x; i < kBins; i += NT) lds.hist[i] = 0;
    if (threadIdx.x == 0) lds.listed = 0;
    __syncthreads();
}

// Adds the digits of a wave's live lanes to the histogram.  Lanes that share a bin take their turns in LDS, and keys crowd: the held ones
// are all equal, weights next to nothing are in few bins.  The first live lane counts for all that have its bin (histograms of 24
// rows of 40K-131K tokens 16.6 us without that, 6.8 with it).
template <int NT>
__device__ __forceinline__ void count_digit(SearchLds<NT>& lds, bool live, uint32_t digit) {
    const uint64_t all = __ballot(live);
    if (!all) return;
    const int lane = threadIdx.x & 63, first = __builtin_ctzll(all);
    const uint32_t common = __builtin_amdgcn_readlane(digit, first);
    const uint64_t same = __ballot(live && digit == common);
    if (lane == first || (live && digit != common)) atomicAdd(&lds.hist[digit], lane == first ? (uint32_t)__popcll(same) : 1u);
}

// The rest of the search, when `count` tokens have the bits found so far, over the keys that each thread holds.
template <int NT, int VPT>
__device__ __forceinline__ void finish_search(SearchLds<NT>& lds, Search& s, int count, const uint32_t (&key)[VPT], int lines) {
    const int tid = threadIdx.x, lane = tid & 63;
    for (int i = 1; i < kDigits && count != s.left && count > SearchLds<NT>::kList; ++i) {
        clear_hist(lds);
        const int shift = digit_shift(i);
        const uint32_t bins = digit_bins(i) - 1;
#pragma unroll
        for (int r = 0; r < VPT; ++r)
            if (r < lines) count_digit(lds, s.candidate(key[r]), (key[r] >> shift) & bins);
        __syncthreads();
        count = take_digit_from_lds<NT>(lds, s, i);
    }
    if (count == s.left || s.mask == ~0u) return;  // all of them are chosen, or they are all equal
    // Few are left: each one's rank among them.  The one with fewer than `left` above it and at least as many not below it is the last
    // chosen.
    uint32_t mine = 0;
#pragma unroll
    for (int r = 0; r < VPT; ++r) mine += (uint32_t)__popcll(__ballot(s.candidate(key[r])));
    uint32_t at = 0;
    if (lane == 0 && mine) at = atomicAdd(&lds.listed, mine);
    at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
    for (int r = 0; r < VPT; ++r) {
        const bool c = s.candidate(key[r]);
        const uint64_t m = __ballot(c);
        if (c) lds.list[at + lanes_below(m)] = key[r];
        at += (uint32_t)__popcll(m);
    }
    const int padded = (count + 3) & ~3;
    if (tid < padded - count) lds.list[count + tid] = kNoKey;
    __syncthreads();
    if (tid < count) {
        const uint32_t k = lds.list[tid];
        int above = 0, same = 0;
#pragma unroll 4
        for (int j = 0; j < padded; j += 4) {
            const u32x4 o = *reinterpret_cast<const u32x4*>(&lds.list[j]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                above += o[e] > k;
                same += o[e] == k;
            }
        }
        if (above < s.left && above + same >= s.left) {  // every one with this key writes the same
            lds.found[0] = k;
            lds.found[1] = (uint32_t)above;
        }
    }
    __syncthreads();
    s.prefix = lds.found[0];
    s.mask = ~0u;
    s.left -= (int)lds.found[1];
}

// A line is 64 neighbouring positions, a lane each; a wave has VPT of them from position p0 - lane on.  Writes the wave's chosen tokens in
// order: `chosen` and `same_before` are how many come in front of them for certain and how many have the last key there.
template <int NT, int VPT>
__device__ __forceinline__ void write_chosen(SearchLds<NT>& lds, const Search& s, const uint32_t (&key)[VPT], int p0, int chosen, int same_before, int32_t* keep) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint64_t above[VPT], same[VPT];
    uint32_t n_above = 0, n_same = 0;
#pragma unroll
    for (int r = 0; r < VPT; ++r) {
        above[r] = __ballot(s.above(key[r]));
        same[r] = __ballot(s.candidate(key[r]));
        n_above += (uint32_t)__popcll(above[r]);
        n_same += (uint32_t)__popcll(same[r]);
    }
    static_assert(NT * VPT <= 65535, "both counts fit a word");
    if (lane == 0) lds.wave_sum[wave] = n_above | n_same << 16;
    __syncthreads();
    const uint32_t front = sum_before<NT>(lds.wave_sum, wave);
    same_before += (int)(front >> 16);
    int at = chosen + (int)(front & 0xFFFFu) + (same_before < s.left ? same_before : s.left);
#pragma unroll
    for (int r = 0; r < VPT; ++r) {
        uint64_t m = same[r];
        const int n = __popcll(m);
        if (same_before + n > s.left) m = __ballot(__builtin_amdgcn_inverse_ballot_w64(same[r]) && same_before + lanes_below(same[r]) < s.left);
        same_before += n;
        m |= above[r];
        if (__builtin_amdgcn_inverse_ballot_w64(m)) keep[at + lanes_below(m)] = p0 + r * 64;
        at += __popcll(m);
    }
}

// Keys of a thread's lines, from position p0 on.
template <int VPT>
__device__ __forceinline__ void load_keys(const float* w, int len, int sinks, int recent, int p0, int lines, uint32_t (&key)[VPT]) {
    float v[VPT];
#pragma unroll
    for (int r = 0; r < VPT; ++r) {
        const int pos = p0 + r * 64;
        v[r] = 0.f;
        if (r < lines && pos < len) v[r] = w[pos];
    }
#pragma unroll
    for (int r = 0; r < VPT; ++r) {
        const int pos = p0 + r * 64;
        key[r] = r >= lines || pos >= len ? kNoKey : pos < sinks || pos >= len - recent ? kHeldKey : weight_key(v[r]);
    }
}

// One workgroup to a sequence and KV head, whose weights it reads once and holds in registers: wave w has the lines w * lines ..
// (w + 1) * lines - 1, at most VPT of them.
template <int NT, int VPT>
__global__ __launch_bounds__(NT) void ppd_select_kernel(const SelectParams P) {
    __shared__ SearchLds<NT> lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = blockIdx.y, head = blockIdx.x, len = P.length[b];
    const float* w = P.weights + ((int64_t)b * P.Hkv + head) * P.weight_stride;
    int32_t* keep = P.keep + ((int64_t)b * P.Hkv + head) * P.keep_stride;
    if (len <= P.budget) {
        for (int t = tid; t < len; t += NT) keep[t] = t;
        return;
    }
    const int lines = ((len + 63) / 64 + NT / 64 - 1) / (NT / 64);
    const int p0 = wave * lines * 64 + lane;
    uint32_t key[VPT];
    load_keys(w, len, P.sinks, P.recent, p0, lines, key);
    Search s;
    s.left = P.budget;
    clear_hist(lds);
#pragma unroll
    for (int r = 0; r < VPT; ++r)
        if (r < lines) count_digit(lds, true, key[r] >> digit_shift(0));
    __syncthreads();
    const int count = take_digit_from_lds<NT>(lds, s, 0);
    finish_search(lds, s, count, key, lines);
    write_chosen(lds, s, key, p0, 0, 0, keep);
}

// Longer rows are cut into chunks of kSelectChunk positions, a workgroup each, in three launches: the first leaves every chunk's
// histogram of the upper bits; the second finds the bits from all of the row's, and leaves the row's candidates (the tokens that
// have them) and how many are above them in every chunk; the third finds the rest from the candidates, which every chunk's
// workgroup reads for itself, and writes its chunk.
constexpr int kChunkThreads = 1024, kChunkLines = kSelectChunk / kChunkThreads;
static_assert(kChunkLines * kChunkThreads == kSelectChunk, "whole lines");

struct ChunkRow {  // what a chunk's workgroup knows of its row
    int row, chunk, len, chunks, p0;
    const float* w;
    int32_t* counts;  // the row's: candidates, the bits found, how many are chosen of them; then per chunk how many are above
};
__device__ __forceinline__ ChunkRow chunk_row(const SelectParams& P) {
    ChunkRow c;
    c.row = blockIdx.x / P.max_chunks;
    c.chunk = blockIdx.x % P.max_chunks;
    c.len = P.length[c.row / P.Hkv];
    c.chunks = (c.len + kSelectChunk - 1) / kSelectChunk;
    c.p0 = c.chunk * kSelectChunk + (int)(threadIdx.x >> 6) * (kChunkLines * 64) + (int)(threadIdx.x & 63);
    c.w = P.weights + (int64_t)c.row * P.weight_stride;
    c.counts = P.counts + (int64_t)c.row * (P.max_chunks + kSelectRowWords);
    return c;
}

__global__ __launch_bounds__(kChunkThreads) void ppd_select_digits_kernel(const SelectParams P) {
    __shared__ SearchLds<kChunkThreads> lds;
    const ChunkRow c = chunk_row(P);
    if (c.chunk >= c.chunks || c.len <= P.budget) return;
    uint32_t key[kChunkLines];
    load_keys(c.w, c.len, P.sinks, P.recent, c.p0, kChunkLines, key);
    clear_hist(lds);
#pragma unroll
    for (int r = 0; r < kChunkLines; ++r) count_digit(lds, true, key[r] >> digit_shift(0));
    if (c.chunk == 0 && threadIdx.x == 0) c.counts[0] = 0;
    __syncthreads();
    uint32_t* h = P.hist + ((int64_t)c.row * P.max_chunks + c.chunk) * kBins;
    for (int i = threadIdx.x; i < kBins; i += kChunkThreads) h[i] = lds.hist[i];
}

__global__ __launch_bounds__(kChunkThreads) void ppd_select_candidates_kernel(const SelectParams P) {
    constexpr int PER = kBins / kChunkThreads;
    __shared__ SearchLds<kChunkThreads> lds;
    __shared__ int above, same, list_at;
    const ChunkRow c = chunk_row(P);
    if (c.chunk >= c.chunks || c.len <= P.budget) return;
    const int lane = threadIdx.x & 63;
    uint32_t key[kChunkLines];
    load_keys(c.w, c.len, P.sinks, P.recent, c.p0, kChunkLines, key);
    Search s;
    s.left = P.budget;
    uint32_t n[PER] = {};
    const uint32_t* h = P.hist + (int64_t)c.row * P.max_chunks * kBins + kBins - 1 - threadIdx.x * PER;
#pragma unroll 4
    for (int k = 0; k < c.chunks; ++k)
#pragma unroll
        for (int j = 0; j < PER; ++j) n[j] += h[(int64_t)k * kBins - j];
    if (threadIdx.x == 0) above = same = 0;
    const int count = take_digit<kChunkThreads>(lds, s, 0, n);
    int n_above = 0, n_same = 0;
#pragma unroll
    for (int r = 0; r < kChunkLines; ++r) {
        n_above += __popcll(__ballot(s.above(key[r])));
        n_same += __popcll(__ballot(s.candidate(key[r])));
    }
    int at = 0;
    if (lane == 0) {
        atomicAdd(&above, n_above);
        at = atomicAdd(&same, n_same);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        list_at = atomicAdd(&c.counts[0], same);  // the candidates' order does not matter
        c.counts[kSelectRowWords + c.chunk] = above;
        if (c.chunk == 0) {
            c.counts[1] = (int)s.prefix;
            c.counts[2] = s.left;
            c.counts[3] = count;
        }
    }
    __syncthreads();
    at = __builtin_amdgcn_readfirstlane(at) + list_at;
    u32x2* list = reinterpret_cast<u32x2*>(P.candidates) + (int64_t)c.row * P.max_chunks * kSelectChunk;
#pragma unroll
    for (int r = 0; r < kChunkLines; ++r) {
        const bool cand = s.candidate(key[r]);
        const uint64_t m = __ballot(cand);
        if (cand) list[at + lanes_below(m)] = u32x2{key[r], (uint32_t)c.chunk};
        at += __popcll(m);
    }
}

__global__ __launch_bounds__(kChunkThreads) void ppd_select_finish_kernel(const SelectParams P) {
    __shared__ SearchLds<kChunkThreads> lds;
    __shared__ int before[2];
    const ChunkRow c = chunk_row(P);
    if (c.chunk >= c.chunks) return;
    const int tid = threadIdx.x, lane = tid & 63;
    int32_t* keep = P.keep + (int64_t)c.row * P.keep_stride;
    if (c.len <= P.budget) {
        for (int t = c.chunk * kSelectChunk + tid; t < c.len && t < (c.chunk + 1) * kSelectChunk; t += kChunkThreads) keep[t] = t;
        return;
    }
    Search s;
    s.prefix = (uint32_t)c.counts[1];
    s.mask = (uint32_t)(digit_bins(0) - 1) << digit_shift(0);
    s.left = c.counts[2];
    int count = c.counts[3];
    uint32_t key[kChunkLines];
    load_keys(c.w, c.len, P.sinks, P.recent, c.p0, kChunkLines, key);
    const u32x2* list = reinterpret_cast<const u32x2*>(P.candidates) + (int64_t)c.row * P.max_chunks * kSelectChunk;
    const int total = count;
    // the candidates, kChunkLines to a thread where they fit, or again and again from the list
    uint32_t cand[kChunkLines];
    uint64_t front[kChunkLines];  // which of them are in chunks in front of this one
    const bool held = total <= kSelectChunk;
    const int lines = held ? (total + kChunkThreads - 1) / kChunkThreads : 0;
#pragma unroll
    for (int r = 0; r < kChunkLines; ++r) {
        const int i = r * kChunkThreads + tid;
        u32x2 v = {kNoKey, ~0u};
        if (r < lines && i < total) v = list[i];
        cand[r] = v[0];
        front[r] = __ballot(v[1] < (uint32_t)c.chunk);
    }
    if (tid < 2) before[tid] = 0;
    if (tid == 0) lds.listed = 0;
    __syncthreads();
    if (held) {
        finish_search(lds, s, count, cand, lines);
    } else {
        for (int i = 1; i < kDigits && count != s.left; ++i) {
            clear_hist(lds);
            for (int t0 = tid - lane; t0 < total; t0 += kChunkThreads) {
                const uint32_t k = t0 + lane < total ? list[t0 + lane][0] : kNoKey;
                count_digit(lds, s.candidate(k), (k >> digit_shift(i)) & (digit_bins(i) - 1));
            }
            __syncthreads();
            count = take_digit_from_lds<kChunkThreads>(lds, s, i);
        }
    }
    __syncthreads();
    // how many are chosen for certain, and how many have the last key, in the chunks in front: those above the upper bits were counted there,
    // the rest is among the candidates
    int above = 0, same = 0;
    if (held) {
#pragma unroll
        for (int r = 0; r < kChunkLines; ++r) {
            if (r >= lines) continue;
            above += __popcll(__ballot(s.above(cand[r])) & front[r]);
            same += __popcll(__ballot(s.candidate(cand[r])) & front[r]);
        }
    } else {
        for (int t0 = tid - lane; t0 < total; t0 += kChunkThreads) {
            const u32x2 v = t0 + lane < total ? list[t0 + lane] : u32x2{kNoKey, ~0u};
            above += __popcll(__ballot(v[1] < (uint32_t)c.chunk && s.above(v[0])));
            same += __popcll(__ballot(v[1] < (uint32_t)c.chunk && s.candidate(v[0])));
        }
    }
    if (lane == 0 && above) atomicAdd(&before[0], above);
    if (lane == 0 && same) atomicAdd(&before[1], same);
    for (int k = tid; k < c.chunk; k += kChunkThreads) atomicAdd(&before[0], c.counts[kSelectRowWords + k]);
    __syncthreads();
    const int chosen = before[0], same_before = before[1];
    write_chosen(lds, s, key, c.p0, chosen, same_before, keep);
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
    // The fewest threads that hold the longest row, eight weights each before sixteen.  Rows of 2048, 8 KV heads: 256 threads 6.4, 7.3 and 12.2 us for
    // 1, 64 and 256 sequences, 1024 threads 6.0, 9.1 and 27.  Rows of 8192: eight weights a thread 7.1, 12.2 and 37 us, sixteen 8.4, 18.5 and 63.
    const dim3 grid((unsigned)p.Hkv, (unsigned)p.B);
    if (longest <= 256 * 8) hipLaunchKernelGGL((ppd_select_kernel<256, 8>), grid, dim3(256), 0, hs, p);
    else if (longest <= 1024 * 8) hipLaunchKernelGGL((ppd_select_kernel<1024, 8>), grid, dim3(1024), 0, hs, p);
    else hipLaunchKernelGGL((ppd_select_kernel<1024, kSelectChunk / 1024>), grid, dim3(1024), 0, hs, p);
    return (int)hipGetLastError();
}

// ---- the move -----------------------------------------------------------------------------------------------
// Token keep[i] of a sequence, KV head and layer goes to position first + i, in place.  The lists ascend and keep[i] >= first + i, so a
// destination is never read by a later token: a workgroup takes kMoves destinations at a time -- `P.step` positions of as many heads as
// that leaves room for -- reads all of them, waits, and writes.  Every d is independent, so K, V and slices of d are workgroups of their
// own; the weights are another.  Entries that do not ascend or lie outside the sequence's pages raise the sticky flag, and their
// tokens stay where they are.
// Bound by memory, in whole lines of 128 bytes: a line of K is 8 d of 8 tokens (of 16 on FP8 pages), a line of V 8 tokens of 8 d, and both
// are read for one token as for all.  32 evictions from 1K-8K to 1024 tokens, every head its own: for 135 MB of kept tokens 392 MB are
// read and 135 MB written (counters), 131 us, 4.0 TB/s, where a large copy reaches 4.9; called again on the same pool, part of which
// the memory side still holds, 108 us.  FP8 pages: 216 and 68 MB, 70 us.  The accepted paths of 16 trees over 32 layers: for 11 MB
// 56 MB read and 19 MB written, 23 us (FP8: 35 and 10 MB, 16 us).  Short lists are a chain of reads -- list, page, token -- so there
// one workgroup takes all heads.
constexpr int kCompactThreads = 256, kMoves = 128, kUnits = 4;  // units (granules) a thread moves at a time
constexpr int kTogether = 2;  // granules of V whose sources a wave asks for at once
constexpr int kCompactWidth = kUnits * kCompactThreads * 8 / kMoves;  // d of a slice

// Workgroup barrier that leaves reads of the next step's lists on their way; what has to be there is waited for before it.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int HD, bool FP8>
__global__ __launch_bounds__(kCompactThreads) void ppd_compact_kernel(const CompactParams P) {
    typedef std::conditional_t<FP8, uint8_t, uint16_t> Elem;
    typedef std::conditional_t<FP8, u32x2, u32x4> Raw;  // eight elements
    constexpr int WIDTH = kCompactWidth, SLICES = HD / WIDTH;
    static_assert(WIDTH == 64 && kMoves / 8 == kUnits * kCompactThreads / 64, "a wave moves a granule of V of 64 d at a time");
    __shared__ int64_t from[kMoves], to[kMoves];  // element offset of a move's page block, -1: it stays
    __shared__ int from_tok[kMoves], to_tok[kMoves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int heads = kMoves / P.step, groups = (P.Hkv + heads - 1) / heads;
    const int b = blockIdx.x / groups, head0 = blockIdx.x % groups * heads, layer = blockIdx.z;
    const int first = P.first[b], end = first + P.count[b];
    // Weights first (a step of theirs is as long a chain as the others', and they are few: started last they would end last), K slices, V slices.
    const int part = (int)blockIdx.y - (P.weights ? 1 : 0);
    const bool is_weights = part < 0, is_v = part >= SLICES;
    const int d0 = (is_weights ? 0 : part % SLICES) * WIDTH;
    const int32_t* pages = P.page_tables + (int64_t)b * P.max_pages;
    int64_t capacity = (int64_t)P.max_pages * kPage;
    if (P.weights && P.weight_stride < capacity) capacity = P.weight_stride;
    // thread t < kMoves looks up move t: position p0 + t % step of head head0 + t / step
    const int head = head0 + tid / P.step;
    const bool looks = tid < kMoves && head < P.Hkv;
    const int32_t* keep = P.keep + layer * P.keep_layer + b * P.keep_seq + (looks ? head : head0) * P.keep_head;
    float* const weights = P.weights ? P.weights + layer * P.weight_layer + ((int64_t)b * P.Hkv + (looks ? head : head0)) * P.weight_stride : nullptr;
    Elem* const pool = static_cast<Elem*>(P.pool) + layer * P.pool_layer + (is_v ? (int64_t)P.Hkv * (kPage * HD) : 0);

    // Looking a move up is a chain of two reads, the list and the page table, which run ahead of the data by a step: `want` holds the
    // list's entries of the next step, `pages_of` their pages.
    struct Move { int pos, src, previous, from_id, to_id; };
    auto ask_list = [&](int p0, Move& m) {
        m.pos = p0 + tid % P.step;
        const int i = m.pos - first;
        m.src = -1;
        m.previous = -1;
        if (looks && i >= 0 && m.pos < end) {
            m.src = keep[i];
            if (i > 0) m.previous = keep[i - 1];
        }
    };
    auto ask_pages = [&](Move& m) {
        const int i = m.pos - first;
        const bool listed = looks && i >= 0 && m.pos < end;
        if (listed && (m.src < m.pos || m.src >= capacity || m.previous >= m.src)) {
            atomicOr(P.err_flags, 8u);
            m.src = -1;
        }
        m.from_id = m.to_id = 0;
        if (m.src >= 0) {
            m.from_id = pages[m.src >> 4];
            m.to_id = pages[m.pos >> 4];
        }
    };

    const int start = first & ~7;  // steps begin on a granule of V
    Move m;
    ask_list(start, m);
    ask_pages(m);
    for (int p0 = start; p0 < end; p0 += P.step) {
        if (m.src >= 0 && ((uint32_t)m.from_id >= (uint64_t)P.num_pages || (uint32_t)m.to_id >= (uint64_t)P.num_pages)) {
            atomicOr(P.err_flags, 2u);
            m.src = -1;
        }
        if (is_weights) {  // a weight stays where its token stays
            const int src = m.src, pos = m.pos;
            float v = 0.f;
            if (src >= 0) v = weights[src];
            ask_list(p0 + P.step, m);
            asm volatile("s_waitcnt vmcnt(0)" : "+v"(v) : : "memory");
            ask_pages(m);
            lds_barrier();
            if (src >= 0) weights[pos] = v;
            continue;
        }
        __syncthreads();  // the lists of the step before are read
        if (tid < kMoves) {
            from[tid] = m.src < 0 ? -1 : m.from_id * P.page_stride + head * (kPage * HD);
            to[tid] = m.src < 0 ? -1 : m.to_id * P.page_stride + head * (kPage * HD);
            from_tok[tid] = m.src & 15;
            to_tok[tid] = m.pos & 15;
        }
        __syncthreads();
        ask_list(p0 + P.step, m);
        if (!is_v) {
            Raw v[kUnits];
#pragma unroll
            for (int j = 0; j < kUnits; ++j) {
                const int u = tid + j * kCompactThreads, k = u % kMoves, g = d0 / 8 + u / kMoves;
                v[j] = Raw{};
                if (from[k] >= 0) v[j] = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(pool + from[k] + (g * kPage + from_tok[k]) * 8));
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            ask_pages(m);
            lds_barrier();
#pragma unroll
            for (int j = 0; j < kUnits; ++j) {
                const int u = tid + j * kCompactThreads, k = u % kMoves, g = d0 / 8 + u / kMoves;
                if (to[k] >= 0) __builtin_nontemporal_store(v[j], reinterpret_cast<Raw*>(pool + to[k] + (g * kPage + to_tok[k]) * 8));
            }
        } else {
            // A wave takes a granule of destinations and 64 d, so that where its eight tokens come from is the same for all lanes.  A
            // source granule is read once, whole, for all of the tokens in it (an element at a time the lanes asked for lines that
            // were still on their way, and 32 evictions from 1K-8K to 1024 tokens took 203 us, this way 151).
            Raw v[kUnits];
            // lane 8 j + e has the move of element e of the wave's granule j; `fresh`: not out of the granule that the element before is from
            const int my_move = (wave + (lane >> 3) % kUnits * (kCompactThreads / 64)) * 8 + (lane & 7);
            const uint64_t my_to = (uint64_t)to[my_move];
            const int my_from_tok = from_tok[my_move], my_to_tok = to_tok[my_move];
            const uint64_t my_from = (uint64_t)(from[my_move] + (my_from_tok >> 3) * (HD * 8));
            const uint64_t moving = __ballot((int64_t)my_to >= 0);
            const uint32_t before_lo = __shfl_up((uint32_t)my_from, 1, 64), before_hi = __shfl_up((uint32_t)(my_from >> 32), 1, 64);
            const bool same = (lane & 7) != 0 && (moving >> (lane - 1) & 1) && before_lo == (uint32_t)my_from && before_hi == (uint32_t)(my_from >> 32);
            const uint64_t fresh = moving & ~__ballot(same);
            auto of_lane = [&](uint64_t x, int l) {
                return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, l);
            };
#pragma unroll
            for (int j0 = 0; j0 < kUnits; j0 += kTogether) {
                Raw r[kTogether][8];  // of the fresh ones
#pragma unroll
                for (int j = 0; j < kTogether; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int l = (j0 + j) * 8 + e;
                        r[j][e] = Raw{};
                        if (fresh >> l & 1) r[j][e] = *reinterpret_cast<const Raw*>(pool + (int64_t)of_lane(my_from, l) + (d0 + lane) * 8);
                    }
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                if (j0 == 0) ask_pages(m);
                uint64_t taken = fresh;
                asm volatile("" : "+s"(taken));  // not to be merged with the branches above
#pragma unroll
                for (int j = 0; j < kTogether; ++j) {
                    Raw cur = {};
                    v[j0 + j] = Raw{};
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        constexpr int PW = 4 / (int)sizeof(Elem);  // elements of a word
                        const int l = (j0 + j) * 8 + e, tok = __builtin_amdgcn_readlane(my_from_tok, l) & 7;
                        const bool takes = taken >> l & 1;
#pragma unroll
                        for (int i = 0; i < (int)(sizeof(Raw) / 4); ++i) cur[i] = takes ? r[j][e][i] : cur[i];
                        uint32_t w = cur[0];
#pragma unroll
                        for (int i = 1; i < (int)(sizeof(Raw) / 4); ++i) w = tok / PW == i ? cur[i] : w;
                        w = (w >> (tok % PW * (int)sizeof(Elem) * 8)) & (Elem)~(Elem)0;
                        v[j0 + j][e / PW] |= w << (e % PW * (int)sizeof(Elem) * 8);
                    }
                    asm volatile("" : "+v"(v[j0 + j]) : : "memory");  // taken apart before the next ones are asked for: registers
                }
            }
            lds_barrier();
#pragma unroll
            for (int j = 0; j < kUnits; ++j) {
                const uint32_t places = moving >> (j * 8) & 255u;  // the granule's eight places are neighbours in one page
                if (places == 0) continue;
                const int l = j * 8 + __builtin_ctz(places);
                Elem* const at = pool + (int64_t)of_lane(my_to, l) + (__builtin_amdgcn_readlane(my_to_tok, l) >> 3) * (HD * 8);
                if (places == 255) {
                    __builtin_nontemporal_store(v[j], reinterpret_cast<Raw*>(at + (d0 + lane) * 8));
                } else {
                    constexpr int PW = 4 / (int)sizeof(Elem);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (places >> e & 1) at[(d0 + lane) * 8 + e] = (Elem)(v[j][e / PW] >> (e % PW * (int)sizeof(Elem) * 8));
                }
            }
        }
    }
}

int launch_compact(const CompactParams& p, int head_dim, bool fp8_pages, int layers, void* stream) {
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const int heads = kMoves / p.step, groups = (p.Hkv + heads - 1) / heads, slices = head_dim / kCompactWidth;
    const dim3 grid((unsigned)(p.B * groups), (unsigned)(2 * slices + (p.weights ? 1 : 0)), (unsigned)layers);
    if (head_dim == 128 && fp8_pages) hipLaunchKernelGGL((ppd_compact_kernel<128, true>), grid, dim3(kCompactThreads), 0, hs, p);
    else if (head_dim == 128) hipLaunchKernelGGL((ppd_compact_kernel<128, false>), grid, dim3(kCompactThreads), 0, hs, p);
    else if (fp8_pages) hipLaunchKernelGGL((ppd_compact_kernel<64, true>), grid, dim3(kCompactThreads), 0, hs, p);
    else hipLaunchKernelGGL((ppd_compact_kernel<64, false>), grid, dim3(kCompactThreads), 0, hs, p);
    return (int)hipGetLastError();
}

}  // namespace ppd
