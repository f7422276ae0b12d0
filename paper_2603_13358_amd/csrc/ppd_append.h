// What the kernels that append tokens to the page pool share: which slots a workgroup's tokens go to, and the stores of V.
#pragma once
#include "ppd_device.h"
#include "ppd_internal.h"

namespace ppd {

// source and pool are each touched once: non-temporal loads and stores (the landing of a whole request runs 7 %
// faster with them)
#define APPEND_LOAD(p) __builtin_nontemporal_load(p)
#define APPEND_STORE(v, p) __builtin_nontemporal_store(v, p)

// The slots around a workgroup's tokens.  A V granule is 8 tokens of one d, i.e. 8 consecutive slots starting at a multiple of 8;
// an octet is a run of 8 batch tokens that fills one.
struct AppendWindow {
    int64_t slot;          // lane 7 + i: of the workgroup's token i; negative: skipped
    uint32_t single;       // a bit for each of its tokens that belongs to no octet and is not skipped
    uint32_t own_octets;   // a bit for each of its tokens that an octet starts at
    int extra;             // rows behind its own ones that the last octet reaches into
};

// TOK tokens from t0 on; all lanes of every wave call it.  `reports`: this workgroup raises the flag for slots beyond the pool.
template <int TOK>
__device__ __forceinline__ AppendWindow append_window(const int64_t* __restrict__ slots, int64_t t0, int64_t T, int64_t num_pages, bool reports,
                                                      uint32_t* err_flags) {
    const int tid = threadIdx.x, lane = tid & 63;
    // Window of slots: batch tokens t0-7 .. t0+TOK+6, one per lane (lane 7 holds token t0), in every wave; tokens
    // outside the batch and slots outside the pool count as skipped.  What follows is a handful of wave-wide
    // votes: the per-workgroup bookkeeping has to stay far below the cost of moving the tokens.
    constexpr int kWin = TOK + 14;
    constexpr uint32_t kOwn = (1u << TOK) - 1;
    const int64_t tw = t0 - 7 + lane;
    int64_t ws = -1;
    if (lane < kWin && tw >= 0 && tw < T) ws = slots[tw];
    const bool outside = ws >= num_pages * kPage;
    if (__ballot(outside && lane >= 7 && lane < 7 + TOK) != 0 && tid == 0 && reports) atomicOr(err_flags, 1u);
    if (outside) ws = -1;
    // bit i of `runs`: entry i+1 holds the slot after entry i's; bit c of `octets`: the 8 tokens from entry c on
    // sit in the 8 slots of one V granule, in order
    const int64_t ws_next = __shfl_down(ws, 1);
    const uint64_t runs = __ballot(lane < kWin - 1 && ws_next == ws + 1);
    const uint64_t starts = __ballot(ws >= 0 && (ws & 7) == 0);
    const uint32_t octets = (uint32_t)(starts & runs & (runs >> 1) & (runs >> 2) & (runs >> 3) & (runs >> 4) &
                                       (runs >> 5) & (runs >> 6)) & ((1u << (TOK + 7)) - 1);
    // own tokens: which of them no octet covers (a token with slot s would be entry s % 8 of one), and the
    // octets that start at one of them
    const int my_start = (ws >= 0 && lane >= 7) ? lane - (int)(ws & 7) : 0;
    AppendWindow w;
    w.slot = ws;
    w.single = (uint32_t)(__ballot(lane >= 7 && lane < 7 + TOK && ws >= 0 && !((octets >> my_start) & 1u)) >> 7) & kOwn;
    w.own_octets = (octets >> 7) & kOwn;  // at most TOK / 8
    // rows beyond the own ones that the last octet reaches into
    const int last_oct = w.own_octets ? 31 - __builtin_clz(w.own_octets) : 0;
    w.extra = w.own_octets && last_oct + 8 > TOK ? last_oct + 8 - TOK : 0;
    return w;
}

// Writes the V rows that are staged in LDS, `row` elements apart (the workgroup's own and `extra` more): its octets as whole granules,
// tokens of no octet element by element.  `to`: the head's V block of page 0, pages `page_stride` elements apart.
template <int D, int TOK, bool FP8, class Elem>
__device__ __forceinline__ void store_v(const AppendWindow& w, const uint16_t* sv, int row, Elem* to, int64_t page_stride, float inv_v) {
    const int tid = threadIdx.x;
    // whole granules: work unit = (octet, d)
    uint32_t left = w.own_octets;
#pragma unroll
    for (int o = 0; o < TOK / 8; ++o) {
        if (!left) break;
        const int tok = __builtin_ctz(left);
        left &= left - 1;
        const int64_t s = __shfl(w.slot, 7 + tok);
        // the octets take turns at starting with the first thread, so that at D < 256 each has threads of its own
        const int d = (tid + o * D) % kSmallThreads;
        if (d < D) {
            uint32_t g[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                g[e] = (uint32_t)sv[(tok + 2 * e) * row + d] | ((uint32_t)sv[(tok + 2 * e + 1) * row + d] << 16);
            auto* dst = to + (s >> 4) * page_stride + (int)((s & 15) >> 3) * (D * 8) + d * 8;
            if constexpr (FP8) {
                const u32x2 codes = {e4m3_codes(g[0], g[1], inv_v), e4m3_codes(g[2], g[3], inv_v)};
                APPEND_STORE(codes, reinterpret_cast<u32x2*>(dst));
            } else {
                APPEND_STORE((u32x4{g[0], g[1], g[2], g[3]}), reinterpret_cast<u32x4*>(dst));
            }
        }
    }
    // element by element: work unit = (token, d)
    if (w.single) {
        for (int u = tid; u < D * TOK; u += kSmallThreads) {
            const int tok = u / D, d = u % D;
            const int64_t s = __shfl(w.slot, 7 + tok);  // before any lane drops out
            if (!((w.single >> tok) & 1u)) continue;
            const int off = (int)(s & 15);
            const uint16_t x = sv[tok * row + d];
            auto* dst = to + (s >> 4) * page_stride + (off >> 3) * (D * 8) + d * 8 + (off & 7);
            if constexpr (FP8) *dst = (uint8_t)e4m3_codes(x, 0u, inv_v); else *dst = x;
        }
    }
}

}  // namespace ppd
