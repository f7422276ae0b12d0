// gfx950 kernels of tree and weighted attention over the page pool.
//
//   out[j, h] = sum_t p_t v_t,   p = softmax over the visible t of scale * q[j, h] . k_t
//   weights[b, kvh, t] (+)= sum over the sequence's rows j and the group's heads h of p_t
//
// As in the mixed kernels the products are the transposed ones, S^T = K Q^T and O^T = V^T P^T: the accumulators of the first
// are the operands of the second, and every quantity of a row's softmax lives in the lanes that own its column.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ppd_device.h"
#include "ppd_ops.h"

namespace ppd {

namespace {

template <bool FP8> struct Granule;  // eight elements of the pool as they are loaded
template <> struct Granule<false> { typedef u32x4 type; };
template <> struct Granule<true> { typedef u32x2 type; };

__device__ __forceinline__ u32x4 operand(u32x4 g) { return g; }
__device__ __forceinline__ u32x4 operand(u32x2 g) { return fp8x8_to_bf16x8(g); }

// Page ids of the tile's keys, checked, to LDS: an id outside the pool raises the sticky flag and is replaced by page 0.
__device__ __forceinline__ void stage_pages(const TreeParams& P, int seq, int kv_begin, int kv_total, int count, int* ids) {
    const int32_t* row = P.page_tables + (int64_t)seq * P.max_pages;
    const int last = (kv_total - 1) / kPage, first = kv_begin / kPage;
    for (int i = threadIdx.x; i < count; i += blockDim.x) {
        int id = row[first + i < last ? first + i : last];
        if (id < 0 || id >= P.num_pages) {
            atomicOr(P.err_flags, 2u);
            id = 0;
        }
        ids[i] = id;
    }
}

}  // namespace

// A tree tile: up to 32 query columns against a range of keys.  Four waves, each with every fourth slab of 32 keys, which it
// takes from the pool straight into registers in the layouts of the matrix instructions' operands: no LDS, no barrier.  The
// waves' results meet in LDS at the end.  Probabilities enter the second product as bf16 numbers, as the matrix instruction takes them
// (their sum is of the 32-bit ones); everything else is held in 32 bits.
// Bound by memory where there is much to read: 64 decodes of 1K-8K keys (32 query heads, D = 128) 142 us, 6.6 TB/s (with the scores'
// stores 162, on FP8 pages 87, 5.4 TB/s), trees of 4-8 nodes on the same 171 us, 5.8 TB/s (FP8 pages 91); by a chain of
// dependent loads (tile, page ids, K) of 5 us in small launches.  More than 32 columns as several tiles side by side, their keys read
// from L2 once more for every 32, were no faster than row blocks from 64 columns on (32 trees of 8-24 nodes, 8 query heads to a KV
// head: 137-152 us against 137), and two launches where a batch has both kinds.
template <int HD, bool FP8, bool SCORES>
__device__ __forceinline__ void tree_tile(const TreeParams& P) {
    typedef typename Granule<FP8>::type Raw;
    constexpr int EB = FP8 ? 1 : 2, KS = HD / 16, DB = HD / 32;
    constexpr int CB = 16;          // columns that meet in LDS at a time
    constexpr int ROW = HD + 4;     // floats of a staged column: the padding spreads the columns over the banks
    __shared__ int ids[kMaxTreeChunk / kPage];
    // one after the other: the tile's scores (SCORES), the waves' results
    constexpr int AREA = kTreeWaves * CB * ROW;
    __shared__ __attribute__((aligned(16))) float area[SCORES && kKeptScores > AREA ? kKeptScores : AREA];
    float (&stage)[kTreeWaves][CB * ROW] = *reinterpret_cast<float (*)[kTreeWaves][CB * ROW]>(area);
    __shared__ float stage_ml[kTreeWaves][CB][2];

    const TreeItem it = P.items[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, l32 = lane & 31;
    const int col = l32 < it.ncols ? l32 : it.ncols - 1;
    const int jrow = col / P.G, head = it.kvh * P.G + (col - jrow * P.G);
    const float c = P.scale_log2e;
    const uint64_t* const words = P.mask ? P.mask + (int64_t)(it.grow0 + jrow) * P.mask_words : nullptr;

    const int slabs = (it.kv_end - it.kv_begin + kSlab - 1) / kSlab;
    stage_pages(P, it.seq, it.kv_begin, it.kv_total, slabs * 2, ids);
    bf16x8 qreg[KS];
    {
        const uint16_t* qp = P.q + ((int64_t)(it.grow0 + jrow) * P.Hq + head) * HD + h * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qreg[ks] = as_bf16x8(*reinterpret_cast<const u32x4*>(qp + ks * 16));
    }
    __syncthreads();

    // Row r of the K operand is token 8*bit2(r) + 4*bit3(r) + (r & 3) of page bit4(r): registers 8p .. 8p+7 of a lane are then eight
    // consecutive tokens of page p, which is what the second product takes.
    const int k_tok = ((l32 >> 2) & 1) * 8 + ((l32 >> 3) & 1) * 4 + (l32 & 3);
    const char* const pool = static_cast<const char*>(P.pool) + (int64_t)it.kvh * (kPage * HD) * EB;
    const char* const k_lane = pool + (h * 16 + k_tok) * (8 * EB);
    const char* const v_lane = pool + ((int64_t)P.Hkv * (kPage * HD) + (h * HD + l32) * 8) * EB;
    const int64_t page_bytes = P.page_stride * EB;

    // Read once: non-temporal loads (64 decodes of 1K-8K keys with weights 214 -> 190 us).
    Raw kr[KS], vr[2][DB];
    auto load_k = [&](int s) {
        const char* p = k_lane + (int64_t)ids[s * 2 + (l32 >> 4)] * page_bytes;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kr[ks] = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(p + ks * (2 * 16 * 8 * EB)));
    };
    auto load_v = [&](int s) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const char* vp = v_lane + (int64_t)__builtin_amdgcn_readfirstlane(ids[s * 2 + p]) * page_bytes;
#pragma unroll
            for (int db = 0; db < DB; ++db) vr[p][db] = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(vp + db * (32 * 8 * EB)));
        }
    };

    f32x16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[db][i] = 0.f;
    float m_run = NEG_INF, l_run = 0.f;

    // One slab.  The next one's K is asked for when this one's has been used, and its V likewise, so that a slab is on its way while
    // another is worked.  A wave's last slab asks for none; it alone can hold new tokens (at most kSlab of them, in neighbouring slabs,
    // at the end of the range), so only its code looks at masks.  (A load that is asked for in one branch and not in another would
    // have to be waited for together with all that came behind it.)
    auto step = [&](int s, auto last) {
        constexpr bool LAST = decltype(last)::value;
        const int base = it.kv_begin + s * kSlab;
        f32x16 sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(operand(kr[ks])), qreg[ks], sc, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!LAST) load_k(s + kTreeWaves);
        __builtin_amdgcn_sched_barrier(0);
        uint32_t seen = ~0u;
        bool strange = false;  // a new token's V that is not finite: not every row may see it
        u32x4 vv[2][DB];
        if constexpr (LAST) {
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int db = 0; db < DB; ++db) vv[p][db] = operand(vr[p][db]);
            if (base + kSlab > it.L) {
                seen = (uint32_t)visible_keys(words, P.mask_words, jrow, base - it.L, it.kv_total - base);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((seen >> ((i >> 3) * 16 + h * 8 + (i & 7))) & 1u)) sc[i] = NEG_INF;
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int pos = base + p * 16 + h * 8 + e;
                            const bool odd = pos >= it.L && not_finite_bf16(vv[p][db][e >> 1] >> ((e & 1) * 16));
                            strange |= odd && pos < it.kv_total;
                            if (odd || pos >= it.kv_total) vv[p][db][e >> 1] &= (e & 1) ? 0x0000FFFFu : 0xFFFF0000u;
                        }
            }
        }
        if constexpr (SCORES) {
            if (it.score_off >= 0 && l32 < it.ncols) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4*>(&area[(s * it.ncols + l32) * kSlab + h * 8 + (i >> 1) * 16 + (i & 1) * 4]) = f32x4{sc[4 * i], sc[4 * i + 1], sc[4 * i + 2], sc[4 * i + 3]};
            }
        }
        // The exponentials are taken against the running reference as it is; only where a lane's sum of 16 of them is above
        // 2^kLazyRescale (or not a number: no reference yet) is the maximum looked for and everything rescaled.
        u32x4 pw[2];
        float psum = 0.f;
        auto exponentials = [&](float mc) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float p0 = fast_exp2(__builtin_fmaf(sc[2 * e], c, -mc));
                const float p1 = fast_exp2(__builtin_fmaf(sc[2 * e + 1], c, -mc));
                psum += p0 + p1;
                pw[e >> 2][e & 3] = pack_bf16(p0, p1);
            }
        };
        exponentials(m_run * c);
        if (__any(!(psum <= kMaxLazyP))) {
            float mx = sc[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
            // a column whose own sums are in range keeps its reference, so that no other row decides how it is rounded
            mx = max_halves(mx);
            mx = max_halves(!(psum <= kMaxLazyP) ? 1.f : 0.f) > 0.f ? mx : m_run;
            const float m_new = fmaxf(m_run, mx);
            const float m_use = m_new == NEG_INF ? 0.f : m_new;
            const float alpha = fast_exp2((m_run - m_use) * c);  // m_run = -inf gives 0, the same reference exactly 1
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) oacc[db][i] *= alpha;
            m_run = m_new;
            psum = 0.f;
            exponentials(m_use * c);
        }
        l_run += psum;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const u32x4 v = LAST ? vv[p][db] : operand(vr[p][db]);
                oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v), as_bf16x8(pw[p]), oacc[db], 0, 0, 0);
            }
        if constexpr (LAST) {
            if (__any(strange)) {
                // Elements that are not finite were left out of the product, where rows that do not see them would have taken NaN from
                // them; rows that do get them here, whatever their probability.
                for (int t = 0; t < kSlab; ++t) {
                    const int pos = base + t;
                    if (pos < it.L || pos >= it.kv_total || !__any((seen >> t) & 1u)) continue;
                    const char* vt = pool + ((int64_t)ids[s * 2 + (t >> 4)] * P.page_stride + (int64_t)P.Hkv * (kPage * HD) + ((t >> 3) & 1) * (HD * 8) + (t & 7)) * EB;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int d = db * 32 + (i >> 2) * 8 + h * 4 + (i & 3);
                            uint32_t bits;
                            if constexpr (FP8) bits = fp8x4_to_bf16x4(*reinterpret_cast<const uint8_t*>(vt + d * 8))[0] & 0xFFFFu;
                            else bits = *reinterpret_cast<const uint16_t*>(vt + d * 16);
                            if (((seen >> t) & 1u) && not_finite_bf16(bits)) oacc[db][i] += __builtin_bit_cast(float, bits << 16);
                        }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!LAST) load_v(s + kTreeWaves);
        __builtin_amdgcn_sched_barrier(0);
    };
    if (wave < slabs) {
        load_k(wave);
        load_v(wave);
        int s = wave;
        for (; s + kTreeWaves < slabs; s += kTreeWaves) step(s, std::false_type{});
        step(s, std::true_type{});
    }

    // The scores leave at the end, all at once: 64 decodes of 1K-8K keys took 173 us with stores of every slab on its own among the
    // loads, whether or not behind a branch, and as whole lines too; 142 without stores; 159 this way, 165 without device scope.
    if constexpr (SCORES) {
        __syncthreads();
        if (it.score_off >= 0) {
            const int floats = slabs * it.ncols * kSlab;
            const auto to = __builtin_amdgcn_make_buffer_rsrc(P.scores + it.score_off + (int64_t)(it.kv_begin / kSlab) * (it.ncols * kSlab), 0, floats * 4, 0x00020000);
            constexpr int DEVICE_SCOPE = 16;  // sc1
            for (int i = tid * 4; i < floats; i += kTreeThreads * 4) __builtin_amdgcn_raw_buffer_store_b128(*reinterpret_cast<const u32x4*>(&area[i]), to, i * 4, 0, DEVICE_SCOPE);
        }
    }
    const float l_tot = sum_halves(l_run);
    for (int c0 = 0; c0 < it.ncols; c0 += CB) {
        __syncthreads();
        if (l32 >= c0 && l32 < c0 + CB) {
            float* to = &stage[wave][(l32 - c0) * ROW + h * 4];
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4*>(to + db * 32 + i * 8) = f32x4{oacc[db][4 * i], oacc[db][4 * i + 1], oacc[db][4 * i + 2], oacc[db][4 * i + 3]};
            if (h == 0) {
                stage_ml[wave][l32 - c0][0] = m_run;
                stage_ml[wave][l32 - c0][1] = l_tot;
            }
        }
        __syncthreads();
        const int nc = it.ncols - c0 < CB ? it.ncols - c0 : CB;
        for (int idx = tid; idx < nc * (HD / 4); idx += kTreeThreads) {
            const int cl = idx / (HD / 4), d = (idx % (HD / 4)) * 4;
            float mm = NEG_INF;
#pragma unroll
            for (int w = 0; w < kTreeWaves; ++w) mm = fmaxf(mm, stage_ml[w][cl][0]);
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
            float l = 0.f;
#pragma unroll
            for (int w = 0; w < kTreeWaves; ++w) {
                const float mw = stage_ml[w][cl][0];
                const float f = mw == NEG_INF ? 0.f : fast_exp2((mw - mm) * c);
                l += f * stage_ml[w][cl][1];
                if (mw != NEG_INF) o += f * *reinterpret_cast<const f32x4*>(&stage[w][cl * ROW + d]);
            }
            const int cc = c0 + cl;
            if (it.part_off >= 0) {
                float* to = P.partials + it.part_off;
                *reinterpret_cast<partial4*>(to + cc * HD + d) = o;
                if (d == 0) *reinterpret_cast<f32x2*>(to + it.ncols * HD + cc * 2) = f32x2{mm, l};
            } else {
                const int row = cc / P.G;
                const int64_t at = (int64_t)(it.grow0 + row) * P.Hq + it.kvh * P.G + (cc - row * P.G);
                const float inv = l == 0.f ? 0.f : 1.0f / l;  // a row that sees nothing gives zeros
                const f32x4 r = o * (inv * P.v_scale);
                *reinterpret_cast<u32x2*>(P.out + at * HD + d) = u32x2{pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
                if (P.stats && d == 0) *reinterpret_cast<f32x2*>(P.stats + at * 2) = f32x2{mm == NEG_INF ? 0.f : mm, inv};
            }
        }
    }
}

template <int HD, bool FP8>
__global__ __launch_bounds__(kTreeThreads, 2) void ppd_tree_kernel(const TreeParams P) { tree_tile<HD, FP8, false>(P); }
template <int HD, bool FP8>
__global__ __launch_bounds__(kTreeThreads, 2) void ppd_tree_scores_kernel(const TreeParams P) { tree_tile<HD, FP8, true>(P); }

// Joins the partials of split key ranges, splits in order.  Bound by latency: the (m, l) pairs of a workgroup's columns go to LDS all at
// once, and a lane asks for eight splits' values before it adds the first.  One lane after the other over 32 splits took 24 us.
constexpr int kJoinPairs = 2048;
template <int HD>
__device__ __forceinline__ void join_columns(const TreeParams& P, int group, int part, f32x2* ml) {
    constexpr int LANES = HD / 4, COLS = 256 / LANES, AT_ONCE = 8;
    const TreeGroup g = P.groups[group];
    const int c0 = part * COLS, cl = threadIdx.x / LANES, col = c0 + cl, d = (threadIdx.x % LANES) * 4;
    if (c0 >= g.ncols) return;
    const float c = P.scale_log2e;
    const float* base = P.partials + g.part_off;
    const float* pairs = base + (int64_t)g.ncols * HD;
    const bool staged = g.nsplit * COLS <= kJoinPairs;
    // the first splits' values are asked for before the pairs have arrived (one decode of 4000 keys 14.0 -> 13.1 us a call)
    f32x4 v[AT_ONCE];
    const float* values = base + (int64_t)(col < g.ncols ? col : g.ncols - 1) * HD + d;
    auto ask = [&](int j0) {
#pragma unroll
        for (int t = 0; t < AT_ONCE; ++t) v[t] = *reinterpret_cast<const partial4*>(values + g.part_stride * (j0 + t < g.nsplit ? j0 + t : j0));
    };
    auto staged_pair = [&](int i) {
        const int cc = c0 + i % COLS;
        return *reinterpret_cast<const f32x2*>(pairs + g.part_stride * (i / COLS) + (cc < g.ncols ? cc : c0) * 2);
    };
    const int n_pairs = staged ? g.nsplit * COLS : 0;
    f32x2 mine = {};
    if ((int)threadIdx.x < n_pairs) mine = staged_pair(threadIdx.x);
    ask(0);
    if ((int)threadIdx.x < n_pairs) ml[threadIdx.x] = mine;
    for (int i = threadIdx.x + 256; i < n_pairs; i += 256) ml[i] = staged_pair(i);
    __syncthreads();
    if (col >= g.ncols) return;
    auto pair = [&](int j) { return staged ? ml[j * COLS + cl] : *reinterpret_cast<const f32x2*>(pairs + g.part_stride * j + col * 2); };
    float mm = NEG_INF;
    for (int j = 0; j < g.nsplit; ++j) mm = fmaxf(mm, pair(j)[0]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    for (int j0 = 0; j0 < g.nsplit; j0 += AT_ONCE) {
        if (j0 > 0) ask(j0);
#pragma unroll
        for (int t = 0; t < AT_ONCE; ++t) {
            if (j0 + t >= g.nsplit) continue;
            const f32x2 w = pair(j0 + t);
            if (w[0] == NEG_INF) {  // no key that the row sees, or none but scores of minus infinity; the sum is 0, or NaN where a score was NaN
                l += w[1];
                continue;
            }
            const float f = fast_exp2((w[0] - mm) * c);
            l += f * w[1];
            o += f * v[t];
        }
    }
    const int oc = g.col0 + col, row = oc / P.G;
    const int64_t at = (int64_t)(g.grow0 + row) * P.Hq + g.kvh * P.G + (oc - row * P.G);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const f32x4 r = o * (inv * P.v_scale);
    *reinterpret_cast<u32x2*>(P.out + at * HD + d) = u32x2{pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
    if (P.stats && d == 0) *reinterpret_cast<f32x2*>(P.stats + at * 2) = f32x2{mm == NEG_INF ? 0.f : mm, inv};
}

// Adds up the weights of sequences with many query columns: S = Q K^T with the keys as columns, so that a lane owns a key and the sum
// over the queries runs over its own registers.  A wave holds K of 64 keys, read once, and goes over the sequence's query columns, 32 at
// a time, which the workgroup brings to LDS, the next ones on their way meanwhile (each wave for itself, in pieces of 16 bytes of 32
// rows, they kept the load unit busy: the last 16-33 rows of 4 prompts of 4K-32K, 40
// query heads, 55 us, this way 50: 2.9 TB/s of K; a workgroup's start -- tile, page ids, K -- and 5 steps of 32 columns, two workgroups
// to a unit, three no faster).  The reference and one over the sum of every row come from the attention before.
constexpr int kWeighCols = 256;  // columns whose references are in LDS at a time
template <int HD, bool FP8>
__global__ __launch_bounds__(256, 2) void ppd_weigh_kernel(const TreeParams P) {
    typedef typename Granule<FP8>::type Raw;
    constexpr int EB = FP8 ? 1 : 2, KS = HD / 16, SLABS = kWeighKeys / 4 / kSlab;
    constexpr int QG = HD / 64, QROW = HD * 2 + 16;  // granules of 32 columns that a thread fetches; bytes of a column in LDS
    __shared__ int ids[kWeighKeys / kPage];
    __shared__ __attribute__((aligned(16))) char queries[2][32 * QROW];
    __shared__ f32x2 ml[kWeighCols];
    __shared__ int rows[kWeighCols];
    const WeighItem it = P.weighs[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, l32 = lane & 31;
    auto q_at = [&](int cc) {  // element offset of a column's query
        cc = cc < it.cols ? cc : it.cols - 1;
        const int row = cc / P.G;
        return ((int64_t)(it.grow0 + row) * P.Hq + it.kvh * P.G + (cc - row * P.G));
    };
    u32x4 qnext[QG];
    auto load_q = [&](int c0) {
#pragma unroll
        for (int j = 0; j < QG; ++j) {
            const int i = tid + j * 256;
            qnext[j] = *reinterpret_cast<const u32x4*>(P.q + q_at(c0 + i / (HD / 8)) * HD + i % (HD / 8) * 8);
        }
    };
    stage_pages(P, it.seq, it.kv_begin, it.kv_total, kWeighKeys / kPage, ids);
    load_q(0);
    __syncthreads();
    const char* const pool = static_cast<const char*>(P.pool) + ((int64_t)it.kvh * (kPage * HD) + (h * 16 + (l32 & 15)) * 8) * EB;
    u32x4 kreg[SLABS][KS];
#pragma unroll
    for (int s = 0; s < SLABS; ++s) {
        const char* p = pool + (int64_t)ids[(wave * SLABS + s) * 2 + (l32 >> 4)] * P.page_stride * EB;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kreg[s][ks] = operand(*reinterpret_cast<const Raw*>(p + ks * (2 * 16 * 8 * EB)));
    }
    const float c = P.scale_log2e;
    float sum[SLABS];
#pragma unroll
    for (int s = 0; s < SLABS; ++s) sum[s] = 0.f;
    const int base = it.kv_begin + wave * (SLABS * kSlab);
    const bool tail = base + SLABS * kSlab > it.L;  // new tokens among the wave's keys: not every row sees them
    for (int b0 = 0; b0 < it.cols; b0 += kWeighCols) {
        const int b1 = b0 + kWeighCols < it.cols ? b0 + kWeighCols : it.cols;
        if (b0 > 0) __syncthreads();
        {
            const int cc = b0 + tid;  // columns past the end count nothing: their exponentials are 0, and so is the factor
            ml[tid] = cc < it.cols ? *reinterpret_cast<const f32x2*>(P.stats + q_at(cc) * 2) : f32x2{1e30f, 0.f};
            ml[tid][0] *= c;
            rows[tid] = cc < it.cols ? cc / P.G : -1;
        }
        __syncthreads();
        for (int c0 = b0; c0 < b1; c0 += 32) {
            char* const qcols = queries[c0 / 32 & 1];
#pragma unroll
            for (int j = 0; j < QG; ++j) {
                const int i = tid + j * 256;
                *reinterpret_cast<u32x4*>(qcols + i / (HD / 8) * QROW + i % (HD / 8) * 16) = qnext[j];
            }
            __syncthreads();
            if (c0 + 32 < it.cols) load_q(c0 + 32);
            bf16x8 qreg[KS];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qreg[ks] = as_bf16x8(*reinterpret_cast<const u32x4*>(qcols + l32 * QROW + ks * 32 + h * 16));
            f32x16 sc[SLABS];
#pragma unroll
            for (int s = 0; s < SLABS; ++s)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[s][i] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int s = 0; s < SLABS; ++s) sc[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qreg[ks], as_bf16x8(kreg[s][ks]), sc[s], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = c0 - b0 + (i & 3) + 8 * (i >> 2) + 4 * h;
                const f32x2 w = ml[r];
#pragma unroll
                for (int s = 0; s < SLABS; ++s) {
                    const float p = fast_exp2(__builtin_fmaf(sc[s][i], c, -w[0])) * w[1];
                    if (!tail || (rows[r] >= 0 && base + s * kSlab + l32 <= it.L + rows[r])) sum[s] += p;
                }
            }
        }
    }
#pragma unroll
    for (int s = 0; s < SLABS; ++s) {
        const float total = sum_halves(sum[s]);
        const int key = base + s * kSlab + l32;
        if (h == 0 && key < it.kv_total) {
            float* to = P.weights + ((int64_t)it.seq * P.Hkv + it.kvh) * P.weight_stride + key;
            *to = key < it.L ? *to + total : total;
        }
    }
}

// Adds up the weights of sequences with few query columns, whose scores ppd_tree_kernel has left in the workspace: a thread to a key.
// The scores of G columns are 8 G bytes a key, written and read, where K again would be 2 D: 64 decodes of 1K-8K keys (32 query
// heads, D = 128) 106 us that way, 14 this way.  Where the range was split, the references come from the partials' own pairs, so
// that nothing waits for the join.
template <int HD>
__device__ __forceinline__ void weigh_scores(const TreeParams& P, const WeighItem& it, f32x2* ml) {
    const int tid = threadIdx.x, cols = it.cols;
    const float c = P.scale_log2e;
    constexpr int PARTS = kWeighKeys / kTreeCols;  // threads that go over a column's splits
    constexpr int AHEAD = 8;  // scores asked for before the references are known
    const int key = it.kv_begin + tid, safe = key < it.kv_total ? key : it.kv_total - 1;
    const float* scores = P.scores + it.score_off + (int64_t)(safe / kSlab) * (cols * kSlab) + safe % kSlab;
    float* to = P.weights + ((int64_t)it.seq * P.Hkv + it.kvh) * P.weight_stride + safe;
    float ahead[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ahead[i] = scores[(i < cols ? i : 0) * kSlab];
    const float old = *to;
    if (it.group >= 0) {
        const TreeGroup g = P.groups[it.group];
        const int cc = tid % kTreeCols, part = tid / kTreeCols;
        const float* pairs = P.partials + g.part_off + (int64_t)cols * HD + cc * 2;
        float m = NEG_INF, l = 0.f;
        if (cc < cols) {
            for (int j = part; j < g.nsplit; j += PARTS) {
                const f32x2 w = *reinterpret_cast<const f32x2*>(pairs + g.part_stride * j);
                const float top = fmaxf(m, w[0]);
                if (w[0] == NEG_INF) {  // as in join_columns
                    l += w[1];
                    continue;
                }
                l = l * fast_exp2((m - top) * c) + w[1] * fast_exp2((w[0] - top) * c);
                m = top;
            }
        }
        ml[tid] = f32x2{m, l};
        __syncthreads();
        m = NEG_INF;
        l = 0.f;
        if (tid < kTreeCols) {
#pragma unroll
            for (int k = 0; k < PARTS; ++k) m = fmaxf(m, ml[k * kTreeCols + tid][0]);
#pragma unroll
            for (int k = 0; k < PARTS; ++k) {
                const f32x2 w = ml[k * kTreeCols + tid];
                l += w[0] != NEG_INF ? w[1] * fast_exp2((w[0] - m) * c) : w[1];
            }
        }
        __syncthreads();
        if (tid < kTreeCols) ml[tid] = f32x2{m == NEG_INF ? 0.f : m * c, l == 0.f ? 0.f : 1.0f / l};
    } else if (tid < cols) {
        const int row = tid / P.G;
        const f32x2 w = *reinterpret_cast<const f32x2*>(P.stats + ((int64_t)(it.grow0 + row) * P.Hq + it.kvh * P.G + (tid - row * P.G)) * 2);
        ml[tid] = f32x2{w[0] * c, w[1]};
    }
    __syncthreads();
    if (key >= it.kv_total) return;
    float sum = 0.f;
    auto add = [&](float score, int cc) { sum += fast_exp2(__builtin_fmaf(score, c, -ml[cc][0])) * ml[cc][1]; };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (i < cols) add(ahead[i], i);
    for (int cc = AHEAD; cc < cols; ++cc) add(scores[cc * kSlab], cc);
    *to = key < it.L ? old + sum : sum;
}

// Behind the tiles: joins their partials and adds up the weights of kept scores, in one launch (one decode of 4000 keys 17.1 us with
// a launch each, 13.8 with one, before values were asked for ahead; 64 of 1K-8K 178 and 175).
static_assert(kWeighKeys == 256, "both parts work with 256 threads");
template <int HD>
__global__ __launch_bounds__(256) void ppd_tree_join_kernel(const TreeParams P, int parts) {
    __shared__ f32x2 ml[kJoinPairs];
    const int joins = P.n_groups * parts;
    if ((int)blockIdx.x < joins) join_columns<HD>(P, blockIdx.x / parts, blockIdx.x % parts, ml);
    else weigh_scores<HD>(P, P.score_weighs[blockIdx.x - joins], ml);
}

#define PPD_BY_FORM(KERNEL, GRID, THREADS)                                                                                        \
    do {                                                                                                                          \
        if (head_dim == 128 && fp8_pages) hipLaunchKernelGGL((KERNEL<128, true>), GRID, dim3(THREADS), 0, hs, p);                 \
        else if (head_dim == 128) hipLaunchKernelGGL((KERNEL<128, false>), GRID, dim3(THREADS), 0, hs, p);                        \
        else if (fp8_pages) hipLaunchKernelGGL((KERNEL<64, true>), GRID, dim3(THREADS), 0, hs, p);                                \
        else hipLaunchKernelGGL((KERNEL<64, false>), GRID, dim3(THREADS), 0, hs, p);                                              \
    } while (0)

int launch_tree(const TreeParams& p, int head_dim, bool fp8_pages, void* stream) {
    hipStream_t hs = static_cast<hipStream_t>(stream);
    if (p.n_score_weighs > 0) PPD_BY_FORM(ppd_tree_scores_kernel, dim3((unsigned)p.n_items), kTreeThreads);
    else PPD_BY_FORM(ppd_tree_kernel, dim3((unsigned)p.n_items), kTreeThreads);
    return (int)hipGetLastError();
}

int launch_tree_join(const TreeParams& p, int head_dim, void* stream) {
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const int cols = 256 / (head_dim / 4), parts = (p.join_cols + cols - 1) / cols;  // columns of a workgroup, workgroups of a group
    const dim3 grid((unsigned)(p.n_groups * parts + p.n_score_weighs));
    if (head_dim == 128) hipLaunchKernelGGL(ppd_tree_join_kernel<128>, grid, dim3(256), 0, hs, p, parts);
    else hipLaunchKernelGGL(ppd_tree_join_kernel<64>, grid, dim3(256), 0, hs, p, parts);
    return (int)hipGetLastError();
}

int launch_weigh(const TreeParams& p, int head_dim, bool fp8_pages, void* stream) {
    hipStream_t hs = static_cast<hipStream_t>(stream);
    PPD_BY_FORM(ppd_weigh_kernel, dim3((unsigned)p.n_weighs), 256);
    return (int)hipGetLastError();
}

}  // namespace ppd
