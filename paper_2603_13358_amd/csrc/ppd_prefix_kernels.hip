// gfx950 kernels of attention over shared prefixes.
//
//   out[j, h] = sum_t p_t v_t,   p = softmax over t <= L + j of scale * q[j, h] . k_t
//
// The keys of a row are a chain of ranges: some that it shares with the rows of neighbouring sequences, and its sequence's own.  A tile
// takes the columns (rows x heads of a group) of all rows that have a range, so that the range is read once for all of them; the
// tiles' partial sums, each with the maximum and the sum of its exponentials, are joined row by row.
// As in the other attention kernels the products are the transposed ones, S^T = K Q^T and O^T = V^T P^T: the accumulators of the first
// are the operands of the second, and every quantity of a row's softmax lives in the lanes that own its column.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ppd_device.h"
#include "ppd_prefix.h"

namespace ppd {

namespace {

template <bool FP8> struct Granule;  // eight elements of the pool as they are loaded
template <> struct Granule<false> { typedef u32x4 type; };
template <> struct Granule<true> { typedef u32x2 type; };

__device__ __forceinline__ u32x4 operand(u32x4 g) { return g; }
__device__ __forceinline__ u32x4 operand(u32x2 g) { return fp8x8_to_bf16x8(g); }

// Where element d (a multiple of 4) of a column's sum is in a tile's partial: four columns at a time, four elements of each side by side.
template <int HD>
__device__ __forceinline__ int partial_at(int ncols, int col, int d) {
    const int first = col & ~3, width = ncols - first < 4 ? ncols - first : 4;
    return first * HD + (d / 4 * width + (col & 3)) * 4;
}

constexpr int kPrefixWaves = 4, kPrefixThreads = 64 * kPrefixWaves;
constexpr int kStageCols = 16;  // columns of a wave that meet in LDS at a time

}  // namespace

// What a wave holds of its 32 columns: O^T, and of a lane's column the running reference and its part of the sum.
template <int HD>
struct Columns {
    static constexpr int DB = HD / 32;
    f32x16 o[DB];
    float m, l;

    __device__ __forceinline__ void clear() {
        m = NEG_INF;
        l = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
    }

    // Turns the scores of a slab into probabilities, as operands of the second product.  The exponentials are taken against the running
    // reference as it is; only where a lane's sum of 16 of them is above 2^kLazyRescale (or not a number: no reference yet) is the maximum
    // looked for and everything rescaled.
    __device__ __forceinline__ void weigh(const f32x16& sc, float c, u32x4 (&pw)[2]) {
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
        exponentials(m * c);
        if (__any(!(psum <= kMaxLazyP))) {
            float mx = sc[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
            // a column whose own sums are in range keeps its reference, so that no other row decides how it is rounded
            mx = max_halves(mx);
            mx = max_halves(!(psum <= kMaxLazyP) ? 1.f : 0.f) > 0.f ? mx : m;
            const float m_new = fmaxf(m, mx);
            const float m_use = m_new == NEG_INF ? 0.f : m_new;
            const float alpha = fast_exp2((m - m_use) * c);  // m = -inf gives 0, the same reference exactly 1
            l *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
            m = m_new;
            psum = 0.f;
            exponentials(m_use * c);
        }
        l += psum;
    }
};

// What the two kinds of tile share: where a lane is, and what it does with tokens that not every row sees.
template <int HD, bool FP8>
struct Lane {
    typedef typename Granule<FP8>::type Raw;
    static constexpr int EB = FP8 ? 1 : 2, KS = HD / 16, DB = HD / 32;
    static constexpr int BLOCK = kPage * HD * EB;  // bytes of a page's K, or V, of a head
    const PrefixParams& P;
    const PrefixItem& it;
    int lane, wave, h, l32;
    int k_at, v_at;       // bytes: of the lane's first operand in a block of K, of V
    const char* pool;     // the head's K block of page 0
    int64_t page_bytes;

    __device__ __forceinline__ Lane(const PrefixParams& params, const PrefixItem& item) : P(params), it(item) {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        h = lane >> 5;
        l32 = lane & 31;
        // Row r of the K operand is token 8*bit2(r) + 4*bit3(r) + (r & 3) of page bit4(r): registers 8p .. 8p+7 of a lane are then eight
        // consecutive tokens of page p, which is what the second product takes.
        const int k_tok = ((l32 >> 2) & 1) * 8 + ((l32 >> 3) & 1) * 4 + (l32 & 3);
        k_at = (h * 16 + k_tok) * (8 * EB);
        v_at = (h * HD + l32) * (8 * EB);
        pool = static_cast<const char*>(P.pool) + (int64_t)it.kvh * BLOCK;
        page_bytes = P.page_stride * EB;
    }
    __device__ __forceinline__ int64_t v_offset() const { return (int64_t)P.Hkv * BLOCK; }
    __device__ __forceinline__ int row_of(int col) const { return (int)(((unsigned)col * (unsigned)P.invG) >> 16); }

    // Q^T of the column: d = 16 ks + 8 h + ..
    __device__ __forceinline__ void load_q(int col, bf16x8 (&q)[KS]) const {
        const int row = row_of(col);
        const uint16_t* from = P.q + ((int64_t)(it.grow0 + row) * P.Hq + it.kvh * P.G + (col - row * P.G)) * HD + h * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[ks] = as_bf16x8(*reinterpret_cast<const u32x4*>(from + ks * 16));
    }
    __device__ __forceinline__ void mask(f32x16& sc, int base, int limit) const {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (base + (i >> 3) * 16 + h * 8 + (i & 7) > limit) sc[i] = NEG_INF;
    }
    // V of tokens that no row may take from the product: keys behind the last, which were never written, and elements of new tokens that are
    // not finite, where rows that do not see them would take NaN from them.  True where there is one of these.  A dword holds tokens
    // 2e and 2e + 1 of one d; both halves are looked at together: an exponent of all ones, and nothing else, carries into a half's top bit.
    __device__ __forceinline__ bool drop(u32x4 (&v)[2][DB], int base) const {
        uint32_t found = 0;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int pos = base + p * 16 + h * 8 + 2 * e;
                const uint32_t there = pos + 1 < it.kv_total ? ~0u : pos < it.kv_total ? 0x0000FFFFu : 0u;
                const uint32_t is_new = pos >= it.L ? 0x80008000u : pos + 1 >= it.L ? 0x80000000u : 0u;
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    v[p][db][e] &= there;
                    found |= ((v[p][db][e] & 0x7F807F80u) + 0x00800080u) & is_new;
                }
            }
        if (!__any(found != 0)) return false;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int pos = base + p * 16 + h * 8 + 2 * e;
                const uint32_t is_new = pos >= it.L ? 0x80008000u : pos + 1 >= it.L ? 0x80000000u : 0u;
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const uint32_t odd = (((v[p][db][e] & 0x7F807F80u) + 0x00800080u) & is_new) >> 15;
                    v[p][db][e] &= ~(odd * 0xFFFFu);
                }
            }
        return true;
    }
    // Rows that see such elements get them here, whatever their probability.
    __device__ __forceinline__ void add_dropped(Columns<HD>& acc, const int* ids, int base, int limit) const {
        for (int t = 0; t < kSlab; ++t) {
            const int pos = base + t;
            const bool seen = pos <= limit;
            if (pos < it.L || pos >= it.kv_total || !__any(seen)) continue;
            const char* vt = pool + (int64_t)ids[t >> 4] * page_bytes + v_offset() + (((t >> 3) & 1) * (HD * 8) + (t & 7)) * EB;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int d = db * 32 + (i >> 2) * 8 + h * 4 + (i & 3);
                    uint32_t bits;
                    if constexpr (FP8) bits = fp8x4_to_bf16x4(*reinterpret_cast<const uint8_t*>(vt + d * 8))[0] & 0xFFFFu;
                    else bits = *reinterpret_cast<const uint16_t*>(vt + d * 16);
                    if (seen && not_finite_bf16(bits)) acc.o[db][i] += bf16_bits_to_f32(bits);
                }
        }
    }
    // Waves that have the same columns meet in LDS, kStageCols columns at a time; the result leaves as a partial, column after column, or as the
    // rows'.
    template <int KEY_WAVES>
    __device__ __forceinline__ void finish(const Columns<HD>& acc, float* stage, f32x2* stage_ml) const {
        constexpr int ROW = HD + 4;  // the padding spreads the columns over the banks
        const int tid = threadIdx.x;
        const float c = P.scale_log2e, l_tot = sum_halves(acc.l);
        for (int c0 = 0; c0 < 32; c0 += kStageCols) {
            if (c0 >= it.ncols) break;
            __syncthreads();
            if (l32 >= c0 && l32 < c0 + kStageCols && l32 < it.ncols) {
                float* to = stage + (wave * kStageCols + l32 - c0) * ROW + h * 4;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32x4*>(to + db * 32 + i * 8) = f32x4{acc.o[db][4 * i], acc.o[db][4 * i + 1], acc.o[db][4 * i + 2], acc.o[db][4 * i + 3]};
                if (h == 0) stage_ml[wave * kStageCols + l32 - c0] = f32x2{acc.m, l_tot};
            }
            __syncthreads();
            constexpr int BLOCKS = kPrefixWaves / KEY_WAVES;  // of 32 columns
            for (int block = 0; block < BLOCKS; ++block) {
                const int left = it.ncols - block * 32 - c0, cols = left < kStageCols ? left : kStageCols;
                for (int idx = tid; idx < cols * (HD / 4); idx += kPrefixThreads) {
                    const int cl = idx / (HD / 4), d = idx % (HD / 4) * 4;
                    const int cc = block * 32 + c0 + cl;
                    float mm = NEG_INF;
#pragma unroll
                    for (int w = 0; w < KEY_WAVES; ++w) mm = fmaxf(mm, stage_ml[(block * KEY_WAVES + w) * kStageCols + cl][0]);
                    f32x4 o = {0.f, 0.f, 0.f, 0.f};
                    float l = 0.f;
#pragma unroll
                    for (int w = 0; w < KEY_WAVES; ++w) {
                        const int from = (block * KEY_WAVES + w) * kStageCols + cl;
                        const f32x2 ml = stage_ml[from];
                        if (ml[0] == NEG_INF) {  // no key, or none but scores of minus infinity; the sum is 0, or NaN where one was NaN
                            l += ml[1];
                            continue;
                        }
                        const float f = fast_exp2((ml[0] - mm) * c);
                        l += f * ml[1];
                        o += f * *reinterpret_cast<const f32x4*>(stage + from * ROW + d);
                    }
                    if (it.part_off >= 0) {
                        float* to = P.partials + it.part_off;
                        *reinterpret_cast<partial4*>(to + cc * HD + d) = o;
                        if (d == 0) *reinterpret_cast<f32x2*>(to + it.ncols * HD + cc * 2) = f32x2{mm, l};
                    } else {
                        store_result(cc, d, o, l);
                    }
                }
            }
        }
    }
    __device__ __forceinline__ void store_result(int cc, int d, const f32x4& o, float l) const {
        const int row = row_of(cc);
        const int64_t at = (int64_t)(it.grow0 + row) * P.Hq + it.kvh * P.G + (cc - row * P.G);
        const f32x4 r = o * ((l == 0.f ? 0.f : 1.0f / l) * P.v_scale);  // a row whose scores are all minus infinity gives zeros
        *reinterpret_cast<u32x2*>(P.out + at * HD + d) = u32x2{pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
    }
    // A wave whose columns no other has: from registers.  Partials lie as the registers do, so that a store is one run of memory
    // (through LDS and by rows it took 5 us of a tile's 25).
    __device__ __forceinline__ void finish_alone(const Columns<HD>& acc, int col0) const {
        const float l_tot = sum_halves(acc.l);
        const int cc = col0 + l32;
        if (cc >= it.ncols) return;
        float* const to = P.partials + it.part_off;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 o = {acc.o[db][4 * i], acc.o[db][4 * i + 1], acc.o[db][4 * i + 2], acc.o[db][4 * i + 3]};
                const int d = db * 32 + i * 8 + h * 4;
                if (it.part_off >= 0) *reinterpret_cast<partial4*>(to + partial_at<HD>(it.ncols, cc, d)) = o;
                else store_result(cc, d, o, l_tot);
            }
        if (it.part_off >= 0 && h == 0) *reinterpret_cast<f32x2*>(to + it.ncols * HD + cc * 2) = f32x2{acc.m, l_tot};
    }
};

// Up to 32 columns, which all waves have: each takes every fourth slab of 32 keys from the pool straight into registers in the layouts of
// the matrix instructions' operands: no LDS, no barrier, until the waves' results meet.  Probabilities enter the second product as bf16
// numbers, as the matrix instruction takes them (their sum is of the 32-bit ones); everything else is held in 32 bits.
// 512 tiles of 72-679 keys beside others (64 decodes behind 8000 tokens): 4.5-17 us each, a line through them 5.7 us and 2.4 for every 128
// keys; 18-192 keys on an empty chip 2.5 us and 0.4: memory.
template <int HD, bool FP8>
__device__ __forceinline__ void few_columns(const PrefixParams& P, const PrefixItem& it, const int* ids, float* stage, f32x2* stage_ml) {
    typedef Lane<HD, FP8> At;
    typedef typename At::Raw Raw;
    constexpr int KS = At::KS, DB = At::DB, EB = At::EB;
    const At at(P, it);
    const int col = at.l32 < it.ncols ? at.l32 : it.ncols - 1;
    const float c = P.scale_log2e;
    const int limit = it.L + at.row_of(col);  // the last key that the row sees
    const int slabs = (it.kv_end - it.kv_begin + kSlab - 1) / kSlab;
    bf16x8 q[KS];
    at.load_q(col, q);
    const char* const k_lane = at.pool + at.k_at;
    const char* const v_lane = at.pool + at.v_offset() + at.v_at;
    // Read once: non-temporal loads.
    Raw kr[KS], vr[2][DB];
    auto load_k = [&](int s) {
        const char* p = k_lane + (int64_t)ids[s * 2 + (at.l32 >> 4)] * at.page_bytes;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kr[ks] = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(p + ks * (2 * 16 * 8 * EB)));
    };
    auto load_v = [&](int s) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const char* vp = v_lane + (int64_t)__builtin_amdgcn_readfirstlane(ids[s * 2 + p]) * at.page_bytes;
#pragma unroll
            for (int db = 0; db < DB; ++db) vr[p][db] = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(vp + db * (32 * 8 * EB)));
        }
    };
    Columns<HD> acc;
    acc.clear();
    // One slab.  The next one's K is asked for when this one's has been used, and its V likewise, so that a slab is on its way while another
    // is worked.  A wave's last slab asks for none; with at most 32 new tokens, in neighbouring slabs at the end of the range, it alone can
    // hold any, so only its code looks at what is seen.  (A load that is asked for in one branch and not in another would have to
    // be waited for together with all that came behind it.)
    auto step = [&](int s, auto last) {
        constexpr bool LAST = decltype(last)::value;
        const int base = it.kv_begin + s * kSlab;
        f32x16 sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(operand(kr[ks])), q[ks], sc, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!LAST) load_k(s + kPrefixWaves);
        __builtin_amdgcn_sched_barrier(0);
        bool strange = false;
        u32x4 vv[2][DB], pw[2];
        if constexpr (LAST) {
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int db = 0; db < DB; ++db) vv[p][db] = operand(vr[p][db]);
            if (base + kSlab > it.L) {
                at.mask(sc, base, limit);
                strange = at.drop(vv, base);
            }
        }
        acc.weigh(sc, c, pw);
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const u32x4 v = LAST ? vv[p][db] : operand(vr[p][db]);
                acc.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v), as_bf16x8(pw[p]), acc.o[db], 0, 0, 0);
            }
        if constexpr (LAST) {
            if (strange) at.add_dropped(acc, ids + s * 2, base, limit);
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!LAST) load_v(s + kPrefixWaves);
        __builtin_amdgcn_sched_barrier(0);
    };
    int s = at.wave;
    if (s < slabs) {
        load_k(s);
        load_v(s);
        for (; s + kPrefixWaves < slabs; s += kPrefixWaves) step(s, std::false_type{});
        step(s, std::true_type{});
    }
    at.template finish<kPrefixWaves>(acc, stage, stage_ml);
}

// 33 to 128 columns: KEY_WAVES waves have the same 32, each with every KEY_WAVES-th slab of 32 keys.  A slab's K and V go from the pool
// straight to a ring in LDS, a quarter by each wave, and are read from there by all (64 decodes behind 8000 tokens
// 44 us as first built, 49 with each wave reading for itself from L2; on two boxes).
// A slab of 128 columns takes 1.02 us with two workgroups to a unit, 1.07 on FP8 pages; three documents of 18000 tokens with 256 columns each
// 73 us for 57 GFLOP, 0.78 PFLOP/s, matrix pipes 30 % busy.  LDS, matrix and vector instructions follow each other in a wave, and two waves to a
// SIMD overlap them in part.  Without the loads the same batch took 71 us a call instead of 93, without the conversions of FP8 84 instead of 90.
template <int HD, bool FP8>
struct Ring {
    static constexpr int SLAB = 4 * Lane<HD, FP8>::BLOCK;  // bytes: K of two pages, V of two pages
    static constexpr int STAGES = 65536 / SLAB < 8 ? 65536 / SLAB : 8;
    static constexpr int BYTES = STAGES * SLAB;
};
template <int HD, bool FP8, int KEY_WAVES>
__device__ __forceinline__ void many_columns(const PrefixParams& P, const PrefixItem& it, const int* ids, char* ring, f32x2* stage_ml) {
    typedef Lane<HD, FP8> At;
    typedef typename At::Raw Raw;
    constexpr int KS = At::KS, DB = At::DB, EB = At::EB, BLOCK = At::BLOCK;
    constexpr int SLAB = Ring<HD, FP8>::SLAB, STAGES = Ring<HD, FP8>::STAGES, LOADS = BLOCK / 1024;
    static_assert(BLOCK % 1024 == 0, "a wave moves 1 KiB at a time");
    const At at(P, it);
    const int col0 = at.wave / KEY_WAVES * 32;  // it may lie behind the last
    const int col = col0 + at.l32 < it.ncols ? col0 + at.l32 : it.ncols - 1;
    const float c = P.scale_log2e;
    const int limit = it.L + at.row_of(col);
    const int slabs = (it.kv_end - it.kv_begin + kSlab - 1) / kSlab;
    // wave w brings block w of a slab: K of its two pages, V of its two pages
    const char* const from = at.pool + (at.wave >> 1 ? at.v_offset() : 0);
    const uint32_t ring_addr = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)ring) + (uint32_t)at.wave * BLOCK;
    auto bring = [&](int s) {
        const char* page = from + (int64_t)__builtin_amdgcn_readfirstlane(ids[s * 2 + (at.wave & 1)]) * at.page_bytes;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) lds_direct_load16_at(page + j * 1024, (uint32_t)at.lane * 16u, ring_addr + (uint32_t)(s % STAGES * SLAB + j * 1024));
    };
    bf16x8 q[KS];
    at.load_q(col, q);
    for (int s = 0; s < STAGES - KEY_WAVES && s < slabs; ++s) bring(s);
    Columns<HD> acc;
    acc.clear();
    const bool active = col0 < it.ncols;
    f32x16 sc;
    auto k_operand = [&](int s, int ks) { return operand(*reinterpret_cast<const Raw*>(ring + s % STAGES * SLAB + (at.l32 >> 4) * BLOCK + at.k_at + ks * (2 * 16 * 8 * EB))); };
    auto v_operand = [&](int s, int j) { return operand(*reinterpret_cast<const Raw*>(ring + s % STAGES * SLAB + (2 + j / DB) * BLOCK + at.v_at + j % DB * (32 * 8 * EB))); };
    auto scores = [&](int s) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k_operand(s, ks)), q[ks], sc, 0, 0, 0);
    };
    // Exponentials of slab s, whose scores are in sc, then its part of O, and, NEXT, the scores of slab s + 1 in one run of products, whose
    // operands are read ahead of them.  (After the last slab: of whatever the ring holds, not used.)
    auto work = [&](int s, auto masked, auto next) {
        constexpr bool MASKED = decltype(masked)::value, NEXT = decltype(next)::value;
        const int base = it.kv_begin + s * kSlab;
        u32x4 vv[2][DB], pw[2];
        bool strange = false;
        if constexpr (MASKED) {
#pragma unroll
            for (int j = 0; j < 2 * DB; ++j) vv[j / DB][j % DB] = v_operand(s, j);
            at.mask(sc, base, limit);
            strange = at.drop(vv, base);
        }
        acc.weigh(sc, c, pw);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (MASKED || !NEXT) {
#pragma unroll
            for (int j = 0; j < 2 * DB; ++j) {
                const u32x4 v = MASKED ? vv[j / DB][j % DB] : v_operand(s, j);
                acc.o[j % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v), as_bf16x8(pw[j / DB]), acc.o[j % DB], 0, 0, 0);
            }
            if constexpr (NEXT) scores(s + 1);
        } else {
            constexpr int PRODUCTS = 2 * DB + KS, AHEAD = 4;
            __builtin_amdgcn_s_setprio(1);  // before the other workgroup's exponentials (96 decodes over documents, FP8, 113 -> 109 us)
            auto read = [&](int j) { return j < 2 * DB ? v_operand(s, j) : k_operand(s + 1, j - 2 * DB); };
            u32x4 buf[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) buf[j] = read(j);
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
            for (int j = 0; j < PRODUCTS; ++j) {
                const bf16x8 a = as_bf16x8(buf[j % AHEAD]);
                if (j < 2 * DB) acc.o[j % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, as_bf16x8(pw[j / DB]), acc.o[j % DB], 0, 0, 0);
                else sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[j - 2 * DB], sc, 0, 0, 0);
                if (j + AHEAD < PRODUCTS) buf[j % AHEAD] = read(j + AHEAD);
            }
            if constexpr (!FP8) {
                __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
                for (int j = 0; j < PRODUCTS - AHEAD; ++j) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
            }
            __builtin_amdgcn_s_setprio(0);
        }
        if constexpr (MASKED) {
            if (strange) at.add_dropped(acc, ids + s * 2, base, limit);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // Behind it every wave's part of what was waited for is there, and what was worked before is free.
    auto barrier = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    // A wave's own slabs are there once it has waited for all but the newest of its loads.
    auto wait_all_but = [](auto newer, bool all_issued) {
        if (all_issued) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(newer)::value) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    // One loop for the slabs that all rows see and one for the others: with a branch between the two in one loop O changes its registers in
    // every iteration.
    const int clear = it.L <= it.kv_begin ? 0 : (it.L - it.kv_begin) / kSlab;
    int s = 0;
    if constexpr (KEY_WAVES == 1) {
        // slab s is worked, s + 1 there, the others on their way
        auto turn = [&](auto masked) {
            wait_all_but(std::integral_constant<int, (STAGES - 3) * LOADS>{}, s + STAGES - 1 <= slabs);
            barrier();
            if (s + STAGES - 1 < slabs) bring(s + STAGES - 1);
            if (active) work(s, masked, yes);
        };
        wait_all_but(std::integral_constant<int, (STAGES - 2) * LOADS>{}, STAGES - 1 <= slabs);
        barrier();
        if (active) scores(0);
        for (; s < slabs && s < clear; ++s) turn(no);
        for (; s < slabs; ++s) turn(yes);
    } else {
        // KEY_WAVES slabs are worked, the others on their way
        auto turn = [&](auto masked) {
            wait_all_but(std::integral_constant<int, (STAGES - 2 * KEY_WAVES) * LOADS>{}, s + STAGES - KEY_WAVES <= slabs);
            barrier();
#pragma unroll
            for (int j = 0; j < KEY_WAVES; ++j)
                if (s + STAGES - KEY_WAVES + j < slabs) bring(s + STAGES - KEY_WAVES + j);
            const int mine = s + at.wave % KEY_WAVES;
            if (mine >= slabs || !active) return;
            scores(mine);
            work(mine, masked, no);
        };
        for (; s < slabs && s + KEY_WAVES <= clear; s += KEY_WAVES) turn(no);
        for (; s < slabs; s += KEY_WAVES) turn(yes);
    }
    if constexpr (KEY_WAVES == 1) at.finish_alone(acc, col0);
    else at.template finish<KEY_WAVES>(acc, reinterpret_cast<float*>(ring), stage_ml);
}

template <int HD, bool FP8>
__global__ __launch_bounds__(kPrefixThreads, 2) void ppd_prefix_kernel(const PrefixParams P) {
    constexpr int STAGE = kPrefixWaves * kStageCols * (HD + 4) * 4;
    __shared__ int ids[kMaxPrefixChunk / kPage];
    __shared__ __attribute__((aligned(1024))) char area[Ring<HD, FP8>::BYTES > STAGE ? Ring<HD, FP8>::BYTES : STAGE];  // the ring, then the waves' results
    __shared__ f32x2 stage_ml[kPrefixWaves * kStageCols];
    const PrefixItem it = P.items[blockIdx.x];
    // Page ids of the tile's keys, checked, to LDS: an id outside the pool raises the sticky flag and is replaced by page 0.
    {
        const int32_t* row = P.page_tables + (int64_t)it.seq * P.max_pages;
        const int last = (it.kv_total - 1) / kPage, first = it.kv_begin / kPage;
        const int count = (it.kv_end - it.kv_begin + kSlab - 1) / kSlab * (kSlab / kPage);
        for (int i = threadIdx.x; i < count; i += kPrefixThreads) {
            int id = row[first + i < last ? first + i : last];
            if (id < 0 || id >= P.num_pages) {
                atomicOr(P.err_flags, 2u);
                id = 0;
            }
            ids[i] = id;
        }
    }
    __syncthreads();
    switch (prefix_key_waves(it.ncols)) {
        case 4: few_columns<HD, FP8>(P, it, ids, reinterpret_cast<float*>(area), stage_ml); break;
        case 2: many_columns<HD, FP8, 2>(P, it, ids, area, stage_ml); break;
        default: many_columns<HD, FP8, 1>(P, it, ids, area, stage_ml); break;
    }
}

// Joins the partials of a unit's columns, sources in order and splits in order: a workgroup has up to 256 / (HD / 4) columns of one KV head,
// and where they are fewer, its threads share the splits.  64 decodes of 32 query heads with 16 partials each 6.6 us (one thread through all of
// them 15), 1140 rows of 40 with 3 22 us, 3.6 TB/s.  Bound by latency: where each partial is goes to LDS first, then all (m, l)
// pairs at once, and a lane asks for eight partials' values before it adds the first.
constexpr int kJoinParts = 256;   // partials that are looked at at a time
constexpr int kJoinPairs = 1024;  // (m, l) pairs in LDS
template <int HD>
__global__ __launch_bounds__(256) void ppd_prefix_join_kernel(const PrefixParams P) {
    constexpr int LANES = HD / 4, COLS = 256 / LANES, AT_ONCE = 8;
    __shared__ JoinSource sources[kMaxNested + 1];
    __shared__ int64_t part_at[kJoinParts];  // floats: the partial
    __shared__ int part_cols[kJoinParts], part_col0[kJoinParts];  // its columns (negative: of a row block), the workgroup's first among them
    __shared__ f32x2 ml[kJoinPairs];
    __shared__ f32x4 other[256];
    const JoinUnit u = P.units[blockIdx.x];
    const int tid = threadIdx.x, kvh = blockIdx.y, col0 = (int)blockIdx.z * COLS, cols = u.nrows * P.G - col0 < COLS ? u.nrows * P.G - col0 : COLS;
    if (tid < P.source_stride) sources[tid] = P.sources[(int64_t)blockIdx.x * P.source_stride + tid];
    if (cols <= 0) return;
    __syncthreads();
    int parts = 0;
    for (int i = 0; i < u.nsources; ++i) parts += sources[i].nsplit;
    int share = 1;  // threads of a column and d: each has every share-th partial
    while (2 * share * cols <= COLS && share < parts) share *= 2;
    const float c = P.scale_log2e;
    // in the order in which the partials lie: four columns side by side, or row after row
    const bool by_rows = sources[0].by_rows;
    const int cl = by_rows ? tid / LANES % cols : tid % cols, d = (by_rows ? tid % LANES : tid / cols % LANES) * 4, mine = tid / LANES / cols;
    const bool works = mine < share;
    const int most = kJoinPairs / cols < kJoinParts ? kJoinPairs / cols : kJoinParts;
    float m = NEG_INF, l = 0.f;  // of the column, all threads alike
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < parts; p0 += most) {
        const int count = parts - p0 < most ? parts - p0 : most;
        if (p0 > 0) __syncthreads();
        for (int i = tid; i < count; i += 256) {
            int part = p0 + i, from = 0;
            while (part >= sources[from].nsplit) part -= sources[from++].nsplit;
            const JoinSource x = sources[from];
            part_at[i] = x.part_off + ((int64_t)kvh * x.nsplit + part) * x.ncols * (HD + 2);
            part_cols[i] = x.by_rows ? -x.ncols : x.ncols;
            part_col0[i] = x.col0 + col0;
        }
        __syncthreads();
        for (int i = tid; i < count * cols; i += 256) {
            const int part = i / cols;
            const int ncols = part_cols[part] < 0 ? -part_cols[part] : part_cols[part];
            ml[i] = *reinterpret_cast<const f32x2*>(P.partials + part_at[part] + ncols * HD + (part_col0[part] + i - part * cols) * 2);
        }
        f32x4 v[AT_ONCE];
        auto ask = [&](int j0) {
#pragma unroll
            for (int t = 0; t < AT_ONCE; ++t) {
                if (j0 - mine + t * share >= count) break;  // for all threads alike; where it is for some, the first one's again
                const int j = j0 + t * share < count ? j0 + t * share : 0;
                const int cc = part_col0[j] + cl;
                v[t] = *reinterpret_cast<const partial4*>(P.partials + part_at[j] + (part_cols[j] < 0 ? cc * HD + d : partial_at<HD>(part_cols[j], cc, d)));
            }
        };
        ask(mine);
        __syncthreads();
        float top = m;
        for (int j = 0; j < count; ++j) top = fmaxf(top, ml[j * cols + cl][0]);
        const float f0 = m == NEG_INF ? 0.f : fast_exp2((m - top) * c);
        l *= f0;
        o *= f0;
        m = top;
        for (int j = 0; j < count; ++j) {
            const f32x2 w = ml[j * cols + cl];
            l += w[0] != NEG_INF ? fast_exp2((w[0] - top) * c) * w[1] : w[1];  // 0, or NaN where a score was NaN
        }
        if (works) {
            for (int j0 = mine; j0 < count; j0 += AT_ONCE * share) {
                if (j0 > mine) ask(j0);
#pragma unroll
                for (int t = 0; t < AT_ONCE; ++t) {
                    if (j0 + t * share >= count) continue;
                    const float mw = ml[(j0 + t * share) * cols + cl][0];
                    if (mw != NEG_INF) o += fast_exp2((mw - top) * c) * v[t];
                }
            }
        }
    }
    if (share > 1) {
        other[tid] = o;
        __syncthreads();
        if (mine == 0)
            for (int k = 1; k < share; ++k) o += other[tid + k * cols * LANES];
    }
    if (mine != 0) return;
    const int col = col0 + cl, row = (int)(((unsigned)col * (unsigned)P.invG) >> 16);
    const int64_t at = (int64_t)(u.grow0 + row) * P.Hq + kvh * P.G + (col - row * P.G);
    const f32x4 r = o * ((l == 0.f ? 0.f : 1.0f / l) * P.v_scale);
    *reinterpret_cast<u32x2*>(P.out + at * HD + d) = u32x2{pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
}

int launch_prefix(const PrefixParams& p, int head_dim, bool fp8_pages, void* stream) {
    hipStream_t hs = static_cast<hipStream_t>(stream);
    auto* const kernel = head_dim == 128 ? (fp8_pages ? &ppd_prefix_kernel<128, true> : &ppd_prefix_kernel<128, false>)
                                         : (fp8_pages ? &ppd_prefix_kernel<64, true> : &ppd_prefix_kernel<64, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.n_items), dim3(kPrefixThreads), 0, hs, p);
    return (int)hipGetLastError();
}

int launch_prefix_join(const PrefixParams& p, int head_dim, void* stream) {
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const int cols = 256 / (head_dim / 4);
    const dim3 grid((unsigned)p.n_units, (unsigned)p.Hkv, (unsigned)((p.join_cols + cols - 1) / cols));
    if (head_dim == 128) hipLaunchKernelGGL(ppd_prefix_join_kernel<128>, grid, dim3(256), 0, hs, p);
    else hipLaunchKernelGGL(ppd_prefix_join_kernel<64>, grid, dim3(256), 0, hs, p);
    return (int)hipGetLastError();
}

}  // namespace ppd
