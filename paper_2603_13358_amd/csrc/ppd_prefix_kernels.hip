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

constexpr int kPrefixWaves = 4, kPrefixThreads = 64 * kPrefixWaves;
constexpr int kStageCols = 16;  // columns of a wave that meet in LDS at a time

}  // namespace

// A wave has 32 columns and takes K and V from the pool straight into registers in the layouts of the matrix instructions' operands.
// KEY_WAVES waves have the same columns, each with every KEY_WAVES-th slab of 32 keys; their results meet in LDS at the end.
// Probabilities enter the second product as bf16 numbers, as the matrix instruction takes them (their sum is of the 32-bit ones);
// everything else is held in 32 bits.
template <int HD, bool FP8, int KEY_WAVES>
__device__ __forceinline__ void prefix_tile(const PrefixParams& P, const PrefixItem& it, const int* ids, float (*stage)[kStageCols * (HD + 4)],
                                            float (*stage_ml)[kStageCols][2]) {
    typedef typename Granule<FP8>::type Raw;
    constexpr int EB = FP8 ? 1 : 2, KS = HD / 16, DB = HD / 32, ROW = HD + 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, l32 = lane & 31;
    const int wave_col0 = wave / KEY_WAVES * 32;  // the wave's first column; it may lie behind the last
    const int col = wave_col0 + l32 < it.ncols ? wave_col0 + l32 : it.ncols - 1;
    const int jrow = (int)(((unsigned)col * (unsigned)P.invG) >> 16), head = it.kvh * P.G + (col - jrow * P.G);
    const float c = P.scale_log2e;
    const int limit = it.L + jrow;  // the last key that the row sees
    const int slabs = (it.kv_end - it.kv_begin + kSlab - 1) / kSlab;

    bf16x8 qreg[KS];
    {
        const uint16_t* qp = P.q + ((int64_t)(it.grow0 + jrow) * P.Hq + head) * HD + h * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qreg[ks] = as_bf16x8(*reinterpret_cast<const u32x4*>(qp + ks * 16));
    }
    // Row r of the K operand is token 8*bit2(r) + 4*bit3(r) + (r & 3) of page bit4(r): registers 8p .. 8p+7 of a lane are then eight
    // consecutive tokens of page p, which is what the second product takes.
    const int k_tok = ((l32 >> 2) & 1) * 8 + ((l32 >> 3) & 1) * 4 + (l32 & 3);
    const char* const pool = static_cast<const char*>(P.pool) + (int64_t)it.kvh * (kPage * HD) * EB;
    const char* const k_lane = pool + (h * 16 + k_tok) * (8 * EB);
    const char* const v_lane = pool + ((int64_t)P.Hkv * (kPage * HD) + (h * HD + l32) * 8) * EB;
    const int64_t page_bytes = P.page_stride * EB;

    // What one wave alone reads is read once: non-temporal loads.
    auto load = [](const char* p) {
        if constexpr (KEY_WAVES == kPrefixWaves) return __builtin_nontemporal_load(reinterpret_cast<const Raw*>(p));
        else return *reinterpret_cast<const Raw*>(p);
    };
    Raw kr[KS], vr[2][DB];
    auto load_k = [&](int s) {
        const char* p = k_lane + (int64_t)ids[s * 2 + (l32 >> 4)] * page_bytes;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kr[ks] = load(p + ks * (2 * 16 * 8 * EB));
    };
    auto load_v = [&](int s) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const char* vp = v_lane + (int64_t)__builtin_amdgcn_readfirstlane(ids[s * 2 + p]) * page_bytes;
#pragma unroll
            for (int db = 0; db < DB; ++db) vr[p][db] = load(vp + db * (32 * 8 * EB));
        }
    };

    f32x16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[db][i] = 0.f;
    float m_run = NEG_INF, l_run = 0.f;

    // One slab.  The next one's K is asked for when this one's has been used, and its V likewise.  AHEAD: there is a next one.  MASKED: the
    // slab may hold new tokens, which not every row sees, or keys behind the last.
    auto step = [&](int s, auto ahead, auto masked) {
        constexpr bool AHEAD = decltype(ahead)::value, MASKED = decltype(masked)::value;
        const int base = it.kv_begin + s * kSlab;
        f32x16 sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(operand(kr[ks])), qreg[ks], sc, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (AHEAD) load_k(s + KEY_WAVES);
        __builtin_amdgcn_sched_barrier(0);
        bool strange = false;  // a new token's V that is not finite: not every row may see it
        u32x4 vv[2][DB];
        if constexpr (MASKED) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (base + (i >> 3) * 16 + h * 8 + (i & 7) > limit) sc[i] = NEG_INF;
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    vv[p][db] = operand(vr[p][db]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int pos = base + p * 16 + h * 8 + e;
                        const bool odd = pos >= it.L && not_finite_bf16(vv[p][db][e >> 1] >> ((e & 1) * 16));
                        strange |= odd && pos < it.kv_total;
                        if (odd || pos >= it.kv_total) vv[p][db][e >> 1] &= (e & 1) ? 0x0000FFFFu : 0xFFFF0000u;
                    }
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
                const u32x4 v = MASKED ? vv[p][db] : operand(vr[p][db]);
                oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v), as_bf16x8(pw[p]), oacc[db], 0, 0, 0);
            }
        if constexpr (MASKED) {
            if (__any(strange)) {
                // Elements that are not finite were left out of the product, where rows that do not see them would have taken NaN from
                // them; rows that do get them here, whatever their probability.
                for (int t = 0; t < kSlab; ++t) {
                    const int pos = base + t;
                    const bool seen = pos <= limit;
                    if (pos < it.L || pos >= it.kv_total || !__any(seen)) continue;
                    const char* vt = pool + ((int64_t)ids[s * 2 + (t >> 4)] * P.page_stride + (int64_t)P.Hkv * (kPage * HD) + ((t >> 3) & 1) * (HD * 8) + (t & 7)) * EB;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int d = db * 32 + (i >> 2) * 8 + h * 4 + (i & 3);
                            uint32_t bits;
                            if constexpr (FP8) bits = fp8x4_to_bf16x4(*reinterpret_cast<const uint8_t*>(vt + d * 8))[0] & 0xFFFFu;
                            else bits = *reinterpret_cast<const uint16_t*>(vt + d * 16);
                            if (seen && not_finite_bf16(bits)) oacc[db][i] += bf16_bits_to_f32(bits);
                        }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (AHEAD) load_v(s + KEY_WAVES);
        __builtin_amdgcn_sched_barrier(0);
    };
    int s = wave % KEY_WAVES;
    if (s < slabs && wave_col0 < it.ncols) {
        load_k(s);
        load_v(s);
        constexpr std::true_type yes{};
        constexpr std::false_type no{};
        for (; s + KEY_WAVES < slabs && it.kv_begin + (s + 1) * kSlab <= it.L; s += KEY_WAVES) step(s, yes, no);
        for (; s + KEY_WAVES < slabs; s += KEY_WAVES) step(s, yes, yes);
        step(s, no, yes);
    }

    const float l_tot = sum_halves(l_run);
    for (int c0 = 0; c0 < 32; c0 += kStageCols) {
        if (c0 >= it.ncols) break;
        __syncthreads();
        if (l32 >= c0 && l32 < c0 + kStageCols) {
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
        constexpr int BLOCKS = kPrefixWaves / KEY_WAVES;  // of 32 columns
        for (int idx = tid; idx < BLOCKS * kStageCols * (HD / 4); idx += kPrefixThreads) {
            const int d = idx % (HD / 4) * 4, cl = idx / (HD / 4) % kStageCols, block = idx / (HD / 4 * kStageCols);
            const int cc = block * 32 + c0 + cl;
            if (cc >= it.ncols) continue;
            float mm = NEG_INF;
#pragma unroll
            for (int w = 0; w < KEY_WAVES; ++w) mm = fmaxf(mm, stage_ml[block * KEY_WAVES + w][cl][0]);
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
            float l = 0.f;
#pragma unroll
            for (int w = 0; w < KEY_WAVES; ++w) {
                const float mw = stage_ml[block * KEY_WAVES + w][cl][0];
                const float f = mw == NEG_INF ? 0.f : fast_exp2((mw - mm) * c);
                l += f * stage_ml[block * KEY_WAVES + w][cl][1];
                if (mw != NEG_INF) o += f * *reinterpret_cast<const f32x4*>(&stage[block * KEY_WAVES + w][cl * ROW + d]);
            }
            if (it.part_off >= 0) {
                float* to = P.partials + it.part_off;
                *reinterpret_cast<f32x4*>(to + cc * HD + d) = o;
                if (d == 0) *reinterpret_cast<f32x2*>(to + it.ncols * HD + cc * 2) = f32x2{mm, l};
            } else {
                const int row = (int)(((unsigned)cc * (unsigned)P.invG) >> 16);
                const int64_t at = (int64_t)(it.grow0 + row) * P.Hq + it.kvh * P.G + (cc - row * P.G);
                const f32x4 r = o * ((l == 0.f ? 0.f : 1.0f / l) * P.v_scale);  // a row whose scores are all minus infinity gives zeros
                *reinterpret_cast<u32x2*>(P.out + at * HD + d) = u32x2{pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
            }
        }
    }
}

template <int HD, bool FP8>
__global__ __launch_bounds__(kPrefixThreads, 2) void ppd_prefix_kernel(const PrefixParams P) {
    __shared__ int ids[kMaxPrefixChunk / kPage];
    __shared__ __attribute__((aligned(16))) float stage[kPrefixWaves][kStageCols * (HD + 4)];  // the padding spreads the columns over the banks
    __shared__ float stage_ml[kPrefixWaves][kStageCols][2];
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
        case 4: prefix_tile<HD, FP8, 4>(P, it, ids, stage, stage_ml); break;
        case 2: prefix_tile<HD, FP8, 2>(P, it, ids, stage, stage_ml); break;
        default: prefix_tile<HD, FP8, 1>(P, it, ids, stage, stage_ml); break;
    }
}

// Joins the partials of a unit's columns, sources in order and splits in order: a workgroup has 256 / (HD / 4) columns of one KV head.
template <int HD>
__global__ __launch_bounds__(256) void ppd_prefix_join_kernel(const PrefixParams P) {
    constexpr int LANES = HD / 4, COLS = 256 / LANES;
    const JoinUnit u = P.units[blockIdx.x];
    const int kvh = blockIdx.y, col = (int)blockIdx.z * COLS + threadIdx.x / LANES, d = threadIdx.x % LANES * 4;
    if (col >= u.nrows * P.G) return;
    const float c = P.scale_log2e;
    float m = NEG_INF, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < u.nsources; ++i) {
        const JoinSource x = P.sources[u.source0 + i];
        const int64_t stride = (int64_t)x.ncols * (HD + 2);
        const float* from = P.partials + x.part_off + (int64_t)kvh * x.nsplit * stride;
        const int cc = x.col0 + col;
        for (int j = 0; j < x.nsplit; ++j, from += stride) {
            const f32x2 w = *reinterpret_cast<const f32x2*>(from + x.ncols * HD + cc * 2);
            if (w[0] == NEG_INF) continue;
            const f32x4 v = *reinterpret_cast<const f32x4*>(from + cc * HD + d);
            const float top = fmaxf(m, w[0]);
            const float f0 = m == NEG_INF ? 0.f : fast_exp2((m - top) * c), f1 = fast_exp2((w[0] - top) * c);
            l = l * f0 + w[1] * f1;
            o = o * f0 + v * f1;
            m = top;
        }
    }
    const int row = (int)(((unsigned)col * (unsigned)P.invG) >> 16);
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
