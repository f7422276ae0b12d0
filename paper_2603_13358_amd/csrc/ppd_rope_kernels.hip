// gfx950 kernels of the rotation by positions.
//
//   (a, b) -> A (a cos t - b sin t, b cos t + a sin t),   t = position * frequency of the pair
//
// The angle is an integer: a frequency is a fraction of a turn in units of 2^-64, so position * frequency modulo 2^64 is the angle
// without its whole turns, for every 64-bit position.  It is off by position * 2^-64 turns at most where a frequency is at most one radian: 2^-65
// is the rounding to units, and 0.7 * 2^-65 what the division by 2 pi in 64-bit significands leaves (2^-63 of the turns).  Its upper 32
// bits become a binary32 fraction of a turn in [-1/2, 1/2), which is what the sine and cosine instructions take: of all 2^32 such fractions
// none is off by more than 2^-22.9 (against 64 bits).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ppd_append.h"
#include "ppd_rope.h"

namespace ppd {

namespace {

// Where pair i of a head is: elements (i, i + rotary_dim / 2) with whole granules of 8 on both sides, or without, or (2i, 2i + 1).
enum Layout { HALF, HALF_ODD, INTERLEAVED };

// 16 elements of a head, two granules: 8 pairs, or, HALF_ODD, elements whose partners other lanes of the wave have.
struct Unit {
    u32x4 g[2];
};

template <Layout LAYOUT>
__device__ __forceinline__ int granule_of(int unit, int which, int rotary_dim) {
    const int rotated = rotary_dim / 16;
    if (LAYOUT == HALF && unit < rotated) return unit + which * rotated;
    return 2 * unit + which;
}

template <Layout LAYOUT>
__device__ __forceinline__ Unit load_unit(const uint16_t* head, int unit, int rotary_dim) {
    Unit x;
#pragma unroll
    for (int w = 0; w < 2; ++w) x.g[w] = APPEND_LOAD(reinterpret_cast<const u32x4*>(head + granule_of<LAYOUT>(unit, w, rotary_dim) * 8));
    return x;
}
template <Layout LAYOUT, bool STREAM = false>
__device__ __forceinline__ void store_unit(uint16_t* head, const Unit& x, int unit, int rotary_dim) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        u32x4* const to = reinterpret_cast<u32x4*>(head + granule_of<LAYOUT>(unit, w, rotary_dim) * 8);
        if constexpr (STREAM) APPEND_STORE(x.g[w], to);
        else *to = x.g[w];
    }
}

__device__ __forceinline__ float element(const u32x4& g, int e) {
    return e & 1 ? __builtin_bit_cast(float, g[e >> 1] & 0xFFFF0000u) : bf16_bits_to_f32(g[e >> 1] & 0xFFFFu);
}

// LDS of HALF_ODD: a row for every head that the workgroup has at hand
template <int D, Layout LAYOUT>
struct Scratch {
    static constexpr int ROW = D + 8;
    static constexpr int ELEMS = LAYOUT == HALF_ODD ? kSmallThreads / (D / 16) * ROW : 8;
};

// The unit's 16 elements after the rotation, in binary32, where they lie in x.  What is not rotated is x itself: infinities there
// meet no sine.
struct Rotated {
    float v[2][8];
};
template <int D, Layout LAYOUT>
__device__ __forceinline__ Rotated rotate(const Unit& x, int unit, int rotary_dim, const f32x4* table, uint16_t* scratch) {
    constexpr int UNITS = D / 16;
    Rotated y;
    if constexpr (LAYOUT == HALF_ODD) {
        // The lanes of a head leave their elements in LDS, each takes its elements' partners from there.  All are of one wave.
        uint16_t* const row = scratch + threadIdx.x / UNITS * Scratch<D, LAYOUT>::ROW;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int w = 0; w < 2; ++w) *reinterpret_cast<u32x4*>(row + unit * 16 + w * 8) = x.g[w];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const int half = rotary_dim / 2;
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = unit * 16 + w * 8 + e;
                const bool turns = i < rotary_dim, first = i < half;
                const int p = !turns ? 0 : first ? i : i - half;
                const f32x2 cs = reinterpret_cast<const f32x2*>(table)[(p % 8 / 2 * UNITS + p / 8) * 2 + p % 2];
                const float a = element(x.g[w], e), b = bf16_bits_to_f32(row[!turns ? i : first ? i + half : p]);
                y.v[w][e] = turns ? __builtin_fmaf(a, cs[0], first ? -(b * cs[1]) : b * cs[1]) : a;
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x4 cs = table[j * UNITS + unit];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int p = 2 * j + k;  // of the unit's 8 pairs
                const int w0 = LAYOUT == INTERLEAVED ? p / 4 : 0, e0 = LAYOUT == INTERLEAVED ? p % 4 * 2 : p;
                const int w1 = LAYOUT == INTERLEAVED ? p / 4 : 1, e1 = LAYOUT == INTERLEAVED ? p % 4 * 2 + 1 : p;
                const float a = element(x.g[w0], e0), b = element(x.g[w1], e1), c = cs[2 * k], s = cs[2 * k + 1];
                const bool turns = unit * 8 + p < rotary_dim / 2;
                y.v[w0][e0] = turns ? __builtin_fmaf(a, c, -(b * s)) : a;
                y.v[w1][e1] = turns ? __builtin_fmaf(b, c, a * s) : b;
            }
        }
    }
    return y;
}
// The same rounded to bf16; what is not rotated keeps its bits.
template <int D, Layout LAYOUT>
__device__ __forceinline__ Unit rotate_bf16(const Unit& x, int unit, int rotary_dim, const f32x4* table, uint16_t* scratch) {
    const Rotated y = rotate<D, LAYOUT>(x, unit, rotary_dim, table, scratch);
    Unit z;
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // rotary_dim is even: both elements of a dword are rotated or neither (HALF: of all)
            const int first = LAYOUT == HALF ? unit * 16 : unit * 16 + w * 8 + 2 * i;
            z.g[w][i] = first < rotary_dim ? pack_bf16(y.v[w][2 * i], y.v[w][2 * i + 1]) : x.g[w][i];
        }
    return z;
}

// Cosines and sines of TOK rows from t0 on, times the amplitude, to LDS: table[row][j][unit] has pairs 2j and 2j + 1 of the unit, so that
// neighbouring units' reads of 16 bytes lie side by side.  Rows behind the last have the last's.
template <int D, int TOK>
__device__ __forceinline__ void fill_table(const Rotation& rot, const int64_t* positions, int64_t t0, int64_t T, float sin_sign, f32x4* table) {
    constexpr int PAIRS = D / 2, UNITS = D / 16;
    for (int i = threadIdx.x; i < TOK * PAIRS; i += kSmallThreads) {
        const int row = i / PAIRS, pair = i % PAIRS;
        if (pair >= rot.rotary_dim / 2) continue;
        const uint64_t angle = (uint64_t)positions[t0 + row < T ? t0 + row : T - 1] * rot.turns[pair];
        const float turn = (float)(int32_t)(angle >> 32) * 0x1p-32f;
        reinterpret_cast<f32x2*>(table)[((row * 4 + pair % 8 / 2) * UNITS + pair / 8) * 2 + pair % 2] =
            f32x2{__builtin_amdgcn_cosf(turn) * rot.amplitude, __builtin_amdgcn_sinf(turn) * (rot.amplitude * sin_sign)};
    }
}

}  // namespace

constexpr int kMaxGridX = 1 << 22;  // workgroups: a dimension of a launch has to stay below 2^32 threads

// A workgroup has TOK rows, whose cosines and sines its threads make together and leave in LDS; 16 elements of a head to a thread, the next
// ones on their way while they are turned.  Bound by memory: 7931 rows of 32 heads, D = 128, from a packed projection 27 us, 4.8 TB/s read and
// written (a copy 4.9), 16132 of 40 heads 69.5 us, 4.75 TB/s; by halves without whole granules (20 pairs) 30 us for the former, where reading
// every element's partner from memory took 107.  Non-temporal stores were slower (28.5 and 82.5 us).  One row and a decode batch are bound
// by the launch: 2.5 us in the kernel, a chain of positions, sines, LDS.
template <int D, int TOK, Layout LAYOUT>
__global__ __launch_bounds__(kSmallThreads) void ppd_rope_kernel(const RopeParams P) {
    constexpr int UNITS = D / 16;
    __shared__ f32x4 table[TOK * 4 * UNITS];
    __shared__ __attribute__((aligned(16))) uint16_t scratch[Scratch<D, LAYOUT>::ELEMS];
    const int64_t t0 = ((int64_t)blockIdx.y * kMaxGridX + blockIdx.x) * TOK;
    if (t0 >= P.T) return;
    const int unit = threadIdx.x % UNITS, rotary = P.rot.rotary_dim;
    const int rows = P.T - t0 < TOK ? (int)(P.T - t0) : TOK;
    int row = 0, head = threadIdx.x / UNITS;
    auto settle = [&] {  // heads beyond a row's are the next row's
        while (head >= P.heads) {
            head -= P.heads;
            ++row;
        }
    };
    auto load = [&] { return load_unit<LAYOUT>(P.x + (t0 + row) * P.x_stride + head * D, unit, rotary); };
    settle();
    Unit x = {};
    if (row < rows) x = load();
    fill_table<D, TOK>(P.rot, P.positions, t0, P.T, P.sin_sign, table);
    __syncthreads();
    while (row < rows) {
        const int r = row, h = head;
        const Unit now = x;
        head += kSmallThreads / UNITS;
        settle();
        if (row < rows) x = load();
        store_unit<LAYOUT>(P.out + (t0 + r) * P.out_stride + h * D, rotate_bf16<D, LAYOUT>(now, unit, rotary, table + r * 4 * UNITS, scratch), unit, rotary);
    }
}

// Append of rotated keys, and of values, to the page pool; queries rotated beside.  A workgroup has TOK tokens and one KV head
// (blockIdx.x < Hkv), whose rows it stages in LDS and writes as ppd_kv_append_kernel does, or kQueryHeads query heads.
// Bound by memory: 9866 packed tokens (32 query heads, 8 KV heads, D = 128) 46.5-48 us, 5.1 TB/s; with the tokens' tiles of one head after the
// other instead of a token's heads 58; with 8 query heads to a workgroup 50, with 2 53.  16000 tokens to FP8 pages 70 us, 5.1 TB/s.  128
// decodes 4.4 us in the kernel, 1116 tokens of 64 query heads to FP8 pages 12 us (3.5 TB/s): start and end of one round.
constexpr int kQueryHeads = 4;
constexpr int kMaxGridY = 65535;
template <int D, int TOK, bool FP8, Layout LAYOUT>
__global__ __launch_bounds__(kSmallThreads) void ppd_rotated_append_kernel(const RotatedAppendParams P) {
    using Elem = std::conditional_t<FP8, uint8_t, uint16_t>;
    constexpr int UNITS = D / 16, GR = D / 8;
    constexpr int KROW = D + 16 / (int)sizeof(Elem);  // elements of a staged row: 16 bytes of padding spread the rows over the banks
    constexpr int VROW = D + 8;
    __shared__ f32x4 table[TOK * 4 * UNITS];
    __shared__ __attribute__((aligned(16))) Elem sk[TOK * KROW];
    __shared__ __attribute__((aligned(16))) uint16_t sv[(TOK + 7) * VROW];
    __shared__ __attribute__((aligned(16))) uint16_t scratch[Scratch<D, LAYOUT>::ELEMS];
    const int tid = threadIdx.x;
    const int64_t t0 = ((int64_t)blockIdx.z * kMaxGridY + blockIdx.y) * TOK;
    const int rotary = P.rot.rotary_dim;
    if (t0 >= P.T) return;
    if ((int)blockIdx.x >= P.Hkv) {
        const int head0 = ((int)blockIdx.x - P.Hkv) * kQueryHeads, unit = tid % UNITS;
        constexpr int STEP = kSmallThreads / UNITS, ROUNDS = (TOK * kQueryHeads + STEP - 1) / STEP;
        Unit x[ROUNDS];
        bool there[ROUNDS];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int i = tid / UNITS + r * STEP, row = i / kQueryHeads, head = head0 + i % kQueryHeads;
            there[r] = row < TOK && t0 + row < P.T && head < P.Hq;
            if (there[r]) x[r] = load_unit<LAYOUT>(P.q + (t0 + row) * P.q_stride + head * D, unit, rotary);
        }
        fill_table<D, TOK>(P.rot, P.positions, t0, P.T, 1.f, table);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int i = tid / UNITS + r * STEP, row = i / kQueryHeads, head = head0 + i % kQueryHeads;
            if (there[r])
                store_unit<LAYOUT, true>(P.q_out + ((t0 + row) * P.Hq + head) * D, rotate_bf16<D, LAYOUT>(x[r], unit, rotary, table + row * 4 * UNITS, scratch), unit, rotary);
        }
        return;
    }
    // K: the first threads, 8 pairs each; V: the last ones, a granule each
    constexpr int KUNITS = TOK * UNITS, VGRANULES = TOK * GR;
    static_assert(KUNITS <= kSmallThreads && VGRANULES <= kSmallThreads, "a round of loads");
    const int kh = blockIdx.x, krow = tid / UNITS, unit = tid % UNITS;
    const int vg = kSmallThreads - 1 - tid, vrow = vg / GR;
    Unit xk;
    u32x4 xv = {0, 0, 0, 0};
    const bool has_k = tid < KUNITS && t0 + krow < P.T, has_v = vg < VGRANULES;
    if (has_k) xk = load_unit<LAYOUT>(P.k + (t0 + krow) * P.k_stride + kh * D, unit, rotary);
    if (has_v && t0 + vrow < P.T) xv = APPEND_LOAD(reinterpret_cast<const u32x4*>(P.v + (t0 + vrow) * P.v_stride + kh * D + vg % GR * 8));
    const AppendWindow w = append_window<TOK>(P.slots, t0, P.T, P.num_pages, blockIdx.x == 0, P.err_flags);
    if (tid < w.extra * GR)
        *reinterpret_cast<u32x4*>(sv + (TOK + tid / GR) * VROW + (tid % GR) * 8) =
            APPEND_LOAD(reinterpret_cast<const u32x4*>(P.v + (t0 + TOK + tid / GR) * P.v_stride + kh * D + (tid % GR) * 8));
    fill_table<D, TOK>(P.rot, P.positions, t0, P.T, 1.f, table);
    if (has_v) *reinterpret_cast<u32x4*>(sv + vrow * VROW + vg % GR * 8) = xv;
    __syncthreads();
    if (has_k) {
        Elem* const row = sk + krow * KROW;
        if constexpr (FP8) {
            const Rotated y = rotate<D, LAYOUT>(xk, unit, rotary, table + krow * 4 * UNITS, scratch);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                u32x2 codes;
#pragma unroll
                for (int i = 0; i < 2; ++i) codes[i] = e4m3_codes(y.v[g][4 * i], y.v[g][4 * i + 1], y.v[g][4 * i + 2], y.v[g][4 * i + 3], P.inv_k);
                *reinterpret_cast<u32x2*>(row + granule_of<LAYOUT>(unit, g, rotary) * 8) = codes;
            }
        } else {
            store_unit<LAYOUT>(row, rotate_bf16<D, LAYOUT>(xk, unit, rotary, table + krow * 4 * UNITS, scratch), unit, rotary);
        }
    }
    __syncthreads();
    const int64_t S = 2LL * P.Hkv * kPage * D;
    Elem* const to = static_cast<Elem*>(P.pool) + (int64_t)kh * kPage * D;
    // K: work unit = (granule, token), token fastest; whole waves take part
#pragma unroll
    for (int p = 0; p < (TOK * GR + kSmallThreads - 1) / kSmallThreads; ++p) {
        const int u = tid + p * kSmallThreads;
        if (u >= TOK * GR) break;
        const int tok = u % TOK, c = u / TOK;
        const int64_t s = __shfl(w.slot, 7 + tok);
        if (s < 0) continue;
        typedef std::conditional_t<FP8, u32x2, u32x4> Granule;
        APPEND_STORE(*reinterpret_cast<const Granule*>(sk + tok * KROW + c * 8), reinterpret_cast<Granule*>(to + (s >> 4) * S + c * (kPage * 8) + (int)(s & 15) * 8));
    }
    store_v<D, TOK, FP8>(w, sv, VROW, to + (int64_t)P.Hkv * kPage * D, S, P.inv_v);
}

namespace {

Layout layout_of(const Rotation& rot) { return rot.interleaved ? INTERLEAVED : rot.rotary_dim % 16 == 0 ? HALF : HALF_ODD; }

// Calls `go` with the layout as a constant.
template <class F>
void by_layout(const Rotation& rot, F go) {
    switch (layout_of(rot)) {
        case HALF: go(std::integral_constant<Layout, HALF>{}); break;
        case HALF_ODD: go(std::integral_constant<Layout, HALF_ODD>{}); break;
        case INTERLEAVED: go(std::integral_constant<Layout, INTERLEAVED>{}); break;
    }
}

template <int D, int TOK, bool FP8>
void append_launch(const RotatedAppendParams& p, hipStream_t hs) {
    const unsigned queries = p.q ? (unsigned)(p.Hq + kQueryHeads - 1) / kQueryHeads : 0u;
    // the heads of a token beside each other: their rows lie together
    const int64_t tiles = (p.T + TOK - 1) / TOK;
    const dim3 grid((unsigned)p.Hkv + queries, (unsigned)(tiles < kMaxGridY ? tiles : kMaxGridY), (unsigned)((tiles + kMaxGridY - 1) / kMaxGridY));
    by_layout(p.rot, [&](auto layout) { hipLaunchKernelGGL((ppd_rotated_append_kernel<D, TOK, FP8, decltype(layout)::value>), grid, dim3(kSmallThreads), 0, hs, p); });
}

}  // namespace

int launch_rope(const RopeParams& p, int head_dim, void* stream) {
    hipStream_t hs = static_cast<hipStream_t>(stream);
    // Four rows to a workgroup share its start and ask for the next while one is worked; few rows have workgroups to gain.  us with four and with
    // one, D = 128, 20 calls in a replayed graph: 256 rows of 32 heads 3.9 and 2.7, 1024 4.8 and 4.0, 2047 7.0 and 6.4, 3000 9.9 and 9.7, 8192 23.9
    // and 23.4; of 8 heads 1024 rows 2.9 and 3.0, 2047 3.3 and 3.4, 8192 6.9 and 8.4; of 2 heads 1024 3.1 and 3.3, 2047 3.3 and 3.8, 8192 4.5 and
    // 8.5.
    const bool wide = p.T >= 2048;
    const int64_t groups = wide ? (p.T + 3) / 4 : p.T;
    const dim3 grid((unsigned)(groups < kMaxGridX ? groups : kMaxGridX), (unsigned)((groups + kMaxGridX - 1) / kMaxGridX));
    by_layout(p.rot, [&](auto layout) {
        constexpr Layout LAYOUT = decltype(layout)::value;
        auto* const kernel = head_dim == 128 ? (wide ? &ppd_rope_kernel<128, 4, LAYOUT> : &ppd_rope_kernel<128, 1, LAYOUT>)
                                             : (wide ? &ppd_rope_kernel<64, 4, LAYOUT> : &ppd_rope_kernel<64, 1, LAYOUT>);
        hipLaunchKernelGGL(kernel, grid, dim3(kSmallThreads), 0, hs, p);
    });
    return (int)hipGetLastError();
}

int launch_rotated_append(const RotatedAppendParams& p, int head_dim, bool fp8_pages, void* stream) {
    hipStream_t hs = static_cast<hipStream_t>(stream);
    // As in ppd_kv_append 8 tokens to a workgroup where they are few, 16 where they are many: 512 decodes of 8 KV heads 7.6 us with 8 and 8.0 with 16,
    // 1000 tokens 6.3 with either, 2000 11.6 and 10.1, 4000 21.5 and 20.8, 9866 51.8 and 48.3, on FP8 pages 4000 22.0 and 19.9.
    const bool wide = p.T * p.Hkv >= 8192;
    if (head_dim == 128) {
        if (wide) fp8_pages ? append_launch<128, 16, true>(p, hs) : append_launch<128, 16, false>(p, hs);
        else fp8_pages ? append_launch<128, 8, true>(p, hs) : append_launch<128, 8, false>(p, hs);
    } else {
        if (wide) fp8_pages ? append_launch<64, 16, true>(p, hs) : append_launch<64, 16, false>(p, hs);
        else fp8_pages ? append_launch<64, 8, true>(p, hs) : append_launch<64, 8, false>(p, hs);
    }
    return (int)hipGetLastError();
}

}  // namespace ppd
