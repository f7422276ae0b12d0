// Device helpers that the kernels of libppd share: vector types, packing, lane exchanges, FP8 codes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ppd_internal.h"

namespace ppd {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float partial4 __attribute__((ext_vector_type(4), aligned(4 * kPartialAlign)));  // four values of a partial, in the workspace
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#define NEG_INF (-__builtin_inff())

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    f32x2 f = {a, b};
    bf16x2 r = __builtin_convertvector(f, bf16x2);  // round to nearest even
    return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ float xor_shuffle(float v, int mask) { return __shfl_xor(v, mask, 64); }

// max / sum of v over lanes l and l^32 (v_permlane32_swap: no LDS round trip).  The instruction exchanges
// the upper half of its first register with the lower half of its second.  It is written as inline asm on
// two copies of v (the builtin's second result was folded into the first by the compiler when both inputs
// hold the same value); the s_nop cover the VALU-write -> permlane-read wait states on both sides.
__device__ __forceinline__ void swap_halves(float v, float* lo, float* hi) {
    float a = v, b = v;
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
    *lo = a;  // {v[0..31], v[0..31]}
    *hi = b;  // {v[32..63], v[32..63]}
}
__device__ __forceinline__ float max_halves(float v) {
    float lo, hi;
    swap_halves(v, &lo, &hi);
    return fmaxf(lo, hi);
}
__device__ __forceinline__ float sum_halves(float v) {
    float lo, hi;
    swap_halves(v, &lo, &hi);
    return lo + hi;
}

// The running maximum is only raised (and the accumulators rescaled) when it would grow by more than this many
// powers of two; until then probabilities may exceed 1, by at most 2^kLazyRescale.  The final o / l is unchanged.
// (Row-block tiles do not look for the maximum: there the bound is on the sum of a lane's 32 probabilities.)
#ifndef kLazyRescale
#define kLazyRescale 8.0f
#endif
constexpr float power_of_two(float e) { return e >= 1.0f ? 2.0f * power_of_two(e - 1.0f) : 1.0f; }
constexpr float kMaxLazyP = power_of_two(kLazyRescale);
static_assert((int)kLazyRescale == kLazyRescale, "a whole number of powers of two");

// FP8 pages hold OCP FP8 E4M3 codes (1 sign, 4 exponent bits of bias 7, 3 mantissa bits).  Every code's value is a
// bf16 number, so the tiles turn codes into bf16 MFMA operands exactly; the tensor's scale is applied once, to the
// scores (K) and to the final output (V).
// Four codes of a dword -> four bf16, in order (the conversion instruction takes the two codes of one 16-bit half).
__device__ __forceinline__ u32x2 fp8x4_to_bf16x4(uint32_t w) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
    return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}
__device__ __forceinline__ u32x4 fp8x8_to_bf16x8(u32x2 w) {
    const u32x2 a = fp8x4_to_bf16x4(w[0]), b = fp8x4_to_bf16x4(w[1]);
    return u32x4{a[0], a[1], b[0], b[1]};
}

// Clamp to the code's range with the NaN-propagating minimum and maximum: magnitudes from 448 on (infinities included)
// become 448, a NaN stays one.
__device__ __forceinline__ float e4m3_clamp(float y) {
    return __builtin_elementwise_minimum(__builtin_elementwise_maximum(y, -448.0f), 448.0f);
}
__device__ __forceinline__ float bf16_bits_to_f32(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

// Codes of x * inv for the four bf16 of two dwords, in order: one binary32 product each, clamped, then the conversion
// instruction (two values each; nearest, ties to the even code; a clamped value cannot overflow).  Its treatment of
// ties and subnormals is what the definition asks for -- the tests compare every bf16 bit pattern with the oracle.
// 5 vector instructions per element; the same decision in integer arithmetic on the bits took ~25 and bound the
// append of FP8 pages (landing of 5589 tokens x 32 layers: 314 us, now 255).
__device__ __forceinline__ uint32_t e4m3_codes(uint32_t lo, uint32_t hi, float inv) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(bf16_bits_to_f32(lo & 0xFFFFu) * inv),
                                            e4m3_clamp(__builtin_bit_cast(float, lo & 0xFFFF0000u) * inv), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(bf16_bits_to_f32(hi & 0xFFFFu) * inv),
                                        e4m3_clamp(__builtin_bit_cast(float, hi & 0xFFFF0000u) * inv), w, true);
    // the instruction gives every NaN the same sign: the codes take theirs from the inputs (inv > 0)
    const uint32_t signs = __builtin_amdgcn_perm(hi, lo, 0x07050301u);  // the upper byte of each bf16
    return ((uint32_t)w & 0x7F7F7F7Fu) | (signs & 0x80808080u);
}

// The same of four binary32 numbers.
__device__ __forceinline__ uint32_t e4m3_codes(float a, float b, float c, float d, float inv) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(a * inv), e4m3_clamp(b * inv), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(c * inv), e4m3_clamp(d * inv), w, true);
    const uint32_t lo = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x0C0C0703u);
    const uint32_t hi = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, d), __builtin_bit_cast(uint32_t, c), 0x07030C0Cu);
    return ((uint32_t)w & 0x7F7F7F7Fu) | ((lo | hi) & 0x80808080u);
}

// 16 bytes per lane from global memory straight into LDS: lane i of the wave writes lds_base + 16*i
// (lds_base is wave-uniform and travels in M0).  Written as inline asm so that the compiler's wait-count pass
// does not see an LDS write it would have to order every later LDS read behind (it would drain the memory
// counter before the first operand read of each tile); completion is awaited explicitly with s_waitcnt vmcnt.
// The global address is a wave-uniform base (scalar register pair) plus a 32-bit byte offset per lane.
__device__ __forceinline__ void lds_direct_load16_at(const void* gbase, uint32_t lane_off, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(lane_off), "s"(gbase), "s"(lds_addr)
                 : "memory", "m0");
}

// Zeroes the bf16 elements e of a granule of 8 tokens whose position first + e is >= kv_total (never written).
__device__ __forceinline__ u32x4 zero_unwritten(u32x4 v, int first, int kv_total) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (first + e >= kv_total) v[e >> 1] &= (e & 1) ? 0x0000FFFFu : 0xFFFF0000u;
    return v;
}

// Which of the 64 keys from new token `off` on (off > -64; below 0 are cached ones) a row may see, a bit each: all cached ones, and of
// the new ones those in its mask, or, where `words` is NULL, those up to `own`.  Keys from `valid` on are not there.
__device__ __forceinline__ uint64_t visible_keys(const uint64_t* words, int n_words, int own, int off, int valid) {
    uint64_t seen;
    if (words) {
        if (off < 0) {
            seen = (words[0] << -off) | ((1ull << -off) - 1);
        } else {
            const int w = off >> 6, b = off & 63;
            seen = w < n_words ? words[w] >> b : 0;
            if (b > 0 && w + 1 < n_words) seen |= words[w + 1] << (64 - b);
        }
    } else {
        const int count = own - off + 1;
        seen = count >= 64 ? ~0ull : count <= 0 ? 0 : (1ull << count) - 1;
    }
    if (valid < 64) seen &= valid <= 0 ? 0 : (1ull << valid) - 1;
    return seen;
}

__device__ __forceinline__ bool not_finite_bf16(uint32_t bits) { return (bits & 0x7F80u) == 0x7F80u; }

}  // namespace ppd
