// Host side of the rotation by positions: its setting, argument checks and launches behind the C ABI.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>
#include <cstring>

#include "ppd_context.h"
#include "ppd_rope.h"

namespace {

constexpr long double kTwoPi = 6.283185307179586476925286766559005768L;

// A range of memory that strided rows take: [begin, end)
struct Range {
    uintptr_t begin, end;
    Range(const void* p, int64_t rows, int64_t stride, int64_t row_elems)
        : begin(reinterpret_cast<uintptr_t>(p)), end(begin + 2 * (uintptr_t)((rows - 1) * stride + row_elems)) {}
    bool meets(const Range& o) const { return begin < o.end && o.begin < end; }
};

// Rows `stride` elements apart that each hold `row_elems`: in whole 16-byte granules, inside 2^62 bytes.
bool good_stride(int64_t rows, int64_t stride, int64_t row_elems) {
    return rows <= 1 || (stride >= row_elems && stride % 8 == 0 && stride <= (int64_t(1) << 60) / rows);
}

ppd_status frequencies_impl(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_length, double low_turns, double high_turns, double* inv_freq) {
    if (!inv_freq) return fail(nullptr, PPD_ERR_NULL, "inv_freq is NULL");
    if (rotary_dim < 2 || rotary_dim % 2 != 0 || rotary_dim > 2 * ppd::kMaxPairs) return fail(nullptr, PPD_ERR_SHAPE, "rotary_dim must be even, in [2, 128]");
    if (!(base > 0) || !std::isfinite(base)) return fail(nullptr, PPD_ERR_RANGE, "base must be finite and > 0");
    if (scaling < PPD_ROPE_SCALE_NONE || scaling > PPD_ROPE_SCALE_BY_PARTS) return fail(nullptr, PPD_ERR_RANGE, "unknown scaling");
    if (scaling != PPD_ROPE_SCALE_NONE && (!(factor > 0) || !std::isfinite(factor))) return fail(nullptr, PPD_ERR_RANGE, "factor must be finite and > 0");
    if (scaling == PPD_ROPE_SCALE_BASE && rotary_dim < 4) return fail(nullptr, PPD_ERR_SHAPE, "a stretched base needs a rotary_dim of 4 or more");
    if (scaling == PPD_ROPE_SCALE_BY_PARTS && (!(original_length > 0) || !std::isfinite(original_length) || !(low_turns >= 0) || !(high_turns > low_turns) || !std::isfinite(high_turns)))
        return fail(nullptr, PPD_ERR_RANGE, "original_length must be finite and > 0, 0 <= low_turns < high_turns");
    double f[ppd::kMaxPairs];
    for (int i = 0; i < rotary_dim / 2; ++i) {
        f[i] = std::pow(base, -2.0 * i / rotary_dim);
        // (base * factor^(rotary_dim / (rotary_dim - 2)) itself may be beyond the largest number)
        if (scaling == PPD_ROPE_SCALE_BASE) f[i] *= std::pow(factor, -2.0 * i / (rotary_dim - 2));
        if (scaling == PPD_ROPE_SCALE_LINEAR) f[i] /= factor;
        if (scaling == PPD_ROPE_SCALE_BY_PARTS) {
            const double turns = original_length * f[i] / (double)kTwoPi;
            const double keep = std::fmin(1.0, std::fmax(0.0, (turns - low_turns) / (high_turns - low_turns)));
            f[i] = keep * f[i] + (1.0 - keep) * f[i] / factor;
        }
        if (!std::isfinite(f[i])) return fail(nullptr, PPD_ERR_RANGE, "a frequency is not finite");
    }
    std::memcpy(inv_freq, f, sizeof(double) * (rotary_dim / 2));
    return PPD_OK;
}

ppd_status set_rope_impl(ppd_ctx* ctx, const double* inv_freq, int32_t rotary_dim, int32_t layout, float amplitude) {
    if (!ctx) return PPD_ERR_NULL;
    if (!inv_freq) return fail(ctx, PPD_ERR_NULL, "inv_freq is NULL");
    if (rotary_dim < 2 || rotary_dim % 2 != 0 || rotary_dim > ctx->shape.head_dim) return fail(ctx, PPD_ERR_SHAPE, "rotary_dim must be even, in [2, head_dim]");
    if (layout != PPD_ROPE_HALF && layout != PPD_ROPE_INTERLEAVED) return fail(ctx, PPD_ERR_RANGE, "layout must be PPD_ROPE_HALF or PPD_ROPE_INTERLEAVED");
    if (!std::isfinite(amplitude)) return fail(ctx, PPD_ERR_RANGE, "amplitude must be finite");
    ppd::Rotation rot;
    std::memset(&rot, 0, sizeof rot);
    for (int i = 0; i < rotary_dim / 2; ++i) {
        if (!std::isfinite(inv_freq[i])) return fail(ctx, PPD_ERR_RANGE, "a frequency is not finite");
        // the fraction of a turn, in units of 2^-64; a position is an integer, so whole turns do not count
        const long double turns = (long double)inv_freq[i] / kTwoPi;
        const long double units = std::round(std::ldexp(turns - std::floor(turns), 64));
        rot.turns[i] = units < 18446744073709551616.0L ? (uint64_t)units : 0;
    }
    rot.rotary_dim = rotary_dim;
    rot.interleaved = layout == PPD_ROPE_INTERLEAVED;
    rot.amplitude = amplitude;
    ctx->rotation = rot;
    return PPD_OK;
}

ppd_status rope_impl(ppd_ctx* ctx, const void* x, int64_t x_stride, int32_t heads, const int64_t* positions, int64_t T, int32_t transpose, void* out,
                     int64_t out_stride, void* stream) {
    if (!ctx) return PPD_ERR_NULL;
    if (T < 0 || T >= (int64_t(1) << 31)) return fail(ctx, PPD_ERR_RANGE, "T out of range");
    if (heads < 1 || heads > ppd::kMaxRopeHeads) return fail(ctx, PPD_ERR_RANGE, "heads must be in [1, 4096]");
    if (ctx->rotation.rotary_dim == 0) return fail(ctx, PPD_ERR_RANGE, "no rotation is set: call ppd_set_rope first");
    if (T == 0) return PPD_OK;
    if (!x || !positions || !out) return fail(ctx, PPD_ERR_NULL, "x / positions / out is NULL");
    if (!aligned16(x) || !aligned16(out) || (reinterpret_cast<uintptr_t>(positions) & 7u))
        return fail(ctx, PPD_ERR_RANGE, "x / out must be 16-byte aligned, positions 8-byte aligned");
    const int64_t row = (int64_t)heads * ctx->shape.head_dim;
    if (!good_stride(T, x_stride, row) || !good_stride(T, out_stride, row))
        return fail(ctx, PPD_ERR_RANGE, "x_stride and out_stride must be multiples of 8, at least a row");
    if (Range(x, T, x_stride, row).meets(Range(out, T, out_stride, row)) && !(x == out && (x_stride == out_stride || T == 1)))
        return fail(ctx, PPD_ERR_RANGE, "out overlaps x: it must be x itself or lie apart from it");
    PPD_HIP(ctx, hipSetDevice(ctx->device));
    ppd::RopeParams p;
    std::memset(&p, 0, sizeof p);
    p.x = static_cast<const uint16_t*>(x);
    p.out = static_cast<uint16_t*>(out);
    p.positions = positions;
    p.T = T;
    p.x_stride = x_stride;
    p.out_stride = out_stride;
    p.heads = heads;
    p.sin_sign = transpose ? -1.f : 1.f;
    p.rot = ctx->rotation;
    const int rc = ppd::launch_rope(p, ctx->shape.head_dim, stream);
    if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "launch rope");
    if (ctx->log_calls) std::fprintf(stderr, "ppd: rope T=%lld heads=%d%s\n", (long long)T, (int)heads, transpose ? " transposed" : "");
    return PPD_OK;
}

ppd_status append_rotated_impl(ppd_ctx* ctx, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                               const int64_t* positions, void* kv_pages, const int64_t* slot_mapping, int64_t T, void* q_out, void* stream) {
    if (!ctx) return PPD_ERR_NULL;
    if (T < 0 || T >= (int64_t(1) << 31)) return fail(ctx, PPD_ERR_RANGE, "T out of range");
    if (ctx->rotation.rotary_dim == 0) return fail(ctx, PPD_ERR_RANGE, "no rotation is set: call ppd_set_rope first");
    if (T == 0) return PPD_OK;
    if (!k || !v || !positions || !kv_pages || !slot_mapping) return fail(ctx, PPD_ERR_NULL, "k / v / positions / kv_pages / slot_mapping is NULL");
    if (!q != !q_out) return fail(ctx, PPD_ERR_NULL, "one of q and q_out is NULL: give both or neither");
    if (!aligned16(q) || !aligned16(q_out) || !aligned16(k) || !aligned16(v) || !aligned16(kv_pages) || (reinterpret_cast<uintptr_t>(slot_mapping) & 7u) ||
        (reinterpret_cast<uintptr_t>(positions) & 7u))
        return fail(ctx, PPD_ERR_RANGE, "q / q_out / k / v / kv_pages must be 16-byte aligned, positions and slot_mapping 8-byte aligned");
    const int64_t q_row = (int64_t)ctx->shape.num_q_heads * ctx->shape.head_dim, kv_row = (int64_t)ctx->shape.num_kv_heads * ctx->shape.head_dim;
    if ((q && !good_stride(T, q_stride, q_row)) || !good_stride(T, k_stride, kv_row) || !good_stride(T, v_stride, kv_row))
        return fail(ctx, PPD_ERR_RANGE, "q_stride, k_stride and v_stride must be multiples of 8, at least a row");
    if (q) {
        const Range written(q_out, T, q_row, q_row);
        if (written.meets(Range(q, T, q_stride, q_row)) && !(q == q_out && (q_stride == q_row || T == 1)))
            return fail(ctx, PPD_ERR_RANGE, "q_out overlaps q: it must be q itself or lie apart from it");
        if (written.meets(Range(k, T, k_stride, kv_row)) || written.meets(Range(v, T, v_stride, kv_row)))
            return fail(ctx, PPD_ERR_RANGE, "q_out overlaps k or v");
    }
    PPD_HIP(ctx, hipSetDevice(ctx->device));
    ppd::RotatedAppendParams p;
    std::memset(&p, 0, sizeof p);
    p.q = static_cast<const uint16_t*>(q);
    p.k = static_cast<const uint16_t*>(k);
    p.v = static_cast<const uint16_t*>(v);
    p.q_out = static_cast<uint16_t*>(q_out);
    p.pool = kv_pages;
    p.positions = positions;
    p.slots = slot_mapping;
    p.err_flags = ctx->d_counters + 9;
    p.T = T;
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.num_pages = ctx->shape.num_pages;
    p.Hq = ctx->shape.num_q_heads;
    p.Hkv = ctx->shape.num_kv_heads;
    p.inv_k = 1.0f / ctx->k_scale;
    p.inv_v = 1.0f / ctx->v_scale;
    p.rot = ctx->rotation;
    const int rc = ppd::launch_rotated_append(p, ctx->shape.head_dim, ctx->fp8_pages, stream);
    if (rc != 0) return hip_fail(ctx, (hipError_t)rc, "launch kv_append_rotated");
    ppd::check_duplicate_slots(ctx, slot_mapping, T, static_cast<hipStream_t>(stream));
    if (ctx->log_calls) std::fprintf(stderr, "ppd: kv_append_rotated T=%lld%s\n", (long long)T, q ? "" : " (no queries)");
    return PPD_OK;
}

}  // namespace

extern "C" {

ppd_status ppd_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_length, double low_turns,
                                double high_turns, double* inv_freq) {
    return guarded(nullptr, [&] { return frequencies_impl(rotary_dim, base, scaling, factor, original_length, low_turns, high_turns, inv_freq); });
}

ppd_status ppd_set_rope(ppd_ctx* ctx, const double* inv_freq, int32_t rotary_dim, int32_t layout, float amplitude) {
    return guarded(ctx, [&] { return set_rope_impl(ctx, inv_freq, rotary_dim, layout, amplitude); });
}

ppd_status ppd_rope(ppd_ctx* ctx, const void* x, int64_t x_stride, int32_t heads, const int64_t* positions, int64_t T, int32_t transpose, void* out,
                    int64_t out_stride, void* stream) {
    return guarded(ctx, [&] { return rope_impl(ctx, x, x_stride, heads, positions, T, transpose, out, out_stride, stream); });
}

ppd_status ppd_kv_append_rotated(ppd_ctx* ctx, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                 const int64_t* positions, void* kv_pages, const int64_t* slot_mapping, int64_t T, void* q_out, void* stream) {
    return guarded(ctx, [&] { return append_rotated_impl(ctx, q, q_stride, k, k_stride, v, v_stride, positions, kv_pages, slot_mapping, T, q_out, stream); });
}

}  // extern "C"
