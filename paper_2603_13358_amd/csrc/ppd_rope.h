// Internal declarations of the rotation by positions: on its own, and on the way into the page pool.
#pragma once
#include <stdint.h>

#include "ppd_internal.h"

namespace ppd {

constexpr int kMaxRopeHeads = 4096;  // heads of a tensor that ppd_rope rotates

struct RopeParams {
    const uint16_t* x;
    uint16_t* out;
    const int64_t* positions;
    int64_t T, x_stride, out_stride;  // rows, elements between them
    int32_t heads;
    float sin_sign;                   // -1: the transpose
    Rotation rot;
};

struct RotatedAppendParams {
    const uint16_t *q, *k, *v;        // q may be NULL
    uint16_t* q_out;
    void* pool;
    const int64_t *positions, *slots;
    uint32_t* err_flags;
    int64_t T, q_stride, k_stride, v_stride, num_pages;
    int32_t Hq, Hkv;
    float inv_k, inv_v;               // FP8 pages: one over the scales
    Rotation rot;
};

// Launchers; stream is a hipStream_t, the result a hipError_t.
int launch_rope(const RopeParams& p, int head_dim, void* stream);
int launch_rotated_append(const RotatedAppendParams& p, int head_dim, bool fp8_pages, void* stream);

}  // namespace ppd
