// Numbers to codes of a page, and the page's scale (lasad_pages_append.hip has the rules).
#pragma once

#include "lasad_pages.h"

namespace lasad {

__device__ inline float finite_size(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }

// y / s rounded once more than exactly at most where it is halfway: a product with 1 / s and one correction.
struct Divide {
    float s, inv;
    __device__ inline explicit Divide(float scale) : s(scale), inv(scale > 0.f ? 1.f / scale : 0.f) {}
    __device__ inline float operator()(float y) const
    {
        const float t = y * inv;
        return fmaf(fmaf(-t, s, y), inv, t);
    }
};

__device__ inline uint32_t code2(float x, float y, uint32_t old, bool high)
{
    return high ? __builtin_amdgcn_cvt_pk_fp8_f32(x, y, old, true) : __builtin_amdgcn_cvt_pk_fp8_f32(x, y, old, false);
}
__device__ inline uint32_t code4(float x, float y, float z, float w) { return code2(z, w, code2(x, y, 0, false), true); }

// Byte e of a word of codes divided (times `by`, a power of two), where `mask` has 0xff.
__device__ inline uint32_t shrink(uint32_t w, float by, uint32_t mask)
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    const uint32_t r = code4(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
    return (r & mask) | (w & ~mask);
}

// The bytes of a word before the first `n`, 0xff each.
__device__ inline uint32_t first_bytes(int n) { return n <= 0 ? 0u : n >= 4 ? 0xffffffffu : (1u << 8 * n) - 1u; }

// The scale of a page whose `earlier` first positions were there before, with scale `old`; their codes are then to be multiplied by `by`.
__device__ inline float page_scale(float most, int earlier, float old, float &by)
{
    by = 1.f;
    if (earlier == 0 || !(old > 0.f)) return most > 0.f ? fmaxf(most / kCodeTop, kLeastScale) : 0.f;
    while (old * kCodeTop < most) {
        old *= 2.f;
        by *= 0.5f;
    }
    return old;
}

// The codes of the `earlier` first positions of a page made smaller, by a wavefront; V: a page of values.
template <int D, bool V>
__device__ inline void shrink_page(uint8_t *codes, int earlier, float by, int lane)
{
    uint4 w[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) w[i] = ((const uint4 *)codes)[i * 64 + lane];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        const int at = i * 64 + lane, g = at % 4;                              // v: positions 16 b + 4 g ..
        const uint32_t whole = at / (D / 16) < earlier ? 0xffffffffu : 0u;      // k: a position's channels
        w[i].x = shrink(w[i].x, by, V ? first_bytes(earlier - 4 * g) : whole);
        w[i].y = shrink(w[i].y, by, V ? first_bytes(earlier - 4 * g - 16) : whole);
        w[i].z = shrink(w[i].z, by, V ? first_bytes(earlier - 4 * g - 32) : whole);
        w[i].w = shrink(w[i].w, by, V ? first_bytes(earlier - 4 * g - 48) : whole);
        ((uint4 *)codes)[at] = w[i];
    }
    __threadfence_block();                               // (one of the call's codes may go there yet, from another lane)
}

}  // namespace lasad
