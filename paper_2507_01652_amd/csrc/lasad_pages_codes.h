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

// The scale of a page whose `earlier` first positions were there before, with scale `old`; where it grows, their codes are made smaller.  By
// a wavefront; V: a page of values.
template <int D, bool V>
__device__ inline float page_scale(float most, int earlier, float old, float *scale, uint8_t *codes, int lane, bool &grown)
{
    float s;
    grown = false;
    if (earlier == 0) old = 0.f;
    if (!(old > 0.f)) {
        s = most > 0.f ? fmaxf(most / kCodeTop, kLeastScale) : 0.f;
    } else {
        float by = 1.f;
        s = old;
        while (s * kCodeTop < most) {
            s *= 2.f;
            by *= 0.5f;
        }
        grown = by < 1.f;
        if (grown) {
            uint32_t *words = (uint32_t *)codes;
            for (int w = lane; w < kPage * D / 4; w += 64) {
                uint32_t mask;
                if (V) {
                    const int t = 16 * (w % 4) + 4 * (w / 4 % 4);          // the word's first position
                    mask = t + 4 <= earlier ? 0xffffffffu : t >= earlier ? 0u : (1u << 8 * (earlier - t)) - 1u;
                } else {
                    mask = w / (D / 4) < earlier ? 0xffffffffu : 0u;
                }
                if (mask) words[w] = shrink(words[w], by, mask);
            }
            __threadfence_block();                       // (a word of v may get one of the call's codes yet, from another lane)
        }
    }
    if (lane == 0) *scale = s;
    return s;
}

}  // namespace lasad
