// Checks of the softmax layers' calls: sizes, types, strides, pointers and options, on the host before anything is launched.
#pragma once

#include <math.h>

#include "lasad_attention.h"

namespace lasad {
namespace checks {

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

// Calls with more workgroups than a launch may have are refused.
inline int too_many() { return fail(LASAD_ERR_UNSUPPORTED, "B * heads * tokens overflows the launch grid"); }
inline bool fits(int64_t heads, int64_t units) { return heads <= lasad::kMostGroups && heads * (units < 1 ? 1 : units) <= lasad::kMostGroups; }
inline int check_groups(int64_t groups) { return groups > lasad::kMostGroups ? too_many() : LASAD_OK; }

// Whether check_sizes lets these through.  A size query answers 0 where the call would be refused: it is asked first.
inline bool known_sizes(int B, int n_q_heads, int n_k_heads, int d, int64_t n_tokens)
{
    return B >= 1 && n_q_heads >= 1 && n_k_heads >= 1 && n_q_heads <= 65535 && n_k_heads <= 65535 && (d == 32 || d == 64 || d == 128) &&
           n_tokens >= 0 && B * n_tokens <= 0x7fffffff;
}

// What all calls have: sizes and types.  (B * n_tokens rows of a launch are counted in 32 bits.)
inline int check_sizes(int B, int n_q_heads, int n_k_heads, int d, int64_t n_tokens, int io_dtype, int out_dtype)
{
    if (B < 1 || n_q_heads < 1 || n_k_heads < 1) return fail(LASAD_ERR_INVALID_ARG, "B = %d, n_q_heads = %d, n_k_heads = %d", B, n_q_heads, n_k_heads);
    if (n_q_heads > 65535 || n_k_heads > 65535) return fail(LASAD_ERR_UNSUPPORTED, "more than 65535 heads");
    if (d != 32 && d != 64 && d != 128) return fail(LASAD_ERR_UNSUPPORTED, "head dim %d (supported: 32, 64, 128)", d);
    if (n_tokens < 0) return fail(LASAD_ERR_INVALID_ARG, "n_tokens < 0");
    if (B * n_tokens > 0x7fffffff) return fail(LASAD_ERR_UNSUPPORTED, "B * n_tokens overflows the launch grid");
    if (io_dtype != LASAD_F32 && io_dtype != LASAD_BF16) return fail(LASAD_ERR_INVALID_ARG, "io_dtype %d", io_dtype);
    if (out_dtype != LASAD_F32 && out_dtype != LASAD_BF16) return fail(LASAD_ERR_INVALID_ARG, "out_dtype %d", out_dtype);
    if (io_dtype == LASAD_F32 && out_dtype == LASAD_BF16) return fail(LASAD_ERR_UNSUPPORTED, "fp32 inputs with bf16 output");
    return LASAD_OK;
}

// Strides of a tensor of `dtype`; an output's rows must not overlap.
inline int check_layout(const char *name, const lasad_layout_t *l, int dtype, bool output, int B, int64_t n, int heads, int d)
{
    if (!l) return fail(LASAD_ERR_INVALID_ARG, "the layout of %s is NULL", name);
    const int vec = dtype == LASAD_BF16 ? 8 : 4;
    if (l->stride_b < 0 || l->stride_n < 0 || l->stride_h < 0 || l->stride_b % vec || l->stride_n % vec || l->stride_h % vec)
        return fail(LASAD_ERR_INVALID_ARG, "the strides of %s must be non-negative multiples of %d elements", name, vec);
    if (output && n > 0 && ((B > 1 && l->stride_b < d) || (n > 1 && l->stride_n < d) || (heads > 1 && l->stride_h < d)))
        return fail(LASAD_ERR_INVALID_ARG, "rows of %s overlap", name);
    return LASAD_OK;
}

inline int check_pointer(const char *name, const void *p, size_t alignment)
{
    if (!p) return fail(LASAD_ERR_INVALID_ARG, "%s is NULL", name);
    if (!aligned(p, alignment)) return fail(LASAD_ERR_INVALID_ARG, "%s must be %d-byte aligned", name, (int)alignment);
    return LASAD_OK;
}

inline bool same_layout(const lasad_layout_t &a, const lasad_layout_t &b)
{
    return a.stride_b == b.stride_b && a.stride_n == b.stride_n && a.stride_h == b.stride_h;
}

inline int check_qk_options(int grid_h, int grid_w, const float *q_weight, const float *k_weight, float norm_eps, int rope, int pairing,
                     float rope_base, lasad::QkArgs &a)
{
    if (grid_h < 1 || grid_w < 1) return fail(LASAD_ERR_INVALID_ARG, "grid %d x %d: both sides must be >= 1", grid_h, grid_w);
    if ((int64_t)grid_h * grid_w > (int64_t)1 << 30) return fail(LASAD_ERR_INVALID_ARG, "grid %d x %d is too large", grid_h, grid_w);
    if (rope < 0 || rope > 2) return fail(LASAD_ERR_INVALID_ARG, "rope %d is not a lasad_rope_t", rope);
    if (pairing < 0 || pairing > 1) return fail(LASAD_ERR_INVALID_ARG, "pairing %d is not a lasad_pairing_t", pairing);
    if (rope != LASAD_ROPE_NONE && !(rope_base > 1.f && rope_base < INFINITY)) return fail(LASAD_ERR_INVALID_ARG, "rope_base must be > 1");
    if (norm_eps != norm_eps || norm_eps == INFINITY) return fail(LASAD_ERR_INVALID_ARG, "norm_eps is not a number");
    if (norm_eps < 0.f && (q_weight || k_weight)) return fail(LASAD_ERR_INVALID_ARG, "norm_eps < 0 (no norm) with a norm weight");
    if (!aligned(q_weight, 16) || !aligned(k_weight, 16)) return fail(LASAD_ERR_INVALID_ARG, "the weights must be 16-byte aligned");
    a.w[0] = q_weight; a.w[1] = k_weight;
    a.grid_w = grid_w; a.last_pos = grid_h * grid_w;
    a.rope = rope; a.pairing = pairing;
    a.log2_base = rope == LASAD_ROPE_NONE ? 0.0 : log2((double)rope_base);
    a.norm = norm_eps >= 0.f; a.eps = norm_eps;
    return LASAD_OK;
}

inline int check_window(int n_q_heads, int n_k_heads, int window, int sinks, float scale)
{
    if (n_q_heads % n_k_heads) return fail(LASAD_ERR_INVALID_ARG, "%d query heads cannot share %d key heads evenly", n_q_heads, n_k_heads);
    if (window < 1 || sinks < 0) return fail(LASAD_ERR_INVALID_ARG, "window = %d, sinks = %d", window, sinks);
    if (!(scale > 0.f && scale < INFINITY)) return fail(LASAD_ERR_INVALID_ARG, "scale must be positive and finite");
    if (scale > 0x1p127f) return fail(LASAD_ERR_UNSUPPORTED, "scale beyond 2^127");       // (times log2 e it would pass fp32)
    return LASAD_OK;
}

}  // namespace checks
}  // namespace lasad
