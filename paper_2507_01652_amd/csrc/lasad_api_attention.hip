// C ABI of the softmax layers' operators: argument validation on the host, then dispatch to the kernel launchers.
// Nothing here allocates device memory or synchronises.
#include <math.h>

#include "lasad_attention.h"

using lasad::fail;
using lasad::hip_fail;

namespace {

bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

// What all calls have: sizes and types.  (B * n_tokens rows of a launch are counted in 32 bits.)
int check_sizes(int B, int n_q_heads, int n_k_heads, int d, int64_t n_tokens, int io_dtype, int out_dtype)
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
int check_layout(const char *name, const lasad_layout_t *l, int dtype, bool output, int B, int64_t n, int heads, int d)
{
    if (!l) return fail(LASAD_ERR_INVALID_ARG, "the layout of %s is NULL", name);
    const int vec = dtype == LASAD_BF16 ? 8 : 4;
    if (l->stride_b < 0 || l->stride_n < 0 || l->stride_h < 0 || l->stride_b % vec || l->stride_n % vec || l->stride_h % vec)
        return fail(LASAD_ERR_INVALID_ARG, "the strides of %s must be non-negative multiples of %d elements", name, vec);
    if (output && n > 0 && ((B > 1 && l->stride_b < d) || (n > 1 && l->stride_n < d) || (heads > 1 && l->stride_h < d)))
        return fail(LASAD_ERR_INVALID_ARG, "rows of %s overlap", name);
    return LASAD_OK;
}

int check_pointer(const char *name, const void *p, size_t alignment)
{
    if (!p) return fail(LASAD_ERR_INVALID_ARG, "%s is NULL", name);
    if (!aligned(p, alignment)) return fail(LASAD_ERR_INVALID_ARG, "%s must be %d-byte aligned", name, (int)alignment);
    return LASAD_OK;
}

bool same_layout(const lasad_layout_t &a, const lasad_layout_t &b)
{
    return a.stride_b == b.stride_b && a.stride_n == b.stride_n && a.stride_h == b.stride_h;
}

int check_qk_options(int grid_h, int grid_w, const float *q_weight, const float *k_weight, float norm_eps, int rope, int pairing,
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

int qk_forward(const void *q, const void *k, void *q_out, void *k_out,
               const lasad_layout_t *q_layout, const lasad_layout_t *k_layout,
               const lasad_layout_t *q_out_layout, const lasad_layout_t *k_out_layout,
               int io_dtype, int out_dtype, int B, int n_q_heads, int n_k_heads, int d,
               int grid_h, int grid_w, int start_pos, const int32_t *pos_rows, int n_tokens,
               const float *q_weight, const float *k_weight, int shared_weight, float norm_eps,
               int rope, int pairing, float rope_base, void *hip_stream, const char *name)
{
    lasad::QkArgs a = {};
    if (int rc = check_sizes(B, n_q_heads, n_k_heads, d, n_tokens, io_dtype, out_dtype)) return rc;
    if (int rc = check_qk_options(grid_h, grid_w, q_weight, k_weight, norm_eps, rope, pairing, rope_base, a)) return rc;
    if (!pos_rows && (start_pos < 0 || (int64_t)start_pos + n_tokens > a.last_pos))
        return fail(LASAD_ERR_INVALID_ARG, "%d tokens from position %d leave the %d x %d grid", n_tokens, start_pos, grid_h, grid_w);
    if (!aligned(pos_rows, 4)) return fail(LASAD_ERR_INVALID_ARG, "pos_rows must be 4-byte aligned");
    if (int rc = check_layout("q", q_layout, io_dtype, false, B, n_tokens, n_q_heads, d)) return rc;
    if (int rc = check_layout("k", k_layout, io_dtype, false, B, n_tokens, n_k_heads, d)) return rc;
    if (int rc = check_layout("q_out", q_out_layout, out_dtype, true, B, n_tokens, n_q_heads, d)) return rc;
    if (int rc = check_layout("k_out", k_out_layout, out_dtype, true, B, n_tokens, n_k_heads, d)) return rc;
    if (n_tokens == 0) return LASAD_OK;
    if (int rc = check_pointer("q", q, 16)) return rc;
    if (int rc = check_pointer("k", k, 16)) return rc;
    if (int rc = check_pointer("q_out", q_out, 16)) return rc;
    if (int rc = check_pointer("k_out", k_out, 16)) return rc;
    if (q_out == k_out || q_out == k || k_out == q) return fail(LASAD_ERR_INVALID_ARG, "buffers alias");
    if ((q_out == q && (io_dtype != out_dtype || !same_layout(*q_layout, *q_out_layout))) ||
        (k_out == k && (io_dtype != out_dtype || !same_layout(*k_layout, *k_out_layout))))
        return fail(LASAD_ERR_INVALID_ARG, "in place needs the same type and strides");
    a.x[0] = q; a.x[1] = k; a.y[0] = q_out; a.y[1] = k_out;
    a.in[0] = *q_layout; a.in[1] = *k_layout; a.out[0] = *q_out_layout; a.out[1] = *k_out_layout;
    a.heads[0] = n_q_heads; a.heads[1] = n_k_heads;
    a.io_dtype = io_dtype; a.out_dtype = out_dtype; a.B = B; a.n = n_tokens; a.d = d;
    a.start_pos = start_pos; a.pos_rows = pos_rows; a.shared = shared_weight != 0;
    const hipError_t e = lasad::launch_qk_forward(a, (hipStream_t)hip_stream);
    if (e != hipSuccess) return hip_fail(name, e);
    return LASAD_OK;
}

}  // namespace

extern "C" {

int lasad_forward_qk(const void *q, const void *k, void *q_out, void *k_out,
                     const lasad_layout_t *q_layout, const lasad_layout_t *k_layout,
                     const lasad_layout_t *q_out_layout, const lasad_layout_t *k_out_layout,
                     int io_dtype, int out_dtype, int B, int n_q_heads, int n_k_heads, int d,
                     int grid_h, int grid_w, int start_pos, int n_tokens,
                     const float *q_weight, const float *k_weight, int shared_weight, float norm_eps,
                     int rope, int pairing, float rope_base, void *hip_stream)
{
    return qk_forward(q, k, q_out, k_out, q_layout, k_layout, q_out_layout, k_out_layout, io_dtype, out_dtype, B, n_q_heads, n_k_heads, d,
                      grid_h, grid_w, start_pos, nullptr, n_tokens, q_weight, k_weight, shared_weight, norm_eps, rope, pairing, rope_base,
                      hip_stream, "lasad_forward_qk launch");
}

int lasad_decode_step_qk(const void *q, const void *k, void *q_out, void *k_out,
                         int io_dtype, int out_dtype, int B, int n_q_heads, int n_k_heads, int d,
                         int grid_h, int grid_w, int pos, const int32_t *pos_rows,
                         const float *q_weight, const float *k_weight, int shared_weight, float norm_eps,
                         int rope, int pairing, float rope_base, void *hip_stream)
{
    const lasad_layout_t lq = {(int64_t)n_q_heads * d, (int64_t)n_q_heads * d, d}, lk = {(int64_t)n_k_heads * d, (int64_t)n_k_heads * d, d};
    return qk_forward(q, k, q_out, k_out, &lq, &lk, &lq, &lk, io_dtype, out_dtype, B, n_q_heads, n_k_heads, d,
                      grid_h, grid_w, pos, pos_rows, 1, q_weight, k_weight, shared_weight, norm_eps, rope, pairing, rope_base,
                      hip_stream, "lasad_decode_step_qk launch");
}

size_t lasad_backward_qk_workspace_bytes(int B, int n_q_heads, int n_k_heads, int n_tokens, int d, int shared_weight)
{
    if (B < 1 || n_q_heads < 1 || n_k_heads < 1 || n_tokens < 1 || d < 1) return 0;
    return lasad::qk_partial_bytes((int64_t)B * n_tokens, n_q_heads + n_k_heads, d, shared_weight != 0);
}

int lasad_backward_qk(const void *q, const void *k, const void *d_q, const void *d_k, void *dq, void *dk,
                      float *dq_weight, float *dk_weight,
                      const lasad_layout_t *q_layout, const lasad_layout_t *k_layout,
                      const lasad_layout_t *d_q_layout, const lasad_layout_t *d_k_layout,
                      const lasad_layout_t *dq_layout, const lasad_layout_t *dk_layout,
                      int io_dtype, int grad_dtype, int B, int n_q_heads, int n_k_heads, int d,
                      int grid_h, int grid_w, int start_pos, int n_tokens,
                      const float *q_weight, const float *k_weight, int shared_weight, float norm_eps,
                      int rope, int pairing, float rope_base,
                      void *workspace, size_t workspace_bytes, void *hip_stream)
{
    lasad::QkArgs a = {};
    if (int rc = check_sizes(B, n_q_heads, n_k_heads, d, n_tokens, io_dtype, grad_dtype)) return rc;
    if (int rc = check_qk_options(grid_h, grid_w, q_weight, k_weight, norm_eps, rope, pairing, rope_base, a)) return rc;
    if (start_pos < 0 || (int64_t)start_pos + n_tokens > a.last_pos)
        return fail(LASAD_ERR_INVALID_ARG, "%d tokens from position %d leave the %d x %d grid", n_tokens, start_pos, grid_h, grid_w);
    if (norm_eps < 0.f && (dq_weight || dk_weight)) return fail(LASAD_ERR_INVALID_ARG, "norm_eps < 0 (no norm) with a weight gradient");
    if (!aligned(dq_weight, 4) || !aligned(dk_weight, 4)) return fail(LASAD_ERR_INVALID_ARG, "the weight gradients must be 4-byte aligned");
    if (int rc = check_layout("q", q_layout, io_dtype, false, B, n_tokens, n_q_heads, d)) return rc;
    if (int rc = check_layout("k", k_layout, io_dtype, false, B, n_tokens, n_k_heads, d)) return rc;
    if (int rc = check_layout("d_q", d_q_layout, io_dtype, false, B, n_tokens, n_q_heads, d)) return rc;
    if (int rc = check_layout("d_k", d_k_layout, io_dtype, false, B, n_tokens, n_k_heads, d)) return rc;
    if (int rc = check_layout("dq", dq_layout, grad_dtype, true, B, n_tokens, n_q_heads, d)) return rc;
    if (int rc = check_layout("dk", dk_layout, grad_dtype, true, B, n_tokens, n_k_heads, d)) return rc;
    if (n_tokens > 0) {
        if (int rc = check_pointer("q", q, 16)) return rc;
        if (int rc = check_pointer("k", k, 16)) return rc;
        if (int rc = check_pointer("d_q", d_q, 16)) return rc;
        if (int rc = check_pointer("d_k", d_k, 16)) return rc;
        if (int rc = check_pointer("dq", dq, 16)) return rc;
        if (int rc = check_pointer("dk", dk, 16)) return rc;
        if (dq == dk || dq == q || dq == k || dk == q || dk == k || dq == d_q || dq == d_k || dk == d_q || dk == d_k)
            return fail(LASAD_ERR_INVALID_ARG, "buffers alias");
        if (dq_weight || dk_weight) {
            const size_t need = lasad_backward_qk_workspace_bytes(B, n_q_heads, n_k_heads, n_tokens, d, shared_weight);
            if (!workspace || workspace_bytes < need)
                return fail(LASAD_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace ? workspace_bytes : (size_t)0, need);
            if (!aligned(workspace, 16)) return fail(LASAD_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
        }
    }
    a.x[0] = q; a.x[1] = k; a.dy[0] = d_q; a.dy[1] = d_k; a.y[0] = dq; a.y[1] = dk;
    a.in[0] = *q_layout; a.in[1] = *k_layout; a.dl[0] = *d_q_layout; a.dl[1] = *d_k_layout; a.out[0] = *dq_layout; a.out[1] = *dk_layout;
    a.heads[0] = n_q_heads; a.heads[1] = n_k_heads;
    a.io_dtype = io_dtype; a.out_dtype = grad_dtype; a.B = B; a.n = n_tokens; a.d = d;
    a.start_pos = start_pos; a.shared = shared_weight != 0;
    a.dw[0] = dq_weight; a.dw[1] = dk_weight; a.partial = (float *)workspace;
    const hipError_t e = lasad::launch_qk_backward(a, (hipStream_t)hip_stream);
    if (e != hipSuccess) return hip_fail("lasad_backward_qk launch", e);
    return LASAD_OK;
}

}  // extern "C"
