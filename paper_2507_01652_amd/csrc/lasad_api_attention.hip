// C ABI of the softmax layers' operators: argument validation on the host, then dispatch to the kernel launchers.
// Nothing here allocates device memory or synchronises.
#include <math.h>

#include "lasad_attention.h"

using lasad::fail;
using lasad::hip_fail;

namespace {

bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

// Calls with more workgroups than a launch may have are refused.
int too_many() { return fail(LASAD_ERR_UNSUPPORTED, "B * heads * tokens overflows the launch grid"); }
bool fits(int64_t heads, int64_t units) { return heads <= lasad::kMostGroups && heads * (units < 1 ? 1 : units) <= lasad::kMostGroups; }
int check_groups(int64_t groups) { return groups > lasad::kMostGroups ? too_many() : LASAD_OK; }

// Whether check_sizes lets these through.  A size query answers 0 where the call would be refused: it is asked first.
bool known_sizes(int B, int n_q_heads, int n_k_heads, int d, int64_t n_tokens)
{
    return B >= 1 && n_q_heads >= 1 && n_k_heads >= 1 && n_q_heads <= 65535 && n_k_heads <= 65535 && (d == 32 || d == 64 || d == 128) &&
           n_tokens >= 0 && B * n_tokens <= 0x7fffffff;
}

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
    if (int rc = check_groups(lasad::qk_forward_groups((int64_t)B * n_tokens, d))) return rc;
    const hipError_t e = lasad::launch_qk_forward(a, (hipStream_t)hip_stream);
    if (e != hipSuccess) return hip_fail(name, e);
    return LASAD_OK;
}

// No kernel has more than 128 queries or keys a workgroup; what is launched in fact is counted once it is known.
bool fit(int B, int n_q_heads, int n_k_heads, int n_tokens, int n_keys)
{
    return fits((int64_t)B * n_q_heads, (n_tokens + 127) / 128) && fits((int64_t)B * n_k_heads, (n_keys + 127) / 128);
}

int check_window(int n_q_heads, int n_k_heads, int window, int sinks, float scale)
{
    if (n_q_heads % n_k_heads) return fail(LASAD_ERR_INVALID_ARG, "%d query heads cannot share %d key heads evenly", n_q_heads, n_k_heads);
    if (window < 1 || sinks < 0) return fail(LASAD_ERR_INVALID_ARG, "window = %d, sinks = %d", window, sinks);
    if (!(scale > 0.f && scale < INFINITY)) return fail(LASAD_ERR_INVALID_ARG, "scale must be positive and finite");
    if (scale > 0x1p127f) return fail(LASAD_ERR_UNSUPPORTED, "scale beyond 2^127");       // (times log2 e it would pass fp32)
    return LASAD_OK;
}

// Sizes of a forward or backward: what a launch counts fits 32 bits.
int check_window_sizes(int B, int n_q_heads, int n_k_heads, int d, int start_pos, int n_tokens, int n_keys, int window, int sinks,
                       float scale, int io_dtype, int out_dtype)
{
    if (int rc = check_sizes(B, n_q_heads, n_k_heads, d, n_tokens, io_dtype, out_dtype)) return rc;
    if (int rc = check_window(n_q_heads, n_k_heads, window, sinks, scale)) return rc;
    if (n_keys < 0 || start_pos < 0) return fail(LASAD_ERR_INVALID_ARG, "n_keys = %d, start_pos = %d", n_keys, start_pos);
    if ((int64_t)start_pos + n_tokens > 1 << 30 || n_keys > 1 << 30) return fail(LASAD_ERR_UNSUPPORTED, "positions beyond 2^30");
    if (!fit(B, n_q_heads, n_k_heads, n_tokens, n_keys)) return too_many();
    return LASAD_OK;
}

lasad::WindowArgs window_args(const void *q, const void *k, const void *v, int io_dtype, int out_dtype, int B, int n_q_heads, int n_k_heads,
                              int d, int start_pos, int n_tokens, int n_keys, int window, int sinks, const int32_t *kv_lens, float scale)
{
    lasad::WindowArgs a = {};
    a.q = q; a.k = k; a.v = v;
    a.io_dtype = io_dtype; a.out_dtype = out_dtype;
    a.B = B; a.Hq = n_q_heads; a.Hk = n_k_heads; a.d = d;
    a.start_pos = start_pos; a.n = n_tokens; a.m = n_keys;
    a.window = window; a.sinks = sinks; a.lens = kv_lens; a.scale = scale;
    return a;
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
    if (!known_sizes(B, n_q_heads, n_k_heads, d, n_tokens) || n_tokens == 0) return 0;
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
    if (int rc = check_groups(lasad::qk_backward_groups((int64_t)B * n_tokens))) return rc;
    const hipError_t e = lasad::launch_qk_backward(a, (hipStream_t)hip_stream);
    if (e != hipSuccess) return hip_fail("lasad_backward_qk launch", e);
    return LASAD_OK;
}

int lasad_forward_window(const void *q, const void *k, const void *v, void *o, float *lse,
                         const lasad_layout_t *q_layout, const lasad_layout_t *k_layout,
                         const lasad_layout_t *v_layout, const lasad_layout_t *o_layout,
                         int io_dtype, int out_dtype, int B, int n_q_heads, int n_k_heads, int d,
                         int start_pos, int n_tokens, int n_keys, int window, int sinks,
                         const int32_t *kv_lens, float scale, void *hip_stream)
{
    if (int rc = check_window_sizes(B, n_q_heads, n_k_heads, d, start_pos, n_tokens, n_keys, window, sinks, scale, io_dtype, out_dtype)) return rc;
    if (int rc = check_layout("q", q_layout, io_dtype, false, B, n_tokens, n_q_heads, d)) return rc;
    if (int rc = check_layout("k", k_layout, io_dtype, false, B, n_keys, n_k_heads, d)) return rc;
    if (int rc = check_layout("v", v_layout, io_dtype, false, B, n_keys, n_k_heads, d)) return rc;
    if (int rc = check_layout("o", o_layout, out_dtype, true, B, n_tokens, n_q_heads, d)) return rc;
    if (!aligned(kv_lens, 4) || !aligned(lse, 4)) return fail(LASAD_ERR_INVALID_ARG, "kv_lens and lse must be 4-byte aligned");
    if (n_tokens == 0) return LASAD_OK;
    if (int rc = check_pointer("q", q, 16)) return rc;
    if (int rc = check_pointer("o", o, 16)) return rc;
    if (n_keys > 0) {
        if (int rc = check_pointer("k", k, 16)) return rc;
        if (int rc = check_pointer("v", v, 16)) return rc;
    }
    if (o == q || o == k || o == v || (void *)lse == o) return fail(LASAD_ERR_INVALID_ARG, "o aliases another buffer");
    lasad::WindowArgs a = window_args(q, k, v, io_dtype, out_dtype, B, n_q_heads, n_k_heads, d, start_pos, n_tokens, n_keys, window, sinks,
                                      kv_lens, scale);
    a.o = o; a.lse = lse;
    a.lq = *q_layout; a.lk = *k_layout; a.lv = *v_layout; a.lo = *o_layout;
    if (int rc = check_groups(lasad::window_forward_groups(a))) return rc;
    const hipError_t e = lasad::launch_window_forward(a, (hipStream_t)hip_stream);
    if (e != hipSuccess) return hip_fail("lasad_forward_window launch", e);
    return LASAD_OK;
}

size_t lasad_backward_window_workspace_bytes(int B, int n_q_heads, int n_k_heads, int d, int n_tokens, int n_keys,
                                             int window, int sinks)
{
    if (!known_sizes(B, n_q_heads, n_k_heads, d, n_tokens) || n_q_heads % n_k_heads || n_tokens < 1 || n_tokens > 1 << 30 || n_keys < 0 ||
        n_keys > 1 << 30 || window < 1 || sinks < 0 || !fit(B, n_q_heads, n_k_heads, n_tokens, n_keys)) return 0;
    return lasad::window_backward_bytes(B, n_q_heads, n_k_heads, d, n_tokens, n_keys, window, sinks);
}

int lasad_backward_window(const void *q, const void *k, const void *v, const void *o, const float *lse, const void *d_o,
                          void *dq, void *dk, void *dv,
                          const lasad_layout_t *q_layout, const lasad_layout_t *k_layout, const lasad_layout_t *v_layout,
                          const lasad_layout_t *o_layout, const lasad_layout_t *d_o_layout,
                          const lasad_layout_t *dq_layout, const lasad_layout_t *dk_layout, const lasad_layout_t *dv_layout,
                          int io_dtype, int grad_dtype, int B, int n_q_heads, int n_k_heads, int d,
                          int start_pos, int n_tokens, int n_keys, int window, int sinks,
                          const int32_t *kv_lens, float scale,
                          void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (int rc = check_window_sizes(B, n_q_heads, n_k_heads, d, start_pos, n_tokens, n_keys, window, sinks, scale, io_dtype, grad_dtype)) return rc;
    // (the bf16 kernels' scores start from -lse / scale: the logarithm of 2^30 keys over 2^-120 is 2^124.4)
    if (io_dtype == LASAD_BF16 && scale < 0x1p-120f) return fail(LASAD_ERR_UNSUPPORTED, "scale below 2^-120 with bf16 inputs");
    const struct { const char *name; const lasad_layout_t *l; bool out, key; } layouts[] = {
        {"q", q_layout, false, false}, {"k", k_layout, false, true}, {"v", v_layout, false, true}, {"o", o_layout, false, false},
        {"d_o", d_o_layout, false, false}, {"dq", dq_layout, true, false}, {"dk", dk_layout, true, true}, {"dv", dv_layout, true, true}};
    for (const auto &x : layouts)
        if (int rc = check_layout(x.name, x.l, x.out ? grad_dtype : io_dtype, x.out, B, x.key ? n_keys : n_tokens, x.key ? n_k_heads : n_q_heads, d))
            return rc;
    if (!aligned(kv_lens, 4) || !aligned(lse, 4)) return fail(LASAD_ERR_INVALID_ARG, "kv_lens and lse must be 4-byte aligned");
    if (n_tokens > 0) {
        if (int rc = check_pointer("q", q, 16)) return rc;
        if (int rc = check_pointer("o", o, 16)) return rc;
        if (int rc = check_pointer("d_o", d_o, 16)) return rc;
        if (int rc = check_pointer("dq", dq, 16)) return rc;
        if (int rc = check_pointer("lse", lse, 4)) return rc;
    }
    if (n_keys > 0) {
        if (int rc = check_pointer("k", k, 16)) return rc;
        if (int rc = check_pointer("v", v, 16)) return rc;
        if (int rc = check_pointer("dk", dk, 16)) return rc;
        if (int rc = check_pointer("dv", dv, 16)) return rc;
    }
    const void *in[] = {q, k, v, o, d_o, lse}, *out[] = {dq, dk, dv};
    for (int i = 0; i < 3; ++i) {
        for (const void *p : in)
            if (out[i] && out[i] == p) return fail(LASAD_ERR_INVALID_ARG, "a gradient aliases an input");
        if (out[i] && out[i] == out[(i + 1) % 3]) return fail(LASAD_ERR_INVALID_ARG, "gradients alias each other");
    }
    const size_t need = lasad_backward_window_workspace_bytes(B, n_q_heads, n_k_heads, d, n_tokens, n_keys, window, sinks);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return fail(LASAD_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace ? workspace_bytes : (size_t)0, need);
    if (!aligned(workspace, 16)) return fail(LASAD_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    lasad::WindowArgs a = window_args(q, k, v, io_dtype, grad_dtype, B, n_q_heads, n_k_heads, d, start_pos, n_tokens, n_keys, window, sinks,
                                      kv_lens, scale);
    a.o = const_cast<void *>(o); a.lse = const_cast<float *>(lse); a.d_o = d_o;
    a.dq = dq; a.dk = dk; a.dv = dv;
    a.lq = *q_layout; a.lk = *k_layout; a.lv = *v_layout; a.lo = *o_layout; a.ldo = *d_o_layout;
    a.ldq = *dq_layout; a.ldk = *dk_layout; a.ldv = *dv_layout;
    if (int rc = check_groups(lasad::window_backward_groups(a))) return rc;
    const hipError_t e = lasad::launch_window_backward(a, workspace, (hipStream_t)hip_stream);
    if (e != hipSuccess) return hip_fail("lasad_backward_window launch", e);
    return LASAD_OK;
}

size_t lasad_decode_step_window_workspace_bytes(int B, int n_q_heads, int n_k_heads, int d, int cache_tokens, int window,
                                                int sinks)
{
    if (!known_sizes(B, n_q_heads, n_k_heads, d, 1) || n_q_heads % n_k_heads || window < 1 || sinks < 0 || cache_tokens <= sinks ||
        !fits((int64_t)B * n_k_heads, 1)) return 0;
    const int64_t seen = (int64_t)window + sinks < cache_tokens ? (int64_t)window + sinks : cache_tokens;
    return lasad::window_step_bytes(B, n_q_heads, d, lasad::window_step_splits(B, n_k_heads, seen));
}

int lasad_decode_step_window(const void *q, const void *k, const void *v, void *o, void *k_cache, void *v_cache,
                             int cache_tokens, int io_dtype, int out_dtype, int B, int n_q_heads, int n_k_heads, int d,
                             int pos, const int32_t *pos_rows, int window, int sinks, float scale,
                             void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (int rc = check_sizes(B, n_q_heads, n_k_heads, d, 1, io_dtype, out_dtype)) return rc;
    if (int rc = check_window(n_q_heads, n_k_heads, window, sinks, scale)) return rc;
    if (!fits((int64_t)B * n_k_heads, 1) || (int64_t)B * n_q_heads > 0x7fffffff) return too_many();
    if (cache_tokens <= sinks) return fail(LASAD_ERR_INVALID_ARG, "a cache of %d rows has no room beside %d sinks", cache_tokens, sinks);
    if (!pos_rows && (pos < 0 || (pos >= cache_tokens && cache_tokens - sinks < window)))
        return fail(LASAD_ERR_INVALID_ARG, "pos %d does not fit a cache of %d rows (window %d, sinks %d)", pos, cache_tokens, window, sinks);
    if (!aligned(pos_rows, 4)) return fail(LASAD_ERR_INVALID_ARG, "pos_rows must be 4-byte aligned");
    const struct { const char *name; const void *p; } pointers[] = {{"q", q}, {"k", k}, {"v", v}, {"o", o}, {"k_cache", k_cache}, {"v_cache", v_cache}};
    for (const auto &x : pointers)
        if (int rc = check_pointer(x.name, x.p, 16)) return rc;
    if (o == q || o == k || o == v || k_cache == v_cache || o == k_cache || o == v_cache || k == k_cache || v == v_cache)
        return fail(LASAD_ERR_INVALID_ARG, "buffers alias");
    const size_t need = lasad_decode_step_window_workspace_bytes(B, n_q_heads, n_k_heads, d, cache_tokens, window, sinks);
    if (workspace && workspace_bytes < need) return fail(LASAD_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (!aligned(workspace, 16)) return fail(LASAD_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    lasad::WindowStepArgs a = {};
    a.q = q; a.k = k; a.v = v; a.o = o; a.k_cache = k_cache; a.v_cache = v_cache;
    a.io_dtype = io_dtype; a.out_dtype = out_dtype;
    a.B = B; a.Hq = n_q_heads; a.Hk = n_k_heads; a.d = d; a.cap = cache_tokens;
    a.pos = pos; a.pos_rows = pos_rows; a.window = window; a.sinks = sinks; a.scale = scale;
    int64_t seen = (int64_t)window + sinks < cache_tokens ? (int64_t)window + sinks : cache_tokens;
    if (!pos_rows && (int64_t)pos + 1 < seen) seen = (int64_t)pos + 1;
    a.parts = (float *)workspace;
    a.splits = workspace && need ? lasad::window_step_splits(B, n_k_heads, seen) : 1;
    const hipError_t e = lasad::launch_window_step(a, (hipStream_t)hip_stream);
    if (e != hipSuccess) return hip_fail("lasad_decode_step_window launch", e);
    return LASAD_OK;
}

}  // extern "C"
