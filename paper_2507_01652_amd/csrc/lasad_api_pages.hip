// C ABI of the paged 8-bit cache: argument validation on the host, then dispatch to the kernel launchers.  Nothing here allocates device
// memory or synchronises.
#include "lasad_checks.h"
#include "lasad_pages.h"

using namespace lasad::checks;
using lasad::fail;
using lasad::hip_fail;

namespace {

int check_pages(const lasad_pages_t *p, int n_k_heads, int d, lasad::Pages &pages)
{
    if (!p) return fail(LASAD_ERR_INVALID_ARG, "pages is NULL");
    if (p->n_pages < 1) return fail(LASAD_ERR_INVALID_ARG, "n_pages = %d", p->n_pages);
    if (p->table_pages < 1 || p->table_pages > 1 << 24) return fail(LASAD_ERR_INVALID_ARG, "table_pages = %d", p->table_pages);
    if (p->table_stride < 0) return fail(LASAD_ERR_INVALID_ARG, "table_stride < 0");
    if (int rc = check_pointer("k_pages", p->k_pages, 16)) return rc;
    if (int rc = check_pointer("v_pages", p->v_pages, 16)) return rc;
    if (int rc = check_pointer("k_scales", p->k_scales, 4)) return rc;
    if (int rc = check_pointer("v_scales", p->v_scales, 4)) return rc;
    if (int rc = check_pointer("table", p->table, 4)) return rc;
    if (p->k_pages == p->v_pages || p->k_scales == p->v_scales) return fail(LASAD_ERR_INVALID_ARG, "the pages of k and v alias");
    pages = {p->k_pages, p->v_pages, p->k_scales, p->v_scales, p->n_pages, n_k_heads, p->table, p->table_pages, p->table_stride};
    return LASAD_OK;
}

// Sizes of packed tokens: what a launch counts fits 32 bits.
int check_rows(int B, int n_q_heads, int n_k_heads, int d, int n_tokens, const int32_t *row_starts, int pos, const int32_t *pos_rows, int last_pos,
               int table_pages, int io_dtype, int out_dtype, lasad::PageRows &rows)
{
    if (B < 1) return fail(LASAD_ERR_INVALID_ARG, "B = %d", B);
    if (int rc = check_sizes(1, n_q_heads, n_k_heads, d, n_tokens, io_dtype, out_dtype)) return rc;
    if (B > 1 << 24 || (int64_t)n_tokens * n_q_heads > 1 << 30) return too_many();
    if (!row_starts && n_tokens != B) return fail(LASAD_ERR_INVALID_ARG, "%d tokens of %d rows without row_starts", n_tokens, B);
    if (!aligned(row_starts, 4) || !aligned(pos_rows, 4)) return fail(LASAD_ERR_INVALID_ARG, "row_starts and pos_rows must be 4-byte aligned");
    if (!pos_rows && (pos < 0 || pos >= last_pos || pos >= (int64_t)table_pages * lasad::kPage))
        return fail(LASAD_ERR_INVALID_ARG, "pos %d is off the grid or behind the table's %d pages", pos, table_pages);
    rows = {B, n_tokens, row_starts, pos, pos_rows, last_pos};
    return LASAD_OK;
}

bool known_rows(int B, int n_q_heads, int n_k_heads, int d, int n_tokens, int table_pages, int window, int sinks)
{
    return B >= 1 && known_sizes(1, n_q_heads, n_k_heads, d, n_tokens) && n_q_heads % n_k_heads == 0 && B <= 1 << 24 && (int64_t)n_tokens * n_q_heads <= 1 << 30 &&
           table_pages >= 1 && table_pages <= 1 << 24 && window >= 1 && sinks >= 0;
}

// Keys that a query sees at most.
int64_t seen_keys(int table_pages, int window, int sinks)
{
    const int64_t held = (int64_t)table_pages * lasad::kPage, seen = (int64_t)window + sinks;
    return seen < held ? seen : held;
}

int check_workspace(void *workspace, size_t bytes, size_t need)
{
    if (workspace && bytes < need) return fail(LASAD_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", bytes, need);
    if (!aligned(workspace, 16)) return fail(LASAD_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    return LASAD_OK;
}

// The arguments of an append, checked (n_tokens = 0: of the sizes).
int append_args(const void *q, const void *k, const void *v, void *q_out,
                const lasad_layout_t *q_layout, const lasad_layout_t *k_layout, const lasad_layout_t *v_layout,
                const lasad_layout_t *q_out_layout, const lasad_pages_t *pages,
                int io_dtype, int out_dtype, int B, int n_q_heads, int n_k_heads, int d, int grid_h, int grid_w,
                int n_tokens, const int32_t *row_starts, int pos, const int32_t *pos_rows,
                const float *q_weight, const float *k_weight, int shared_weight, float norm_eps,
                int rope, int pairing, float rope_base, lasad::AppendArgs &a)
{
    lasad::QkArgs o = {};
    if (int rc = check_qk_options(grid_h, grid_w, q_weight, k_weight, norm_eps, rope, pairing, rope_base, o)) return rc;
    if (int rc = check_pages(pages, n_k_heads, d, a.pages)) return rc;
    if (int rc = check_rows(B, q ? n_q_heads : 1, n_k_heads, d, n_tokens, row_starts, pos, pos_rows, o.last_pos, pages->table_pages, io_dtype, out_dtype, a.rows)) return rc;
    if (q) {
        if (int rc = check_layout("q", q_layout, io_dtype, false, 1, n_tokens, n_q_heads, d)) return rc;
        if (int rc = check_layout("q_out", q_out_layout, out_dtype, true, 1, n_tokens, n_q_heads, d)) return rc;
    } else if (q_out || q_weight) {
        return fail(LASAD_ERR_INVALID_ARG, "q_out or q_weight without q");
    }
    if (int rc = check_layout("k", k_layout, io_dtype, false, 1, n_tokens, n_k_heads, d)) return rc;
    if (int rc = check_layout("v", v_layout, io_dtype, false, 1, n_tokens, n_k_heads, d)) return rc;
    if (n_tokens == 0) return LASAD_OK;
    if (int rc = check_pointer("k", k, 16)) return rc;
    if (int rc = check_pointer("v", v, 16)) return rc;
    if (q) {
        if (int rc = check_pointer("q", q, 16)) return rc;
        if (int rc = check_pointer("q_out", q_out, 16)) return rc;
        if (q_out == k || q_out == v) return fail(LASAD_ERR_INVALID_ARG, "buffers alias");
        if (q_out == q && (io_dtype != out_dtype || q_layout->stride_n != q_out_layout->stride_n || q_layout->stride_h != q_out_layout->stride_h))
            return fail(LASAD_ERR_INVALID_ARG, "in place needs the same type and strides");
        a.lq = *q_layout; a.lo = *q_out_layout;
    }
    a.q = q; a.k = k; a.v = v; a.q_out = q_out;
    a.lk = *k_layout; a.lv = *v_layout;
    a.io_dtype = io_dtype; a.out_dtype = out_dtype; a.Hq = n_q_heads; a.d = d;
    a.w[0] = q_weight; a.w[1] = k_weight; a.shared = shared_weight != 0; a.norm = o.norm; a.eps = o.eps;
    a.rope = rope; a.pairing = pairing; a.grid_w = grid_w; a.log2_base = o.log2_base;
    return LASAD_OK;
}

}  // namespace

extern "C" {

int lasad_append_pages(const void *q, const void *k, const void *v, void *q_out,
                       const lasad_layout_t *q_layout, const lasad_layout_t *k_layout, const lasad_layout_t *v_layout,
                       const lasad_layout_t *q_out_layout, const lasad_pages_t *pages,
                       int io_dtype, int out_dtype, int B, int n_q_heads, int n_k_heads, int d, int grid_h, int grid_w,
                       int n_tokens, const int32_t *row_starts, int pos, const int32_t *pos_rows,
                       const float *q_weight, const float *k_weight, int shared_weight, float norm_eps,
                       int rope, int pairing, float rope_base, void *hip_stream)
{
    lasad::AppendArgs a = {};
    if (int rc = append_args(q, k, v, q_out, q_layout, k_layout, v_layout, q_out_layout, pages, io_dtype, out_dtype, B, n_q_heads, n_k_heads, d, grid_h, grid_w,
                             n_tokens, row_starts, pos, pos_rows, q_weight, k_weight, shared_weight, norm_eps, rope, pairing, rope_base, a)) return rc;
    if (n_tokens == 0) return LASAD_OK;
    if (int rc = check_groups(lasad::append_pages_groups(a))) return rc;
    const hipError_t e = lasad::launch_append_pages(a, (hipStream_t)hip_stream);
    if (e != hipSuccess) return hip_fail("lasad_append_pages launch", e);
    return LASAD_OK;
}

size_t lasad_forward_pages_workspace_bytes(int B, int n_q_heads, int n_k_heads, int d, int n_tokens, int one_each, int table_pages,
                                           int window, int sinks)
{
    if (!known_rows(B, n_q_heads, n_k_heads, d, n_tokens, table_pages, window, sinks) || (one_each && n_tokens != B)) return 0;
    return lasad::attend_pages_bytes(n_tokens, n_q_heads, d, lasad::attend_pages_splits(B, n_tokens, n_q_heads, n_k_heads, one_each, seen_keys(table_pages, window, sinks)));
}

int lasad_forward_pages(const void *q, void *o, const lasad_layout_t *q_layout, const lasad_layout_t *o_layout, const lasad_pages_t *pages,
                        int io_dtype, int out_dtype, int B, int n_q_heads, int n_k_heads, int d,
                        int n_tokens, const int32_t *row_starts, int pos, const int32_t *pos_rows, int window, int sinks, float scale,
                        void *workspace, size_t workspace_bytes, void *hip_stream)
{
    lasad::AttendArgs a = {};
    if (int rc = check_pages(pages, n_k_heads, d, a.pages)) return rc;
    if (int rc = check_rows(B, n_q_heads, n_k_heads, d, n_tokens, row_starts, pos, pos_rows, 0x7fffffff, pages->table_pages, io_dtype, out_dtype, a.rows)) return rc;
    if (int rc = check_window(n_q_heads, n_k_heads, window, sinks, scale)) return rc;
    if (int rc = check_layout("q", q_layout, io_dtype, false, 1, n_tokens, n_q_heads, d)) return rc;
    if (int rc = check_layout("o", o_layout, out_dtype, true, 1, n_tokens, n_q_heads, d)) return rc;
    const size_t need = lasad_forward_pages_workspace_bytes(B, n_q_heads, n_k_heads, d, n_tokens, !row_starts, pages->table_pages, window, sinks);
    if (int rc = check_workspace(workspace, workspace_bytes, need)) return rc;
    if (n_tokens == 0) return LASAD_OK;
    if (int rc = check_pointer("q", q, 16)) return rc;
    if (int rc = check_pointer("o", o, 16)) return rc;
    if (o == q) return fail(LASAD_ERR_INVALID_ARG, "o aliases q");
    a.q = q; a.o = o; a.lq = *q_layout; a.lo = *o_layout;
    a.io_dtype = io_dtype; a.out_dtype = out_dtype; a.Hq = n_q_heads; a.d = d;
    a.window = window; a.sinks = sinks; a.scale = scale;
    a.parts = (float *)workspace;
    a.splits = workspace && need ? lasad::attend_pages_splits(B, n_tokens, n_q_heads, n_k_heads, !row_starts, seen_keys(pages->table_pages, window, sinks)) : 1;
    if (int rc = check_groups(lasad::attend_pages_groups(a))) return rc;
    const hipError_t e = lasad::launch_attend_pages(a, (hipStream_t)hip_stream);
    if (e != hipSuccess) return hip_fail("lasad_forward_pages launch", e);
    return LASAD_OK;
}

size_t lasad_decode_step_pages_workspace_bytes(int B, int n_q_heads, int n_k_heads, int d, int table_pages, int window, int sinks)
{
    if (!known_rows(B, n_q_heads, n_k_heads, d, B, table_pages, window, sinks)) return 0;
    return lasad::attend_pages_bytes(B, n_q_heads, d, lasad::step_pages_splits(B, n_q_heads, n_k_heads, seen_keys(table_pages, window, sinks)));
}

int lasad_decode_step_pages(const void *q, const void *k, const void *v, void *o, const lasad_pages_t *pages,
                            int io_dtype, int out_dtype, int B, int n_q_heads, int n_k_heads, int d, int grid_h, int grid_w,
                            int pos, const int32_t *pos_rows,
                            const float *q_weight, const float *k_weight, int shared_weight, float norm_eps,
                            int rope, int pairing, float rope_base, int window, int sinks, float scale,
                            void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const lasad_layout_t lq = {0, (int64_t)n_q_heads * d, d}, lk = {0, (int64_t)n_k_heads * d, d};
    if (!q || !o) return fail(LASAD_ERR_INVALID_ARG, "q or o is NULL");
    if (o == q || o == k || o == v) return fail(LASAD_ERR_INVALID_ARG, "buffers alias");
    lasad::AppendArgs p = {};
    if (int rc = append_args(q, k, v, o, &lq, &lk, &lk, &lq, pages, io_dtype, out_dtype, B, n_q_heads, n_k_heads, d, grid_h, grid_w, B, nullptr, pos,
                             pos_rows, q_weight, k_weight, shared_weight, norm_eps, rope, pairing, rope_base, p)) return rc;
    if (int rc = check_window(n_q_heads, n_k_heads, window, sinks, scale)) return rc;
    const size_t need = lasad_decode_step_pages_workspace_bytes(B, n_q_heads, n_k_heads, d, pages->table_pages, window, sinks);
    if (int rc = check_workspace(workspace, workspace_bytes, need)) return rc;
    lasad::AttendArgs a = {};
    a.pages = p.pages; a.rows = p.rows;
    a.o = o; a.lo = lq;
    a.io_dtype = io_dtype; a.out_dtype = out_dtype; a.Hq = n_q_heads; a.d = d;
    a.window = window; a.sinks = sinks; a.scale = scale;
    a.parts = (float *)workspace;
    a.splits = workspace && need ? lasad::step_pages_splits(B, n_q_heads, n_k_heads, seen_keys(pages->table_pages, window, sinks)) : 1;
    if (int rc = check_groups(lasad::step_pages_groups(a))) return rc;
    const hipError_t e = lasad::launch_step_pages(p, a, (hipStream_t)hip_stream);
    if (e != hipSuccess) return hip_fail("lasad_decode_step_pages launch", e);
    return LASAD_OK;
}

}  // extern "C"
