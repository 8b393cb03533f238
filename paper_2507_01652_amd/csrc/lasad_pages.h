// What the kernels of the paged 8-bit cache share: its layout, and which rows, tokens and pages a workgroup has.
//
// A page holds the keys (and one the values) of 64 positions of a row, of every key head: k [64][d], v [d][64], e4m3 codes.  In a page of v,
// position 16 b + 4 g + i lies at 16 g + 4 b + i: with products of 16 x 16 x 32 a lane's share of the second product's operand is then 16
// bytes in a row, and so are its channels of a key in the first one; neither passes through LDS.
#pragma once

#include "lasad_window.h"

namespace lasad {

constexpr int kPage = 64;                                // positions of a page
constexpr float kCodeTop = 448.f;                        // the largest e4m3 value
constexpr float kLeastScale = 0x1p-126f;                 // the least scale of a page that is not all zeros

struct Pages {
    uint8_t *k, *v;                                      // [n_pages, heads, 64, d], [n_pages, heads, d, 64]
    float *k_scale, *v_scale;                            // [n_pages, heads]
    int n_pages, heads;
    const int32_t *table;                                // row b's page of its positions 64 j .. : table[b * table_stride + j]
    int table_pages;
    int64_t table_stride;
};

// Packed new tokens of B rows: row b has tokens starts[b] .. starts[b + 1] - 1 of `tokens` (NULL: token b alone), the first of
// them at position pos_rows[b] (NULL: pos).
struct PageRows {
    int B, tokens;
    const int32_t *starts;
    int pos;
    const int32_t *pos_rows;
    int last_pos;                                        // positions 0 .. last_pos - 1 exist
};

struct AppendArgs {
    const void *q, *k, *v;                               // q NULL: keys and values alone
    void *q_out;
    lasad_layout_t lq, lk, lv, lo;                       // (stride_b is not read)
    int io_dtype, out_dtype, Hq, d;
    const float *w[2];                                   // norm weights of queries and keys
    int shared, norm;
    float eps;
    int rope, pairing, grid_w;
    double log2_base;
    Pages pages;
    PageRows rows;
};
hipError_t launch_append_pages(const AppendArgs &a, hipStream_t s);
int64_t append_pages_groups(const AppendArgs &a);         // of a launch, in workgroups of 256 threads

struct AttendArgs {
    const void *q;
    void *o;
    lasad_layout_t lq, lo;
    int io_dtype, out_dtype, Hq, d;
    int window, sinks;
    float scale;
    Pages pages;
    PageRows rows;
    float *parts;                                        // workspace of splits: [tokens * Hq][splits][d + 4]: sums, maximum, sum of P
    int splits;
};
hipError_t launch_attend_pages(const AttendArgs &a, hipStream_t s);
hipError_t launch_join_pages(const AttendArgs &a, hipStream_t s);          // of the splits
int64_t attend_pages_groups(const AttendArgs &a);        // of a launch, splits included
int attend_pages_splits(int64_t B, int64_t tokens, int Hq, int Hk, bool one_each, int64_t seen);
size_t attend_pages_bytes(int64_t tokens, int Hq, int d, int splits);

// One token of every row: a.k, a.v are appended, a.q are the queries; t.o, window, sinks, scale and splits of the attention.
hipError_t launch_step_pages(const AppendArgs &a, const AttendArgs &t, hipStream_t s);
int64_t step_pages_groups(const AttendArgs &t);
int step_pages_splits(int64_t B, int Hq, int Hk, int64_t seen);

// A row as a workgroup sees it.
struct PageRow {
    int b, first, n, pos, unit;                          // first token, number of tokens, position of the first; piece of work of the row
};

// The row and the unit of work of workgroup `slot`, where a row of n tokens has at most n * num / den + extra units (rounded down): its first
// unit is slot starts * num / den + b * extra, so that the launch needs no row's length.  false: there is none, or the row is inactive.
// Wavefronts look for it by themselves, 64 rows at a time.  What lies in `starts` leads to no token outside 0 .. tokens - 1.
__device__ inline bool find_row(const PageRows &r, const Pages &pages, int slot, int num, int den, int extra, PageRow &row)
{
    if (r.starts) {
        const int lane = threadIdx.x & 63;
        int lo = 0, span = r.B;
        const auto clamped = [&](int s) { return min(max(s, 0), r.tokens); };
        const auto first_slot = [&](int b, int s) { return (int64_t)s * num / den + (int64_t)b * extra; };
        while (span > 64) {
            const int step = (span + 63) / 64, b = lo + lane * step;
            const bool before = lane * step < span && first_slot(b, clamped(r.starts[b])) <= slot;
            const int found = max(1, __popcll(__ballot(before))) - 1;
            lo += found * step;
            span = min(step, span - found * step);
        }
        // the rest at once, with what is needed of the one that it will be
        const int start = clamped(r.starts[min(lo + lane, r.B)]), pos = r.pos_rows ? r.pos_rows[min(lo + lane, r.B - 1)] : r.pos;
        const int found = max(1, __popcll(__ballot(lane < span && first_slot(lo + lane, start) <= slot))) - 1;
        row.b = __builtin_amdgcn_readfirstlane(lo + found);
        row.first = __builtin_amdgcn_readlane(start, found);
        row.n = max(found < 63 ? __builtin_amdgcn_readlane(start, found + 1) : clamped(r.starts[row.b + 1]), row.first) - row.first;
        row.pos = __builtin_amdgcn_readlane(pos, found);
        const int64_t unit = slot - first_slot(row.b, row.first);
        if (unit < 0) return false;
        row.unit = (int)unit;
    } else {
        const int each = (num + den - 1) / den;
        row.b = slot / each;
        row.unit = slot - row.b * each;
        row.first = row.b;
        row.n = 1;
        row.pos = r.pos_rows ? r.pos_rows[row.b] : r.pos;
    }
    row.b = __builtin_amdgcn_readfirstlane(row.b);       // (the same in all lanes; so that the compiler knows)
    row.first = __builtin_amdgcn_readfirstlane(row.first);
    row.n = __builtin_amdgcn_readfirstlane(row.n);
    row.pos = __builtin_amdgcn_readfirstlane(row.pos);
    row.unit = __builtin_amdgcn_readfirstlane(row.unit);
    return row.n > 0 && row.pos >= 0 && (int64_t)row.pos + row.n <= min((int64_t)r.last_pos, (int64_t)pages.table_pages * kPage);
}
inline int64_t row_slots(const PageRows &r, int num, int den, int extra)
{
    return r.starts ? (int64_t)r.tokens * num / den + (int64_t)r.B * extra : (int64_t)r.B * ((num + den - 1) / den);
}

// Page number j of row b, -1 if it is none of the pool's.
__device__ inline int page_of(const Pages &p, int b, int j)
{
    const int page = p.table[b * p.table_stride + j];
    return page >= 0 && page < p.n_pages ? page : -1;
}

}  // namespace lasad
