// Attention of packed queries over the paged 8-bit cache:
//     o = sum over the seen keys j of softmax_j(scale q . k_j) v_j,   seen: j <= p, p - j < window or j < sinks,
// with k_j and v_j = code times the page's scale.
//
// A wavefront takes a page at a time for tiles of 16 columns; the columns of a row are its (token, query head of the key head's group) pairs in
// order, so that heads that share keys read them once.  Scores are formed transposed, 16 positions x 16 columns: a column's numbers are then four
// registers of each of four lanes, and as they lie there they are the second operand of the product with v, whose first operand is 16 bytes of a
// page a lane (lasad_pages.h).  Nothing passes through LDS but the join of wavefronts that share columns.  Codes become bf16 exactly; a page's
// scale of k is applied to the scores in fp32, that of v as a power of two with the conversion and the rest in P's exponent.  fp32 queries and P
// are three bf16 parts each; of bf16 queries P is one, rounded to 2^-9, which is what o's own rounding costs: more parts would
// double the second product.  Where o is fp32, and that reason is none, P is two (2^-17).  Its sums are those of the rounded P.
//
// 4 x 24 heads over 8, 4096 tokens, window 1024, d = 64: 138 us a pass in a stream (148 alone), 91 GFLOP, 660 TFLOP/s where a product of 8192^3 reaches 1199.
// The matrix cores are busy for 0.29 of the time, the vector units for 0.55 (exponentials, conversions of codes and of P, 164 instructions a page
// of 64 keys and 32 columns), and three wavefronts a SIMD do not always have one of each.  On the way: sums of P by additions and both
// scales by products 343; with the search for a maximum in every page 197; with the accumulators moved twice a page by it 167; with keys that
// waited for the values behind them 154; 48 columns a wavefront 151 then, 64 176, 16 200.  Rows of 128 to 256 tokens (12 heads, window 128): 8.5 us, a
// launch and four to six pages one behind the other.
#include "lasad_pages_tile.h"

namespace lasad {

namespace {

// Workgroup: WAVES wavefronts, CW of them beside each other over CW * NT * 16 columns of a row's key head, WAVES / CW over the pages.
// (Wavefronts a SIMD: at d = 32 the wide shape's 128 registers are four's, without the bound it takes two more.  With P in two parts and two
// tiles at d = 64 three spill 31 registers: 4 x 24 heads over 8, 4096 tokens, 173 us; two without spills 195, one tile 208.)
template <typename T, typename O, int D, int NQ, int NP, int NT, int CW, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, D == 128 ? (sizeof(T) == 4 ? 1 : 2) : D == 32 && NP * NT < 4 ? 4 : 3)
attend_pages_kernel(AttendArgs a)
{
    constexpr int KW = WAVES / CW, COLS = CW * NT * 16, NC = D / 16, NF = D / 32;
    const int heads = a.pages.heads, G = a.Hq / heads;
    const int split = blockIdx.y, hk = blockIdx.x % heads;
    PageRow row;
    if (!find_row(a.rows, a.pages, blockIdx.x / heads, G, COLS, 1, row)) return;
    const int columns = row.n * G;                       // (at most tokens * Hq, which fits 31 bits)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, quad = lane >> 4, col = lane & 15;
    const int group0 = row.unit * COLS;
    if (group0 >= columns) return;
    const int cw = wave % CW, kw = wave / CW, c0 = group0 + cw * NT * 16;

    Columns<D, NQ, NP, NT> x;
    x.p0 = __builtin_amdgcn_readfirstlane(row.pos + c0 / G);
    x.p1 = __builtin_amdgcn_readfirstlane(c0 < columns ? row.pos + (min(c0 + NT * 16, columns) - 1) / G : -1);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int c = c0 + 16 * n + col, token = c / G, h = hk * G + c - token * G;
        const bool on = c < columns;
        x.p[n] = on ? row.pos + token : -1;
        const T *qp = (const T *)a.q + (row.first + (int64_t)(on ? token : 0)) * a.lq.stride_n + (on ? h : 0) * a.lq.stride_h;
#pragma unroll
        for (int f = 0; f < NF; ++f) query_parts<T, NQ>(qp + page_channel<D>(f, quad), x.q[n][f]);
        x.m[n] = -INFINITY;
        x.l[n] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) x.acc[n][c] = f32x4v{0.f, 0.f, 0.f, 0.f};
    }
    const float scale2 = a.scale * kLog2e;
    const PageList list(x.p0, x.p1, a.window, a.sinks);
    const int step = a.splits * KW;
    const int i = split * KW + kw;
    Walk walk;
    walk.fill(a.pages, list, row.b, i, step);
    const int page = walk.next(a.pages, list, row.b, i, step);
    PagePart<D> t;
    const auto load_k = [&](int page) { t.load_k(a.pages, max(page, 0), hk, lane); };
    const auto load_v = [&](int page) { t.load_v(a.pages, max(page, 0), hk, lane); };
    load_k(page);
    __builtin_amdgcn_sched_barrier(0);
    load_v(page);
    x.template run<false>(t, list, i, step, page, scale2, a.window, a.sinks, lane, [&](int i) { return walk.next(a.pages, list, row.b, i, step); },
                          load_k, load_v, [] {});

    if constexpr (KW == 1) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (x.p[n] < 0) continue;
            const int c = c0 + 16 * n + col, token = c / G, h = hk * G + c - token * G;
            const float inv = x.l[n] == 0.f ? 0.f : 1.f / x.l[n];
            O *op = (O *)a.o + (int64_t)(row.first + token) * a.lo.stride_n + h * a.lo.stride_h + 4 * quad;
#pragma unroll
            for (int b = 0; b < NC; ++b)
                store4(op + 16 * b, x.acc[n][b][0] * inv, x.acc[n][b][1] * inv, x.acc[n][b][2] * inv, x.acc[n][b][3] * inv);
        }
    } else {
        static_assert(CW == 1 && NT == 1, "wavefronts over the pages have one tile of columns");
        __shared__ __align__(16) float red[KW][16][D + 4];
        join_waves<O, D, KW, 1>(red, x.acc[0], x.m[0], x.l[0], kw, lane, min(16, columns - c0), a.splits, split, [&](int cc, int ch) {
            const int c = c0 + cc, token = c / G, h = hk * G + c - token * G;
            const int64_t at = (int64_t)(row.first + token) * a.Hq + h;
            return Result<O>{a.parts + at * a.splits * (D + 4), (O *)a.o + (int64_t)(row.first + token) * a.lo.stride_n + h * a.lo.stride_h + ch};
        });
    }
}

// The splits of a query head joined by a workgroup: a thread has four channels of every EACHth split.
template <typename O, int D>
__global__ void __launch_bounds__(256)
join_pages_kernel(AttendArgs a)
{
    constexpr int EACH = 256 / (D / 4), LD = D + 4;
    __shared__ __align__(16) float red[EACH][LD];
    const int64_t at = blockIdx.x;
    const int token = (int)(at / a.Hq), h = (int)(at - (int64_t)token * a.Hq);
    const int one = threadIdx.x / (D / 4), ch = threadIdx.x % (D / 4) * 4;
    const float *p = a.parts + at * a.splits * LD;
    float top = -INFINITY, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = one; i < a.splits; i += EACH) {
        const float m = p[i * LD + D], l = p[i * LD + D + 1];
        const float4 r = *(const float4 *)(p + i * LD + ch);
        const float most = fmaxf(top, m), use = most == -INFINITY ? 0.f : most;
        const float f = __builtin_amdgcn_exp2f(top - use), g = __builtin_amdgcn_exp2f(m - use);
        top = most;
        sum = fmaf(l, g, sum * f);
        o = make_float4(fmaf(r.x, g, o.x * f), fmaf(r.y, g, o.y * f), fmaf(r.z, g, o.z * f), fmaf(r.w, g, o.w * f));
    }
    *(float4 *)(red[one] + ch) = o;
    if (ch == 0) { red[one][D] = top; red[one][D + 1] = sum; }
    // (a token that belongs to no row, or to an inactive one, has no parts: what was read is not used)
    PageRow row;
    if (a.rows.starts) {
        int lo = 0, hi = a.rows.B;                       // the last row that starts at the token or before it
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (a.rows.starts[mid] <= token) lo = mid; else hi = mid;
        }
        row.b = lo;
        row.first = min(max(a.rows.starts[lo], 0), a.rows.tokens);
        row.n = min(max(a.rows.starts[lo + 1], row.first), a.rows.tokens) - row.first;
    } else {
        row.b = row.first = token;
        row.n = 1;
    }
    row.pos = a.rows.pos_rows ? a.rows.pos_rows[row.b] : a.rows.pos;
    __syncthreads();
    if (token < row.first || token >= row.first + row.n || row.pos < 0 ||
        (int64_t)row.pos + row.n > min((int64_t)a.rows.last_pos, (int64_t)a.pages.table_pages * kPage) || threadIdx.x >= D / 4) return;
    top = -INFINITY;
#pragma unroll
    for (int i = 0; i < EACH; ++i) top = fmaxf(top, red[i][D]);
    const float use = top == -INFINITY ? 0.f : top;
    sum = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const float f = __builtin_amdgcn_exp2f(red[i][D] - use);
        const float4 r = *(const float4 *)(red[i] + ch);
        sum = fmaf(red[i][D + 1], f, sum);
        o.x = fmaf(r.x, f, o.x); o.y = fmaf(r.y, f, o.y); o.z = fmaf(r.z, f, o.z); o.w = fmaf(r.w, f, o.w);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    store4((O *)a.o + token * a.lo.stride_n + h * a.lo.stride_h + ch, o.x * inv, o.y * inv, o.z * inv, o.w * inv);
}

// Workgroups of 128 columns from which on they are taken instead of 64 (bf16, d up to 64; a page's codes are then turned into bf16 once for 32 columns,
// not 16, by three wavefronts a SIMD instead of four).  12 heads, window 512: 288 workgroups 11.8 us, with 64 columns 9.2; 480 17.6 and 18.8; 1632
// 51.9 and 63.9.
constexpr int64_t kFull = 384;

// Up to 32 columns a row on average: a workgroup's wavefronts share 16 of them over the pages, and splits share them over workgroups.
// With more, each wavefront has columns of its own, and writes their results itself.  (8 rows of 12 heads, us with wavefronts over the pages and
// with columns of their own: 32 tokens on 200 keys 5.4 and 6.6, on 1000 10.5 and 15.9, on 4000 22 and 44; 48 tokens 5.5 and 6.7, 10.5 and 16.0,
// 22 and 44; 64 tokens 6.7 and 7.9, 10.6 and 16.2, 22 and 46.  So the border could lie higher; where it should has not been measured.)
bool few_columns(int64_t B, int64_t tokens, int G) { return tokens * G <= 32 * B; }

// How a launch divides its columns.
struct Shape {
    int nt, cw;
    int columns() const { return 16 * nt * cw; }
};
Shape choose(const AttendArgs &a)
{
    const int G = a.Hq / a.pages.heads;
    if (few_columns(a.rows.B, a.rows.tokens, G)) return {1, 1};
    const Shape wide = {2, 4};
    const bool full = row_slots(a.rows, G, wide.columns(), 1) * a.pages.heads >= kFull;
    return {a.io_dtype == LASAD_BF16 && a.d <= 64 && full ? 2 : 1, 4};
}
int64_t groups_of(const AttendArgs &a, const Shape &s) { return row_slots(a.rows, a.Hq / a.pages.heads, s.columns(), 1) * a.pages.heads; }

template <typename O, int D>
void launch_join(const AttendArgs &a, hipStream_t s)
{
    join_pages_kernel<O, D><<<dim3((unsigned)((int64_t)a.rows.tokens * a.Hq)), dim3(256), 0, s>>>(a);
}

template <typename T, typename O, int D, int NQ, int NP>
hipError_t launch(const AttendArgs &a, hipStream_t s)
{
    const Shape shape = choose(a);
    const dim3 grid((unsigned)groups_of(a, shape), (unsigned)a.splits);
    constexpr int WIDE = sizeof(T) == 2 && D <= 64 ? 2 : 1;
    if (shape.cw == 1) attend_pages_kernel<T, O, D, NQ, NP, 1, 1, 4><<<grid, dim3(256), 0, s>>>(a);
    else if (shape.nt == 1) attend_pages_kernel<T, O, D, NQ, NP, 1, 4, 4><<<grid, dim3(256), 0, s>>>(a);
    else attend_pages_kernel<T, O, D, NQ, NP, WIDE, 4, 4><<<grid, dim3(256), 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) {
        launch_join<O, D>(a, s);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int64_t attend_pages_groups(const AttendArgs &a) { return groups_of(a, choose(a)) * a.splits; }

// Splits of a call whose rows see up to `seen` keys, by the step's rule (lasad_pages_step.hip, where it was measured; here: two rows of 24 and fewer
// tokens, 16 heads, 16448 keys for 512 workgroups 17.4 us, 256 18.4, 1024 18.9).
int attend_pages_splits(int64_t B, int64_t tokens, int Hq, int Hk, bool one_each, int64_t seen)
{
    const int G = Hq / Hk;
    if (!few_columns(B, tokens, G)) return 1;
    const int64_t groups = (one_each ? B * ((G + 15) / 16) : tokens * G / 16 + B) * Hk;
    int64_t n = 512 / groups;
    if (seen < 1536 || n < 4) return 1;
    if (n > seen / 512) n = seen / 512;
    return (int)(n > 64 ? 64 : n < 1 ? 1 : n);
}

size_t attend_pages_bytes(int64_t tokens, int Hq, int d, int splits)
{
    return splits > 1 ? (size_t)tokens * Hq * splits * (d + 4) * sizeof(float) : 0;
}

hipError_t launch_join_pages(const AttendArgs &a, hipStream_t s)
{
#define LASAD_JP(O) (a.d == 32 ? launch_join<O, 32>(a, s) : a.d == 64 ? launch_join<O, 64>(a, s) : launch_join<O, 128>(a, s))
    if (a.out_dtype == LASAD_BF16) LASAD_JP(uint16_t); else LASAD_JP(float);
#undef LASAD_JP
    return hipGetLastError();
}

hipError_t launch_attend_pages(const AttendArgs &a, hipStream_t s)
{
#define LASAD_AT(T, O, NQ, NP) (a.d == 32 ? launch<T, O, 32, NQ, NP>(a, s) : a.d == 64 ? launch<T, O, 64, NQ, NP>(a, s) : launch<T, O, 128, NQ, NP>(a, s))
    if (a.io_dtype == LASAD_F32) return LASAD_AT(float, float, 3, 3);
    return a.out_dtype == LASAD_BF16 ? LASAD_AT(uint16_t, uint16_t, 1, 1) : LASAD_AT(uint16_t, float, 1, 2);
#undef LASAD_AT
}

}  // namespace lasad
