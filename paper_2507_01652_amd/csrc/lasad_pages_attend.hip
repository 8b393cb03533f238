// Attention of packed queries over the paged 8-bit cache:
//     o = sum over the seen keys j of softmax_j(scale q . k_j) v_j,   seen: j <= p, p - j < window or j < sinks,
// with k_j and v_j = code times the page's scale.
//
// A wavefront takes a page at a time for tiles of 16 columns; the columns of a row are its (token, query head of the key head's group) pairs in
// order, so that heads that share keys read them once.  Scores are formed transposed, 16 positions x 16 columns: a column's numbers are then four
// registers of each of four lanes, and as they lie there they are the second operand of the product with v, whose first operand is 16 bytes of a
// page a lane (lasad_pages.h).  Nothing passes through LDS but the join of wavefronts that share columns.  Codes become bf16 exactly, scales are
// applied to the scores and to P in fp32.  fp32 queries and P are three bf16 parts each.
#include "lasad_pages.h"

namespace lasad {

namespace {

// Sum or maximum of a column's four lanes, in each of them.
__device__ inline float quads_max(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return both_halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ inline float quads_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return both_halves_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Four codes as bf16.
__device__ inline uint2 codes_bf16(uint32_t w)
{
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true)));
}
__device__ inline Frag codes_frag(uint32_t lo, uint32_t hi)
{
    Frag f;
    f.h[0] = codes_bf16(lo);
    f.h[1] = codes_bf16(hi);
    return f;
}

// x in N bf16 parts, each the rounding of what those before it leave.
template <int N>
__device__ inline void split_pair(float x, float y, uint32_t (&part)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        part[i] = pack2(x, y);
        x -= __uint_as_float(part[i] << 16);
        y -= __uint_as_float(part[i] & 0xffff0000u);
    }
}

__device__ inline uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }     // 0x80 where a code is NaN

// A lane's share of a page: k of four blocks of 16 positions (its position of each, 16 channels of 64), v of all positions that the second
// product has in its lane (its channel of every 16).
template <int D>
struct PagePart {
    static constexpr int KW = D / 16;                    // words of k of a block
    uint32_t k[4][KW];
    uint4 v[D / 16];
    float k_scale, v_scale;
    __device__ inline void load(const Pages &p, int page, int h, int lane)
    {
        const int64_t at = (int64_t)page * p.heads + h;
        const int col = lane & 15, quad = lane >> 4;
        const uint8_t *kp = p.k + at * kPage * D + col * D, *vp = p.v + at * kPage * D + col * kPage + quad * 16;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            if (D == 32) {
                const uint2 x = *(const uint2 *)(kp + b * 16 * D + quad * 8);
                k[b][0] = x.x; k[b][1] = x.y;
            } else {
#pragma unroll
                for (int c = 0; c < D / 64; ++c) {
                    const uint4 x = *(const uint4 *)(kp + b * 16 * D + c * 64 + quad * 16);
                    k[b][4 * c % KW] = x.x; k[b][(4 * c + 1) % KW] = x.y; k[b][(4 * c + 2) % KW] = x.z; k[b][(4 * c + 3) % KW] = x.w;
                }
            }
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) v[c] = *(const uint4 *)(vp + c * 16 * kPage);
        k_scale = p.k_scale[at];
        v_scale = p.v_scale[at];
    }
};
// first of a lane's eight channels in reduction step f of the first product
template <int D>
__device__ inline int page_channel(int f, int quad) { return D == 32 ? 8 * quad : 64 * (f >> 1) + 16 * quad + 8 * (f & 1); }

// A wavefront's columns: NT tiles of 16, this lane's column of each.
template <int D, int NQ, int NP, int NT>
struct Columns {
    static constexpr int NF = D / 32, NC = D / 16;
    Frag q[NT][NF][NQ];
    int p[NT];                                           // position (-1: no column)
    int p0, p1;                                          // first and last position of the wavefront's columns
    float m[NT], l[NT];
    f32x4v acc[NT][NC];

    // Page number j of the row (as `t`): what its keys add.
    __device__ inline void take(const PagePart<D> &t, int j, float scale2, int window, int sinks, int lane)
    {
        const int quad = lane >> 4, j0 = j * kPage;
        const bool edge = j0 + kPage - 1 > p0 || (j0 <= p1 - window && j0 + kPage > sinks);
        const float sc = fmaxf(t.k_scale * scale2, 0x1p-126f);       // (a page of zeros has scale 0, and 0 times -infinity is none)
        f32x4v s[NT][4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            Frag k[NF];
#pragma unroll
            for (int f = 0; f < NF; ++f) k[f] = codes_frag(t.k[b][2 * f], t.k[b][2 * f + 1]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s[n][b] = f32x4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = NQ - 1; i >= 0; --i)
#pragma unroll
                    for (int f = 0; f < NF; ++f) s[n][b] = mfma16(k[f], q[n][f][i], s[n][b]);
            }
        }
        if (edge) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int hi = p[n] - j0 - 4 * quad, lo = max(0, p[n] - window + 1) - j0 - 4 * quad, first = sinks - j0 - 4 * quad;
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (16 * b + i > hi || (16 * b + i < lo && 16 * b + i >= first)) s[n][b][i] = -INFINITY;
            }
        }
        float top[NT];
        bool grows = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            top[n] = -INFINITY;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) top[n] = fmaxf(top[n], s[n][b][i]);
            top[n] = quads_max(top[n]) * sc;
            grows |= top[n] > m[n] + kSlack;
        }
        if (__any(grows)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float m1 = top[n] > m[n] + kSlack ? top[n] : m[n];
                const float fade = m[n] == m1 ? 1.f : __builtin_amdgcn_exp2f(m[n] - m1);
                m[n] = m1;
                l[n] *= fade;
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[n][c][i] *= fade;
            }
        }
        Frag pf[NT][2][NP];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float use = m[n] == -INFINITY ? 0.f : m[n];        // (nothing seen yet: every term is 2^-inf)
            float sum = 0.f;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(s[n][b][i], sc, -use));
                    sum += e;
                    s[n][b][i] = e * t.v_scale;
                }
            l[n] += sum;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t part[NP];
                    split_pair<NP>(s[n][b][2 * i], s[n][b][2 * i + 1], part);
#pragma unroll
                    for (int x = 0; x < NP; ++x) (i ? pf[n][b >> 1][x].h[b & 1].y : pf[n][b >> 1][x].h[b & 1].x) = part[x];
                }
        }
        // A code that not every column sees may be NaN (what is not yet written is anything), and 0 * NaN would reach the sums: such codes
        // are 0 in the product, and the columns that do see one get their NaN from a product of flags.
        if (edge) {
            uint32_t bad = 0;
#pragma unroll
            for (int c = 0; c < NC; ++c) bad |= nan_bytes(t.v[c].x) | nan_bytes(t.v[c].y) | nan_bytes(t.v[c].z) | nan_bytes(t.v[c].w);
            if (__any(bad != 0)) {
                careful(t, j0, window, sinks, quad, pf);
                return;
            }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const Frag v = half ? codes_frag(t.v[c].z, t.v[c].w) : codes_frag(t.v[c].x, t.v[c].y);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int x = NP - 1; x >= 0; --x) acc[n][c] = mfma16(v, pf[n][half][x], acc[n][c]);
            }
    }

    __device__ inline void careful(const PagePart<D> &t, int j0, int window, int sinks, int quad, const Frag (&pf)[NT][2][NP])
    {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int hi = p[n] - j0 - 4 * quad, lo = max(0, p[n] - window + 1) - j0 - 4 * quad, first = sinks - j0 - 4 * quad;
            Frag seen[2];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                uint32_t on[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) on[i] = 16 * b + i > hi || (16 * b + i < lo && 16 * b + i >= first) ? 0u : 0x3f80u;
                seen[b >> 1].h[b & 1] = make_uint2(on[0] | on[1] << 16, on[2] | on[3] << 16);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                f32x4v count = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t w[2] = {half ? t.v[c].z : t.v[c].x, half ? t.v[c].w : t.v[c].y};
                    uint32_t flag[2], clean[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t nan = nan_bytes(w[i]) >> 7;
                        clean[i] = w[i] & ~(nan * 0xffu);
                        flag[i] = nan * 0x38u;                       // (the code of 1)
                    }
                    const Frag v = codes_frag(clean[0], clean[1]);
#pragma unroll
                    for (int x = NP - 1; x >= 0; --x) acc[n][c] = mfma16(v, pf[n][half][x], acc[n][c]);
                    count = mfma16(codes_frag(flag[0], flag[1]), seen[half], count);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (count[i] > 0.f) acc[n][c][i] = __builtin_nanf("");
            }
        }
    }
};

// Eight channels of a query as the parts of a fragment.
template <typename T, int NQ>
__device__ inline void query_parts(const T *p, Frag (&f)[NQ])
{
    if constexpr (sizeof(T) == 2) {
        f[0].u = *(const uint4 *)p;
    } else {
        const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
        uint32_t part[4][NQ];
        split_pair<NQ>(a.x, a.y, part[0]);
        split_pair<NQ>(a.z, a.w, part[1]);
        split_pair<NQ>(b.x, b.y, part[2]);
        split_pair<NQ>(b.z, b.w, part[3]);
#pragma unroll
        for (int i = 0; i < NQ; ++i) f[i].u = make_uint4(part[0][i], part[1][i], part[2][i], part[3][i]);
    }
}

// The pages that positions p0 .. p1 see: those of the sinks before the window's, then the window's.
struct PageList {
    int sink_pages, first, count;
    __device__ inline PageList(int p0, int p1, int window, int sinks)
    {
        first = max(0, p0 - window + 1) / kPage;
        sink_pages = min((int)(((int64_t)sinks + kPage - 1) / kPage), first);
        count = p1 < 0 ? 0 : sink_pages + p1 / kPage - first + 1;
    }
    __device__ inline int number(int i) const { return i < sink_pages ? i : first + i - sink_pages; }
};

// Workgroup: WAVES wavefronts, CW of them beside each other over CW * NT * 16 columns of a row's key head, WAVES / CW over the pages.
template <typename T, typename O, int D, int NQ, int NP, int NT, int CW, int WAVES>
__global__ void __launch_bounds__(WAVES * 64)
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
    x.p0 = row.pos + c0 / G;
    x.p1 = c0 < columns ? row.pos + (min(c0 + NT * 16, columns) - 1) / G : -1;
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
    for (int i = split * KW + kw; i < list.count; i += a.splits * KW) {
        const int j = list.number(i), page = page_of(a.pages, row.b, j);
        if (page < 0) continue;
        PagePart<D> t;
        t.load(a.pages, page, hk, lane);
        x.take(t, j, scale2, a.window, a.sinks, lane);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) x.l[n] = quads_sum(x.l[n]);

    if constexpr (KW == 1) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (x.p[n] < 0) continue;
            const int c = c0 + 16 * n + col, token = c / G, h = hk * G + c - token * G;
            const float inv = x.l[n] == 0.f ? 0.f : 1.f / x.l[n];
            if (a.splits > 1) {
                float *p = a.parts + (((int64_t)(row.first + token) * a.Hq + h) * a.splits + split) * (D + 4);
#pragma unroll
                for (int b = 0; b < NC; ++b) *(float4 *)(p + 16 * b + 4 * quad) = make_float4(x.acc[n][b][0], x.acc[n][b][1], x.acc[n][b][2], x.acc[n][b][3]);
                if (quad == 0) { p[D] = x.m[n]; p[D + 1] = x.l[n]; }
            } else {
                O *op = (O *)a.o + (int64_t)(row.first + token) * a.lo.stride_n + h * a.lo.stride_h + 4 * quad;
#pragma unroll
                for (int b = 0; b < NC; ++b)
                    store4(op + 16 * b, x.acc[n][b][0] * inv, x.acc[n][b][1] * inv, x.acc[n][b][2] * inv, x.acc[n][b][3] * inv);
            }
        }
    } else {
        static_assert(CW == 1 && NT == 1, "wavefronts over the pages have one tile of columns");
        __shared__ __align__(16) float red[KW][16][D + 4];
        float *mine = red[kw][col];
#pragma unroll
        for (int b = 0; b < NC; ++b) *(float4 *)(mine + 16 * b + 4 * quad) = make_float4(x.acc[0][b][0], x.acc[0][b][1], x.acc[0][b][2], x.acc[0][b][3]);
        if (quad == 0) { mine[D] = x.m[0]; mine[D + 1] = x.l[0]; }
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * D / 4; i += WAVES * 64) {
            const int cc = i / (D / 4), ch = i % (D / 4) * 4, c = c0 + cc;
            if (c >= columns) continue;
            float top = red[0][cc][D];
#pragma unroll
            for (int w = 1; w < KW; ++w) top = fmaxf(top, red[w][cc][D]);
            const float use = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float f = __builtin_amdgcn_exp2f(red[w][cc][D] - use);
                const float4 r = *(const float4 *)&red[w][cc][ch];
                sum = fmaf(red[w][cc][D + 1], f, sum);
                o.x = fmaf(r.x, f, o.x); o.y = fmaf(r.y, f, o.y); o.z = fmaf(r.z, f, o.z); o.w = fmaf(r.w, f, o.w);
            }
            const int token = c / G, h = hk * G + c - token * G;
            if (a.splits > 1) {
                float *p = a.parts + (((int64_t)(row.first + token) * a.Hq + h) * a.splits + split) * (D + 4);
                *(float4 *)(p + ch) = o;
                if (ch == 0) { p[D] = top; p[D + 1] = sum; }
            } else {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                store4((O *)a.o + (int64_t)(row.first + token) * a.lo.stride_n + h * a.lo.stride_h + ch, o.x * inv, o.y * inv, o.z * inv, o.w * inv);
            }
        }
    }
}

// The splits of every query head joined: a thread has four channels of one (D / 4 of them a head).
template <typename O, int D>
__global__ void __launch_bounds__(256)
join_pages_kernel(AttendArgs a)
{
    constexpr int EACH = 256 / (D / 4);                  // heads of a workgroup
    const int64_t at = (int64_t)blockIdx.x * EACH + threadIdx.x / (D / 4);
    const int ch = threadIdx.x % (D / 4) * 4;
    if (at >= (int64_t)a.rows.tokens * a.Hq) return;
    const int token = (int)(at / a.Hq), h = (int)(at - (int64_t)token * a.Hq);
    // (a token that belongs to no row, or to an inactive one, has no parts)
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
    if (token < row.first || token >= row.first + row.n || row.pos < 0 ||
        (int64_t)row.pos + row.n > min((int64_t)a.rows.last_pos, (int64_t)a.pages.table_pages * kPage)) return;
    const float *p = a.parts + at * a.splits * (D + 4);
    float top = -INFINITY;
    for (int i = 0; i < a.splits; ++i) top = fmaxf(top, p[i * (D + 4) + D]);
    const float use = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < a.splits; ++i) {
        const float f = __builtin_amdgcn_exp2f(p[i * (D + 4) + D] - use);
        const float4 r = *(const float4 *)(p + i * (D + 4) + ch);
        sum = fmaf(p[i * (D + 4) + D + 1], f, sum);
        o.x = fmaf(r.x, f, o.x); o.y = fmaf(r.y, f, o.y); o.z = fmaf(r.z, f, o.z); o.w = fmaf(r.w, f, o.w);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    store4((O *)a.o + token * a.lo.stride_n + h * a.lo.stride_h + ch, o.x * inv, o.y * inv, o.z * inv, o.w * inv);
}

// How a launch divides its columns.
struct Shape {
    int nt, cw, waves;
    int columns() const { return 16 * nt * cw; }
};
Shape choose(const AttendArgs &a)
{
    const int64_t columns = (int64_t)a.rows.tokens * (a.Hq / a.pages.heads);
    if (columns <= 32 * (int64_t)a.rows.B) return {1, 1, 4};
    return {a.io_dtype == LASAD_BF16 && a.d <= 64 ? 2 : 1, 4, 4};
}
int64_t groups_of(const AttendArgs &a, const Shape &s) { return row_slots(a.rows, a.Hq / a.pages.heads, s.columns(), 1) * a.pages.heads; }

template <typename T, typename O, int D, int NP>
hipError_t launch(const AttendArgs &a, hipStream_t s)
{
    const Shape shape = choose(a);
    const dim3 grid((unsigned)groups_of(a, shape), (unsigned)a.splits);
    constexpr int WIDE = sizeof(T) == 2 && D <= 64 ? 2 : 1;
    if (shape.cw == 1) attend_pages_kernel<T, O, D, NP, NP, 1, 1, 4><<<grid, dim3(256), 0, s>>>(a);
    else attend_pages_kernel<T, O, D, NP, NP, WIDE, 4, 4><<<grid, dim3(256), 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) {
        const int64_t heads = (int64_t)a.rows.tokens * a.Hq, each = 1024 / D;
        join_pages_kernel<O, D><<<dim3((unsigned)((heads + each - 1) / each)), dim3(256), 0, s>>>(a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int64_t attend_pages_groups(const AttendArgs &a) { return groups_of(a, choose(a)) * a.splits; }

// Splits of a call whose rows see up to `seen` keys.
int attend_pages_splits(int64_t B, int64_t tokens, int Hq, int Hk, bool one_each, int64_t seen)
{
    const int64_t columns = tokens * (Hq / Hk);
    if (columns > 32 * B) return 1;
    const int64_t groups = (one_each ? B * ((Hq / Hk + 15) / 16) : columns / 16 + B) * Hk;
    int64_t n = 512 / groups;
    if (seen < 1536 || n < 4) return 1;
    if (n > seen / 512) n = seen / 512;
    return (int)(n > 64 ? 64 : n < 1 ? 1 : n);
}

size_t attend_pages_bytes(int64_t tokens, int Hq, int d, int splits)
{
    return splits > 1 ? (size_t)tokens * Hq * splits * (d + 4) * sizeof(float) : 0;
}

hipError_t launch_attend_pages(const AttendArgs &a, hipStream_t s)
{
#define LASAD_AT(T, O, NP) (a.d == 32 ? launch<T, O, 32, NP>(a, s) : a.d == 64 ? launch<T, O, 64, NP>(a, s) : launch<T, O, 128, NP>(a, s))
    if (a.io_dtype == LASAD_F32) return LASAD_AT(float, float, 3);
    return a.out_dtype == LASAD_BF16 ? LASAD_AT(uint16_t, uint16_t, 1) : LASAD_AT(uint16_t, float, 1);
#undef LASAD_AT
}

}  // namespace lasad
