// The forward of the window attention, bf16, for middling numbers of queries and for d = 128 (lasad_window_forward.hip has the formulas).
//
// A wavefront has 16 queries and takes 32 keys at a time, in products of 16 x 16, 64 queries to a workgroup: twice as many workgroups as with
// 32 and 128, and 64 fewer registers of d = 128, where eight times as many wavefronts then hide each other's chains.  A query's maximum lies in
// four lanes instead of two and every key row is read from LDS twice as often, which costs where there is work for all units anyway.
//
// Measured, bf16: d = 64, 24 heads of 2048 tokens, window 256, 16 us (32 queries a wavefront 18.4, 32 a workgroup 20.6); d = 128 23 (27, 63), of 2048
// heads of 64 tokens 27 (39, 97).  4 x 24 heads of 4096 tokens, d = 64, window 1024 190 (142).
#include "lasad_window.h"

namespace lasad {

namespace {

constexpr int kThreads = 256, kQueries = 64;

// One block of 32 keys (from j0 on, rows of kt and vt) for a wavefront's 16 queries.
template <int D>
__device__ inline void forward_block(const Frag (&q)[D / 32], const uint16_t *kt, const uint16_t *vt, int j0, const Range &range, const Edge &edge,
                                       float scale2, int lane, float &m, float &l, f32x4v (&acc)[D / 16])
{
    typedef Mat<uint16_t> M;
    constexpr int LD = D + M::PAD, NF = D / 32, NC = D / 16;
    const int quad = lane >> 4, col = lane & 15;
    const int own = first_row(quad), row = first_row(col >> 2) + 4 * (col & 3);
    f32x4v s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int f = 0; f < NF; ++f) s[t] = mfma16(M::piece(kt + (16 * t + row) * LD + channel<D>(f, quad)), q[f], s[t]);
    if (range.top_edge(j0 + 31) || range.bottom_edge(j0)) {
        const int hi = edge.hi - j0 - own, lo = edge.lo - j0 - own, first = edge.first - j0 - own;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (16 * t + 4 * i > hi || (16 * t + 4 * i < lo && 16 * t + 4 * i >= first)) s[t][i] = -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
    {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(fmaxf(-INFINITY, __uint_as_float(r[0])), __uint_as_float(r[1]));
    }
    top = both_halves_max(top) * scale2;
    if (__any(top > m + kSlack)) {                       // (as in lasad_window_forward.hip)
        const float m1 = top > m + kSlack ? top : m;
        const float fade = m == m1 ? 1.f : __builtin_amdgcn_exp2f(m - m1);
        m = m1;
        l *= fade;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[c][i] *= fade;
    }
    const float use = m == -INFINITY ? 0.f : m;          // (nothing seen yet: every term is 2^-inf)
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], scale2, -use));
            sum += s[t][i];
        }
    l += sum;
    Frag pf;
    pf.u = make_uint4(pack2(s[0][0], s[0][1]), pack2(s[0][2], s[0][3]), pack2(s[1][0], s[1][1]), pack2(s[1][2], s[1][3]));
    const int at = (own + 4 * (col >> 2)) * LD + 4 * (col & 3);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        Frag x;
        x.h[0] = tr_read(vt + at + 16 * c);
        x.h[1] = tr_read(vt + at + 16 * LD + 16 * c);
        acc[c] = mfma16(x, pf, acc[c]);
    }
}

template <typename O, int D>
__global__ void __launch_bounds__(kThreads, 4)
window_forward_16_kernel(WindowArgs a)
{
    typedef uint16_t T;
    typedef Mat<T> M;
    typedef Frag F;
    constexpr int KT = D > 64 ? 32 : 64, LD = D + M::PAD, NC = D / 16, NF = D / 32;
    constexpr int PPR = D / 8, RPP = kThreads / PPR, N = KT / RPP;
    static_assert(N >= 1, "a tile has at least one piece for every thread");
    __shared__ __align__(16) T tile[2][2][KT * LD];
    __shared__ int infinite;                             // whether a value that was taken out of a tile was not finite

    const int qt = (a.n + kQueries - 1) / kQueries;
    const Place place = launch_place(blockIdx.x, a.B * a.Hq, qt);
    if (place.head < 0) return;
    const int i0 = (qt - 1 - place.unit) * kQueries;     // (the first queries see the fewest keys: last)
    const int bh = place.head, b = bh / a.Hq, h = bh % a.Hq, hk = h / (a.Hq / a.Hk);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, quad = lane >> 4, col = lane & 15;
    const int iq = i0 + 16 * wave + col, p = a.start_pos + iq;       // this lane's query
    const int p0 = a.start_pos + i0 + 16 * wave, p1 = p0 + 15;       // the wavefront's
    const int last = min(i0 + kQueries, a.n) - 1;                    // the workgroup's last query
    const int keys = valid_keys(a, b);
    const int hi = min(a.start_pos + last, keys - 1), lo = max(0, a.start_pos + i0 - a.window + 1);
    const T *kp = (const T *)a.k + (int64_t)b * a.lk.stride_b + (int64_t)hk * a.lk.stride_h;
    const T *vp = (const T *)a.v + (int64_t)b * a.lv.stride_b + (int64_t)hk * a.lv.stride_h;

    const float scale2 = a.scale * kLog2e;
    const Edge edge = query_edge(a, keys, p);

    // key tiles: those of the sinks before the window's, then the window's
    const Range mine(a, keys, p0, p1), all(a, keys, a.start_pos + i0, a.start_pos + last);       // the wavefront's, the workgroup's
    const int first = lo / KT, sink_tiles = min((min(a.sinks, hi + 1) + KT - 1) / KT, first);
    const int tiles = hi < 0 ? 0 : sink_tiles + max(0, hi / KT - first + 1);
    const int jump_from = sink_tiles * KT, jump_to = first * KT;
    const auto next = [&](int j0) { return j0 + KT == jump_from ? jump_to : j0 + KT; };
    const int begin = sink_tiles > 0 ? 0 : jump_to;
    // a thread's 16-byte pieces of a tile: PPR to a row, rows RPP apart.  Rows behind the last one that is seen are loaded from
    // there; what no query of the workgroup may see is 0 in LDS (what lies there cannot reach a sum as 0 * NaN).
    uint4 kr[N], vr[N];
    const int row0 = threadIdx.x / PPR, col0 = (threadIdx.x % PPR) * M::VEC;
    const int64_t koff = row0 * a.lk.stride_n + col0, voff = row0 * a.lv.stride_n + col0;
    const auto load = [&](int j0) {
        const T *k0 = kp + j0 * a.lk.stride_n, *v0 = vp + j0 * a.lv.stride_n;
        if (j0 + KT - 1 > hi) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int64_t row = min(row0 + i * RPP, hi - j0);
                kr[i] = *(const uint4 *)(k0 + (row * a.lk.stride_n + col0));
                vr[i] = *(const uint4 *)(v0 + (row * a.lv.stride_n + col0));
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                kr[i] = *(const uint4 *)(k0 + i * RPP * a.lk.stride_n + koff);
                vr[i] = *(const uint4 *)(v0 + i * RPP * a.lv.stride_n + voff);
            }
        }
    };
    const auto store = [&](int j0, int half) {
        if (!all.all(j0, j0 + KT - 1)) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int j = j0 + row0 + i * RPP;
                if (j > hi || (j < lo && j >= a.sinks)) kr[i] = vr[i] = make_uint4(0, 0, 0, 0);
                bad |= make_finite<T>(vr[i]);
            }
            if (bad) infinite = 1;
        }
        T *at = tile[half][0] + row0 * LD + col0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            *(uint4 *)(at + i * RPP * LD) = kr[i];
            *(uint4 *)(at + KT * LD + i * RPP * LD) = vr[i];
        }
    };
    if (threadIdx.x == 0) infinite = 0;
    if (tiles > 0) load(begin);
    F q[NF];
    {
        const T *qp = (const T *)a.q + (int64_t)b * a.lq.stride_b + (int64_t)iq * a.lq.stride_n + (int64_t)h * a.lq.stride_h;
#pragma unroll
        for (int f = 0; f < NF; ++f) q[f] = iq < a.n ? M::piece(qp + channel<D>(f, quad)) : M::zero();
    }
    f32x4v acc[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] = f32x4v{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    // (the loop would wait for everything in flight if it might have to wait for the queries)
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
    if (tiles > 0) store(begin, 0);
    __syncthreads();
    int j0 = begin;
    for (int t = 0; t < tiles; ++t) {
        const T *kt = tile[t & 1][0], *vt = tile[t & 1][1];
        const int j1 = t + 1 < tiles ? next(j0) : j0;    // (the last tile once more rather than a branch around loads in flight)
        load(j1);
#pragma unroll 1
        for (int b = 0; b < KT; b += 32)
            if (mine.some(j0 + b, j0 + b + 31)) forward_block<D>(q, kt + b * LD, vt + b * LD, j0 + b, mine, edge, scale2, lane, m, l, acc);
        if (t + 1 < tiles) store(j1, (t + 1) & 1);
        __syncthreads();
        j0 = j1;
    }
    l += __shfl_xor(l, 16);
    l = both_halves_sum(l);                              // (each quad added up its own rows)
    if (iq >= a.n) return;
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[c][i] *= inv;
    if (infinite) {
        int j0 = begin;
        for (int t = 0; t < tiles; ++t, j0 = next(j0)) {
            if (all.all(j0, j0 + KT - 1)) continue;      // (as it was)
            for (int j = j0; j < min(j0 + KT, keys); ++j) {
                const bool on = sees(a, keys, p, j);
                const T *row = vp + (int64_t)j * a.lv.stride_n + 4 * quad;
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = as_float<T>(row[16 * c + i]);
                        if (on && !(fabsf(x) < INFINITY)) acc[c][i] += x;
                    }
            }
        }
    }
    O *op = (O *)a.o + (int64_t)b * a.lo.stride_b + (int64_t)iq * a.lo.stride_n + (int64_t)h * a.lo.stride_h + 4 * quad;
#pragma unroll
    for (int c = 0; c < NC; ++c) store4(op + 16 * c, acc[c][0], acc[c][1], acc[c][2], acc[c][3]);
    if (a.lse && quad == 0) a.lse[(int64_t)bh * a.n + iq] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace

hipError_t launch_window_forward_16(const WindowArgs &a, hipStream_t s)
{
    const dim3 grid(launch_grid((int64_t)a.B * a.Hq, (a.n + kQueries - 1) / kQueries));
#define LASAD_WF(O, D) window_forward_16_kernel<O, D><<<grid, dim3(kThreads), 0, s>>>(a)
    if (a.out_dtype == LASAD_BF16) {
        if (a.d == 32) LASAD_WF(uint16_t, 32); else if (a.d == 64) LASAD_WF(uint16_t, 64); else LASAD_WF(uint16_t, 128);
    } else {
        if (a.d == 32) LASAD_WF(float, 32); else if (a.d == 64) LASAD_WF(float, 64); else LASAD_WF(float, 128);
    }
#undef LASAD_WF
    return hipGetLastError();
}

}  // namespace lasad
