// Attention with a window and sinks, backward.  With P = exp(scale q k^T - lse) over the seen pairs and
// delta_i = sum_c d_o_i[c] o_i[c] (which is sum_j P_ij dP_ij):
//     dP = d_o v^T,   dS = P (dP - delta) scale,   dq = dS k,   dk = dS^T q,   dv = P^T d_o,
// dk and dv of a shared head summed over its query heads.  Two passes form P and dP each: a sum over keys gives dq, a sum over
// queries gives dk and dv.  One pass would save two of the seven products and add dq up by atomics, in an order
// that changes from run to run.
//
// Query pass: as in the forward, the seen key tiles staged in LDS.  It also forms delta.
// Key pass: a workgroup has keys of one head and walks the tiles of the queries that see any of them,
// head after head of the group.  Ordinary keys are seen from `window` positions on, the sinks from all later ones: their
// tiles are cut into parts of about an ordinary tile's work, whose sums a small kernel adds up in their order.
// In the key pass -delta is what the sums of the second product start from, and in bf16 -lse / scale those of the first, so that an entry
// costs a product and an exponential for P and one more product for dS.  A sum that starts there is carried, and rounded, at the size of
// lse / scale, 44 for lse 5.5 and d = 64, where the scores' own is about 8: nothing beside bf16's operands (2^-8), but in fp32 twice the
// error of dk and dv (256 keys, emulated: 7.4e-7 and 3.8e-7).  There it starts from 0 and lse enters the multiply-add before the exponential.
// P and dS are rounded to the storage type as operands (bf16: half a step of 2^-8); all sums are fp32.  delta is formed from o as it
// was stored.  In the root mean square (16 heads of 576 tokens, window 144, unit variances) storing dq costs 1.7e-3 of it, the rounding
// of dS 1.7e-3, o's 0.7e-3, together 2.5e-3; dS as two operands would take the second part and cost a quarter to a third more products.
//
// bf16: lasad_window_backward_queries.hip and lasad_window_backward_keys.hip, 16 queries (keys) to a wavefront and 64 to a workgroup.
// fp32, here: 32 and 128.  Products of 32 x 32 x 2 bound it, and two wavefronts a SIMD (175 and 229 registers of d = 64) that hide little
// of what is between them: 2 x 20 heads of 1024 tokens, window 256, query pass 78 us and key pass 100, 48 and 50 TFLOP/s of the pairs that
// are seen (a product of 8192^3: 154); the tiles of 128 cover half as many pairs again.
#include "lasad_window.h"

namespace lasad {

namespace {

constexpr int kThreads = 256, kTile = 128;               // queries (keys) of a workgroup

// One block of 32 keys (from j0 on, rows of kt and vt) for a wavefront's queries: dS, and its product with k.
template <int D>
__device__ inline void dq_block(const float4 (&q)[D / 8], const float4 (&g)[D / 8], const float *kt, const float *vt, int j0, const Range &range,
                                const Edge &edge, float scale2, float lse2, float delta, int lane, f32x16 (&acc)[D / 32])
{
    typedef Mat<float> M;
    constexpr int LD = D + M::PAD, NF = D / M::KF, DB = D / 32;
    const int half = lane >> 5, col = lane & 31;
    f32x16 s = zeros16(), dp = zeros16();
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        s = M::mma(M::row(kt + col * LD, f, half), q[f], s);
        dp = M::mma(M::row(vt + col * LD, f, half), g[f], dp);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale2, -lse2)) * (dp[i] - delta);
    const bool top_edge = range.top_edge(j0 + 31), bottom_edge = range.bottom_edge(j0);
    if (top_edge || bottom_edge) hide(s, edge, j0, half, top_edge, bottom_edge, 0.f);
#pragma unroll
    for (int r = 0; r < M::GROUPS; ++r) {
        const float4 ds = M::pack(s, r);
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[d] = M::mma(M::column(kt, LD, d * 32, r, lane), ds, acc[d]);
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, D > 64 ? 1 : D == 32 ? 3 : 2)
window_dq_f32_kernel(WindowArgs a)
{
    typedef float T;
    typedef Mat<T> M;
    typedef float4 F;
    constexpr int KT = 32, LD = D + M::PAD, DB = D / 32, NF = D / M::KF;
    constexpr int PPR = D / M::VEC, RPP = kThreads / PPR, N = KT / RPP;
    __shared__ __align__(16) T tile[2][2][KT * LD];
    __shared__ int infinite;                             // whether a key that was taken out of a tile was not finite

    const int qt = (a.n + kTile - 1) / kTile;
    const Place place = launch_place(blockIdx.x, a.B * a.Hq, qt);
    if (place.head < 0) return;
    const int i0 = (qt - 1 - place.unit) * kTile;        // (the first queries see the fewest keys: last)
    const int bh = place.head, b = bh / a.Hq, h = bh % a.Hq, hk = h / (a.Hq / a.Hk);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int iq = i0 + 32 * wave + col, p = a.start_pos + iq;
    const int p0 = a.start_pos + i0 + 32 * wave, p1 = p0 + 31;
    const int last = min(i0 + kTile, a.n) - 1;
    const int keys = valid_keys(a, b);
    const int hi = min(a.start_pos + last, keys - 1), lo = max(0, a.start_pos + i0 - a.window + 1);
    const T *kp = (const T *)a.k + (int64_t)b * a.lk.stride_b + (int64_t)hk * a.lk.stride_h;
    const T *vp = (const T *)a.v + (int64_t)b * a.lv.stride_b + (int64_t)hk * a.lv.stride_h;

    const float scale2 = a.scale * kLog2e;
    const Edge edge = query_edge(a, keys, p);

    // (the walk over the keys is the forward's)
    const Range mine(a, keys, p0, p1), all(a, keys, a.start_pos + i0, a.start_pos + last);
    const int first = lo / KT, sink_tiles = min((min(a.sinks, hi + 1) + KT - 1) / KT, first);
    const int tiles = hi < 0 ? 0 : sink_tiles + max(0, hi / KT - first + 1);
    const int jump_from = sink_tiles * KT, jump_to = first * KT;
    const auto next = [&](int j0) { return j0 + KT == jump_from ? jump_to : j0 + KT; };
    const int begin = sink_tiles > 0 ? 0 : jump_to;
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
                bad |= make_finite<T>(kr[i]);
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
    F q[NF], g[NF];
    float delta = 0.f, lse2 = INFINITY;
    {
        const T *qp = (const T *)a.q + (int64_t)b * a.lq.stride_b + (int64_t)iq * a.lq.stride_n + (int64_t)h * a.lq.stride_h;
        const T *gp = (const T *)a.d_o + (int64_t)b * a.ldo.stride_b + (int64_t)iq * a.ldo.stride_n + (int64_t)h * a.ldo.stride_h;
        const T *op = (const T *)a.o + (int64_t)b * a.lo.stride_b + (int64_t)iq * a.lo.stride_n + (int64_t)h * a.lo.stride_h;
        const bool on = iq < a.n;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            q[f] = on ? M::row(qp, f, half) : M::zero();
            g[f] = on ? M::row(gp, f, half) : M::zero();
            if (on) delta += M::dot(g[f], M::row(op, f, half));
        }
        delta = both_halves_sum(delta);
        if (on) {
            lse2 = a.lse[(int64_t)bh * a.n + iq] * kLog2e;
            if (half == 0) a.delta[(int64_t)bh * a.n + iq] = delta;
        }
    }
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zeros16();
    // (the loop would wait for everything in flight if it might have to wait for the queries)
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
    if (tiles > 0) store(begin, 0);
    __syncthreads();
    int j0 = begin;
    for (int t = 0; t < tiles; ++t) {
        const T *kt = tile[t & 1][0], *vt = tile[t & 1][1];
        const int j1 = t + 1 < tiles ? next(j0) : j0;
        load(j1);
#pragma unroll 1
        for (int b = 0; b < KT; b += 32)
            if (mine.some(j0 + b, j0 + b + 31))
                dq_block<D>(q, g, kt + b * LD, vt + b * LD, j0 + b, mine, edge, scale2, lse2, delta, lane, acc);
        if (t + 1 < tiles) store(j1, (t + 1) & 1);
        __syncthreads();
        j0 = j1;
    }
    if (infinite) {                                      // (a seen key that is not finite: so is the row's gradient)
        int j0 = begin;
        for (int t = 0; t < tiles; ++t, j0 = next(j0)) {
            if (all.all(j0, j0 + KT - 1)) continue;      // (as it was)
            for (int j = j0; j < min(j0 + KT, keys); ++j) {
                const bool bad = row_infinite<T, D>(kp + (int64_t)j * a.lk.stride_n, lane);
                if (bad && sees(a, keys, p, j)) {
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[d][i] = NAN;
                }
            }
        }
    }
    if (iq >= a.n) return;
    float *dq = (float *)a.dq + (int64_t)b * a.ldq.stride_b + (int64_t)iq * a.ldq.stride_n + (int64_t)h * a.ldq.stride_h;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            store4(dq + d * 32 + 8 * r + 4 * half, acc[d][4 * r] * a.scale, acc[d][4 * r + 1] * a.scale, acc[d][4 * r + 2] * a.scale,
                   acc[d][4 * r + 3] * a.scale);
}

// One block of 32 queries (positions from pb on, rows of qt and gt, their lse (in powers of two) and -delta) for a wavefront's keys: P and
// dS, and their products with d_o and q.
template <int D>
__device__ inline void dkv_block(const WindowArgs &a, const float4 (&k)[D / 8], const float4 (&v)[D / 8],
                                 const float *qt, const float *gt, const float *lse2, const float *delta, int pb, int keys, int w0, const Edge &edge,
                                 float scale2, int lane, f32x16 (&dk)[D / 32], f32x16 (&dv)[D / 32])
{
    typedef Mat<float> M;
    typedef typename M::F F;
    constexpr int LD = D + M::PAD, NF = D / M::KF, DB = D / 32;
    const int half = lane >> 5, col = lane & 31;
    f32x16 s = zeros16(), dp;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float4 y = *(const float4 *)(delta + 8 * r + 4 * half);
        dp[4 * r] = y.x; dp[4 * r + 1] = y.y; dp[4 * r + 2] = y.z; dp[4 * r + 3] = y.w;
    }
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        s = M::mma(M::row(qt + col * LD, f, half), k[f], s);
        dp = M::mma(M::row(gt + col * LD, f, half), v[f], dp);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float4 x = *(const float4 *)(lse2 + 8 * r + 4 * half);
        const float l[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[4 * r + i] = __builtin_amdgcn_exp2f(fmaf(s[4 * r + i], scale2, -l[i]));
            dp[4 * r + i] *= s[4 * r + i];
        }
    }
    const bool first_edge = pb < w0 + 31 || w0 + 31 >= keys, last_edge = pb + 31 - w0 >= a.window;
    if (first_edge || last_edge) {
        hide(s, edge, pb, half, last_edge, first_edge, 0.f);
        hide(dp, edge, pb, half, last_edge, first_edge, 0.f);
    }
#pragma unroll
    for (int r = 0; r < M::GROUPS; ++r) {
        const F pf = M::pack(s, r), df = M::pack(dp, r);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            dv[d] = M::mma(M::column(gt, LD, d * 32, r, lane), pf, dv[d]);
            dk[d] = M::mma(M::column(qt, LD, d * 32, r, lane), df, dk[d]);
        }
    }
}

// Workgroups: first the sinks' key tiles, part after part, then the others.
template <int D>
__global__ void __launch_bounds__(kThreads, D <= 64 ? 2 : 1)
window_dkv_f32_kernel(WindowArgs a)
{
    typedef float T;
    typedef Mat<T> M;
    typedef float4 F;
    constexpr int QT = 32, LD = D + M::PAD, QB = QT / 32, DB = D / 32, NF = D / M::KF;
    constexpr int PPR = D / M::VEC, RPP = kThreads / PPR, N = QT / RPP;
    __shared__ __align__(16) T tile[2][2][QT * LD];
    __shared__ __align__(16) float stat[2][2][QT];       // lse (in powers of two) and -delta of a tile's queries
    __shared__ int infinite;                             // whether a row that was taken out of a tile was not finite

    const int kt = (a.m + kTile - 1) / kTile;
    const int units = a.sink_tiles * a.sink_parts + kt - a.sink_tiles;      // workgroups of a key head
    const Place place = launch_place(blockIdx.x, a.B * a.Hk, units);
    if (place.head < 0) return;
    const int unit = place.unit, bh = place.head, b = bh / a.Hk, hk = bh % a.Hk, G = a.Hq / a.Hk;
    const bool sink = unit < a.sink_tiles * a.sink_parts;
    const int kti = sink ? unit / a.sink_parts : unit - a.sink_tiles * a.sink_parts + a.sink_tiles;
    const int part = sink ? unit % a.sink_parts : 0, parts = sink ? a.sink_parts : 1;
    const int j0 = kti * kTile;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int jk = j0 + 32 * wave + col;                             // this lane's key
    const int w0 = j0 + 32 * wave, w1 = w0 + 31;                     // the wavefront's
    // (keys behind the last query are nobody's; a tile's rows behind it have lse = inf, so that P is 0 for every finite key)
    const int keys = min(valid_keys(a, b), a.start_pos + a.n);

    F k[NF], v[NF];
    {
        const T *kp = (const T *)a.k + (int64_t)b * a.lk.stride_b + (int64_t)jk * a.lk.stride_n + (int64_t)hk * a.lk.stride_h;
        const T *vp = (const T *)a.v + (int64_t)b * a.lv.stride_b + (int64_t)jk * a.lv.stride_n + (int64_t)hk * a.lv.stride_h;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            k[f] = jk < keys ? M::row(kp, f, half) : M::zero();
            v[f] = jk < keys ? M::row(vp, f, half) : M::zero();
        }
    }
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = dv[d] = zeros16();
    const float scale2 = a.scale * kLog2e;
    const Edge edge = key_edge(a, keys, jk);

    // queries that see any key of the tile, in tiles of QT counted from the first query; this part's share of them
    const int j1 = min(j0 + kTile, keys) - 1;                        // (no valid key: j1 < j0)
    int q_lo = max(0, j0 - a.start_pos), q_hi = a.n - 1;
    if (j0 >= a.sinks) q_hi = (int)min((int64_t)q_hi, (int64_t)j1 + a.window - 1 - a.start_pos);
    const int t_lo = q_lo / QT;
    const int t_all = j1 < j0 || q_hi < q_lo ? 0 : q_hi / QT - t_lo + 1;
    const int share = (t_all + parts - 1) / parts, t_first = t_lo + part * share;
    const int t_count = max(0, min(share, t_all - part * share)), steps = t_count * G;

    const T *qp = (const T *)a.q + (int64_t)b * a.lq.stride_b + (int64_t)hk * G * a.lq.stride_h;
    const T *gp = (const T *)a.d_o + (int64_t)b * a.ldo.stride_b + (int64_t)hk * G * a.ldo.stride_h;
    const int64_t stat0 = ((int64_t)b * a.Hq + hk * G) * a.n;
    uint4 qr[N], gr[N];
    float sr = 0.f;
    const int row0 = threadIdx.x / PPR, col0 = (threadIdx.x % PPR) * M::VEC;
    const int64_t qoff = row0 * a.lq.stride_n + col0, goff = row0 * a.ldo.stride_n + col0;
    const float *statp = threadIdx.x < QT ? a.lse : a.delta;
    const auto load = [&](int ti, int hi) {              // tile (of the share) of a head of the group; rows behind the last: the last
        const int i0 = (t_first + ti) * QT;
        const T *q0 = qp + i0 * a.lq.stride_n + hi * a.lq.stride_h, *g0 = gp + i0 * a.ldo.stride_n + hi * a.ldo.stride_h;
        int64_t qo[N], go[N];
#pragma unroll
        for (int i = 0; i < N; ++i) { qo[i] = qoff + i * RPP * a.lq.stride_n; go[i] = goff + i * RPP * a.ldo.stride_n; }
        if (i0 + QT > a.n) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int64_t row = min(row0 + i * RPP, a.n - 1 - i0);
                qo[i] = row * a.lq.stride_n + col0;
                go[i] = row * a.ldo.stride_n + col0;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            qr[i] = *(const uint4 *)(q0 + qo[i]);
            gr[i] = *(const uint4 *)(g0 + go[i]);
        }
        if (threadIdx.x < 2 * QT) sr = statp[stat0 + (int64_t)hi * a.n + min(i0 + (int)threadIdx.x % QT, a.n - 1)];
    };
    const auto whole = [&](int ti) {
        const int p0 = a.start_pos + (t_first + ti) * QT;
        return (t_first + ti + 1) * QT <= a.n && sees_all(a, keys, p0, p0 + QT - 1, j0, j0 + kTile - 1);
    };
    const auto store = [&](int buf, int ti) {            // what was loaded last
        const int i0 = (t_first + ti) * QT;
        if (!whole(ti)) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (i0 + row0 + i * RPP >= a.n) qr[i] = gr[i] = make_uint4(0, 0, 0, 0);
                bad |= make_finite<T>(qr[i]);
                bad |= make_finite<T>(gr[i]);
            }
            if (bad) infinite = 1;
            if (i0 + (int)threadIdx.x % QT >= a.n) sr = threadIdx.x < QT ? INFINITY : 0.f;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            *(uint4 *)(tile[buf][0] + (row0 + i * RPP) * LD + col0) = qr[i];
            *(uint4 *)(tile[buf][1] + (row0 + i * RPP) * LD + col0) = gr[i];
        }
        if (threadIdx.x < 2 * QT) stat[buf][threadIdx.x / QT][threadIdx.x % QT] = threadIdx.x < QT ? sr * kLog2e : -sr;
    };
    if (threadIdx.x == 0) infinite = 0;
    if (steps > 0) load(0, 0);
    __builtin_amdgcn_s_waitcnt(0x0f70);                  // (as in the query pass)
    __syncthreads();
    if (steps > 0) store(0, 0);
    __syncthreads();
    int ti = 0, hi = 0;                                  // tile and head of the present step
    for (int t = 0; t < steps; ++t) {
        const int p0 = a.start_pos + (t_first + ti) * QT;
        if (t + 1 < steps && ++ti == t_count) { ti = 0; ++hi; }
        load(ti, hi);                                    // (the last tile once more rather than a branch around loads in flight)
        const T *qt = tile[t & 1][0], *gt = tile[t & 1][1];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
            if (!sees_none(a, keys, p0 + 32 * qb, p0 + 32 * qb + 31, w0, w1))
                dkv_block<D>(a, k, v, qt + qb * 32 * LD, gt + qb * 32 * LD, stat[t & 1][0] + 32 * qb, stat[t & 1][1] + 32 * qb, p0 + 32 * qb,
                                keys, w0, edge, scale2, lane, dk, dv);
        if (t + 1 < steps) store((t + 1) & 1, ti);
        __syncthreads();
    }
    if (infinite) {                                      // (a query that is not finite: so are the gradients of all keys it sees)
        for (int h = 0; h < G; ++h)
            for (int t = 0; t < t_count; ++t) {
                if (whole(t)) continue;                  // (as they were)
                for (int iq = (t_first + t) * QT; iq < min((t_first + t + 1) * QT, a.n); ++iq) {
                    const bool on = sees(a, keys, a.start_pos + iq, jk), bad = row_infinite<T, D>(qp + iq * a.lq.stride_n + h * a.lq.stride_h, lane);
                    add_infinite<T, DB>(gp + iq * a.ldo.stride_n + h * a.ldo.stride_h, on, half, dv);
                    if (bad && on) {
#pragma unroll
                        for (int d = 0; d < DB; ++d)
#pragma unroll
                            for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = NAN;
                    }
                }
            }
    }
    if (parts > 1) {                                     // (whole tiles, rows past the last key included)
        float *out = a.parts + (((int64_t)bh * a.sink_tiles * a.sink_parts + unit) * 2 * kTile + 32 * wave + col) * D;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int c = d * 32 + 8 * r + 4 * half;
                store4(out + c, dk[d][4 * r], dk[d][4 * r + 1], dk[d][4 * r + 2], dk[d][4 * r + 3]);
                store4(out + (int64_t)kTile * D + c, dv[d][4 * r], dv[d][4 * r + 1], dv[d][4 * r + 2], dv[d][4 * r + 3]);
            }
        return;
    }
    if (jk >= a.m) return;
    float *dkp = (float *)a.dk + (int64_t)b * a.ldk.stride_b + (int64_t)jk * a.ldk.stride_n + (int64_t)hk * a.ldk.stride_h;
    float *dvp = (float *)a.dv + (int64_t)b * a.ldv.stride_b + (int64_t)jk * a.ldv.stride_n + (int64_t)hk * a.ldv.stride_h;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int c = d * 32 + 8 * r + 4 * half;
            store4(dkp + c, dk[d][4 * r] * a.scale, dk[d][4 * r + 1] * a.scale, dk[d][4 * r + 2] * a.scale, dk[d][4 * r + 3] * a.scale);
            store4(dvp + c, dv[d][4 * r], dv[d][4 * r + 1], dv[d][4 * r + 2], dv[d][4 * r + 3]);
        }
}

// The parts of the sinks' tiles added up: a thread has four channels of one row of dk or dv.
template <typename O>
__global__ void __launch_bounds__(kThreads)
window_sink_sum_kernel(WindowArgs a)
{
    const int q = a.d / 4;                               // pieces of a row
    const int64_t total = (int64_t)a.B * a.Hk * a.sink_tiles * 2 * a.key_tile * q;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (id >= total) return;
    const int c = (int)(id % q) * 4;
    const int row = (int)(id / q % a.key_tile), which = (int)(id / q / a.key_tile % 2);
    const int64_t tile = id / q / a.key_tile / 2;             // (b, hk, sink tile)
    const int j = (int)(tile % a.sink_tiles) * a.key_tile + row;
    if (j >= a.m) return;
    const int bh = (int)(tile / a.sink_tiles), b = bh / a.Hk, hk = bh % a.Hk;
    const float *p = a.parts + (tile * a.sink_parts * 2 + which) * a.key_tile * a.d + (int64_t)row * a.d + c;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < a.sink_parts; ++i) {
        const float4 x = *(const float4 *)(p + (int64_t)i * 2 * a.key_tile * a.d);
        s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
    }
    const lasad_layout_t &l = which ? a.ldv : a.ldk;
    const float f = which ? 1.f : a.scale;
    O *out = (O *)(which ? a.dv : a.dk) + (int64_t)b * l.stride_b + (int64_t)j * l.stride_n + (int64_t)hk * l.stride_h + c;
    store4(out, s.x * f, s.y * f, s.z * f, s.w * f);
}

// Few queries or keys: too few workgroups to fill the chip's 256 units; a workgroup then has 32 of them and its wavefronts share out the
// walk.  us, few and many.  fp32, both passes, window 128 of 256 tokens, 12 heads: batch 4 (96 workgroups of 128) 58 and 82, 8 96 and 85;
// d = 128, whose wavefronts fill a SIMD alone, by a smaller count.
bool few_f32(int64_t heads, int64_t count, int d) { return heads * ((count + kTile - 1) / kTile) < (d == 128 ? 96 : 144); }

// bf16, counted in 128 queries, by the walk's tiles of 64 keys too.  d = 64: 2048 tokens, all seen, 96 26 and 33, 144 43 and 36; window
// 256 (5 tiles) 64 9.2 and 10.6, 96 13.0 and 11.4; window 32 64 6.8 and 8.0, 96 9.3 and 9.0.  d = 128, window 256: 64 14 and 16, 96 26 and
// 16; all seen 96 37 and 50, 144 88 and 58.
bool few_queries(int64_t heads, int64_t n, int64_t tiles) { return heads * ((n + 127) / 128) < (tiles < 16 ? 68 : 128); }

bool few_query_pass(const WindowArgs &a)
{
    const int64_t heads = (int64_t)a.B * a.Hq, seen = (int64_t)a.window + 64 < a.start_pos + a.n ? (int64_t)a.window + 64 : a.start_pos + a.n;
    return a.io_dtype == LASAD_BF16 ? few_queries(heads, a.n, (seen + 63) / 64) : few_f32(heads, a.n, a.d);
}

// The same of keys: 2048 tokens, all seen, 96 28 and 51, 144 48 and 55; window 256 64 11.9 and 12.9, 96 15.0 and 13.3; window 32 (2 tiles) 48
// 8.2 and 8.2, 96 9.9 and 8.5.  d = 128, window 256: 64 17 and 20, 96 33 and 20; all seen 96 42 and 78, 144 95 and 87.
bool few_keys(int64_t heads, int64_t m, int64_t tiles) { return heads * ((m + 127) / 128) < (tiles < 4 ? 0 : tiles < 16 ? 72 : 128); }

// The key pass' tiles, those with sinks, and the parts they are cut into.  In steps of 64 queries: an ordinary tile takes
// (window + tile) / 64, one with sinks n / 64.  Uncut it ends last where it takes longer than an ordinary one and than half of what
// the chip's 512 workgroup slots (of 64 keys: 1024) have to do anyway; a part takes about that long.  At most 1024 parts, which bounds the workspace.
struct Plan {
    int tile, sink_tiles, parts;
};
Plan plan(int io_dtype, int64_t heads, int d, int n, int m, int window, int sinks)
{
    Plan r;
    const int64_t sink = (n + 63) / 64;
    const auto ordinary_steps = [&](int tile) { const int64_t near = ((int64_t)window + tile + 63) / 64; return near < sink ? near : sink; };
    if (io_dtype == LASAD_BF16) r.tile = few_keys(heads, m, ordinary_steps(kWindowKeyTile)) ? 32 : kWindowKeyTile;
    else r.tile = few_f32(heads, m, d) ? 32 : kTile;
    r.sink_tiles = (int)(((int64_t)(sinks < m ? sinks : m) + r.tile - 1) / r.tile);
    const int64_t all = ((int64_t)m + r.tile - 1) / r.tile, ordinary = ordinary_steps(r.tile);
    const int64_t slot = heads * ((all - r.sink_tiles) * ordinary + r.sink_tiles * sink) / (r.tile == kWindowKeyTile ? 1024 : 512);
    const int64_t long_enough = ordinary > slot / 2 ? ordinary : slot / 2;
    const int64_t want = long_enough > 0 ? (sink + long_enough - 1) / long_enough : 1, most = r.sink_tiles > 0 ? 1024 / (heads * r.sink_tiles) : 1;
    const int64_t parts = want > most ? most : want;
    r.parts = (int)(parts < 1 ? 1 : parts > 64 ? 64 : parts);
    return r;
}

size_t delta_bytes(int B, int Hq, int n) { return ((size_t)B * Hq * n * sizeof(float) + 255) / 256 * 256; }

}  // namespace

size_t window_backward_bytes(int B, int Hq, int Hk, int d, int n, int m, int window, int sinks)
{
    size_t parts = 0;                                    // (whichever type needs more)
    for (int type : {LASAD_F32, LASAD_BF16}) {
        const Plan r = plan(type, (int64_t)B * Hk, d, n, m, window, sinks);
        const size_t bytes = (size_t)B * Hk * r.sink_tiles * r.parts * 2 * r.tile * d * sizeof(float);
        if (r.parts > 1 && bytes > parts) parts = bytes;
    }
    return delta_bytes(B, Hq, n) + parts;
}

int64_t window_backward_groups(const WindowArgs &a)
{
    const Plan r = plan(a.io_dtype, (int64_t)a.B * a.Hk, a.d, a.n, a.m, a.window, a.sinks);
    const int64_t heads = (int64_t)a.B * a.Hq, queries = few_query_pass(a) ? 32 : a.io_dtype == LASAD_BF16 ? 64 : kTile;
    const int64_t q = launch_groups(heads, (a.n + queries - 1) / queries);
    const int64_t k = launch_groups((int64_t)a.B * a.Hk, (int64_t)r.sink_tiles * r.parts + (a.m + r.tile - 1) / r.tile - r.sink_tiles);
    return q > k ? q : k;
}

hipError_t launch_window_backward(WindowArgs &a, void *workspace, hipStream_t s)
{
    a.delta = (float *)workspace;
    a.parts = (float *)((char *)workspace + delta_bytes(a.B, a.Hq, a.n));
    const Plan r = plan(a.io_dtype, (int64_t)a.B * a.Hk, a.d, a.n, a.m, a.window, a.sinks);
    a.key_tile = r.tile; a.sink_tiles = r.sink_tiles; a.sink_parts = r.parts;
    hipError_t e = hipSuccess;
    if (a.n > 0) {
        if (few_query_pass(a)) {
            e = launch_window_dq_few(a, s);
        } else if (a.io_dtype == LASAD_BF16) {
            e = launch_window_dq_bf16(a, s);
        } else {
            const dim3 grid(launch_grid((int64_t)a.B * a.Hq, (a.n + kTile - 1) / kTile));
            if (a.d == 32) window_dq_f32_kernel<32><<<grid, dim3(kThreads), 0, s>>>(a);
            else if (a.d == 64) window_dq_f32_kernel<64><<<grid, dim3(kThreads), 0, s>>>(a);
            else window_dq_f32_kernel<128><<<grid, dim3(kThreads), 0, s>>>(a);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
    }
    if (a.m == 0) return hipSuccess;
    if (r.tile == 32) {
        e = launch_window_dkv_few(a, s);
    } else if (a.io_dtype == LASAD_BF16) {
        e = launch_window_dkv_bf16(a, s);
    } else {
        const dim3 grid(launch_grid((int64_t)a.B * a.Hk, r.sink_tiles * r.parts + (a.m + kTile - 1) / kTile - r.sink_tiles));
        if (a.d == 32) window_dkv_f32_kernel<32><<<grid, dim3(kThreads), 0, s>>>(a);
        else if (a.d == 64) window_dkv_f32_kernel<64><<<grid, dim3(kThreads), 0, s>>>(a);
        else window_dkv_f32_kernel<128><<<grid, dim3(kThreads), 0, s>>>(a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && r.sink_tiles > 0 && r.parts > 1) {
        const int64_t total = (int64_t)a.B * a.Hk * r.sink_tiles * 2 * r.tile * (a.d / 4);
        const dim3 sums((unsigned)((total + kThreads - 1) / kThreads));
        if (a.out_dtype == LASAD_BF16) window_sink_sum_kernel<uint16_t><<<sums, dim3(kThreads), 0, s>>>(a);
        else window_sink_sum_kernel<float><<<sums, dim3(kThreads), 0, s>>>(a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace lasad
