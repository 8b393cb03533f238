// Attention with a window and sinks, backward.  With P = exp(scale q k^T - lse) over the seen pairs and
// delta_i = sum_c d_o_i[c] o_i[c] (which is sum_j P_ij dP_ij):
//     dP = d_o v^T,   dS = P (dP - delta) scale,   dq = dS k,   dk = dS^T q,   dv = P^T d_o,
// dk and dv of a shared head summed over its query heads.  Two passes form P and dP each: a sum over keys gives dq, a sum over
// queries gives dk and dv.  One pass would save two of the seven products and add dq up by atomics, in an order
// that changes from run to run.
//
// Query pass: as in the forward, 32 queries to a wavefront, the seen key tiles staged in LDS.  It also forms delta.
// Key pass: 32 keys to a wavefront, 128 of one head to a workgroup, which walks the tiles of the queries that see any of them,
// head after head of the group.  Ordinary keys are seen from `window` positions on, the sinks from all later ones: their
// tiles are cut into parts of about an ordinary tile's work, whose sums a small kernel adds up in their order.
// P and dS are rounded to the storage type as operands (bf16: half a step of 2^-8); all sums are fp32.
#include "lasad_window.h"

namespace lasad {

namespace {

constexpr int kThreads = 256, kTile = 128;               // queries (keys) of a workgroup

template <typename T, typename O, int D>
__global__ void __launch_bounds__(kThreads)
window_dq_kernel(WindowArgs a)
{
    typedef Mat<T> M;
    typedef typename M::F F;
    constexpr int KT = sizeof(T) == 2 ? 64 : 32, LD = D + M::PAD, KB = KT / 32, DB = D / 32, NF = D / M::KF;
    constexpr int N = KT * D / M::VEC / kThreads, PPR = D / M::VEC;
    __shared__ __align__(16) T tile[2][2][KT * LD];
    __shared__ int infinite[2];                          // number of the last tile in this half whose keys are not all finite

    const int qt = (a.n + kTile - 1) / kTile;
    const int64_t id = xcd_run(blockIdx.x, (int64_t)qt * a.B * a.Hq);
    if (id >= (int64_t)qt * a.B * a.Hq) return;
    const int i0 = (int)(id % qt) * kTile;
    const int bh = (int)(id / qt), b = bh / a.Hq, h = bh % a.Hq, hk = h / (a.Hq / a.Hk);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int iq = i0 + 32 * wave + col, p = a.start_pos + iq;
    const int p0 = a.start_pos + i0 + 32 * wave, p1 = p0 + 31;
    const int last = min(i0 + kTile, a.n) - 1;
    const int keys = valid_keys(a, b);
    const int hi = min(a.start_pos + last, keys - 1), lo = max(0, a.start_pos + i0 - a.window + 1);
    const T *kp = (const T *)a.k + (int64_t)b * a.lk.stride_b + (int64_t)hk * a.lk.stride_h;
    const T *vp = (const T *)a.v + (int64_t)b * a.lv.stride_b + (int64_t)hk * a.lv.stride_h;

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
        delta += __shfl_xor(delta, 32);
        if (on) {
            lse2 = a.lse[(int64_t)bh * a.n + iq] * kLog2e;
            if (half == 0) a.delta[(int64_t)bh * a.n + iq] = delta;
        }
    }
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zeros16();
    const float scale2 = a.scale * kLog2e;

    const int first = lo / KT, sink_tiles = min((min(a.sinks, hi + 1) + KT - 1) / KT, first);
    const int tiles = hi < 0 ? 0 : sink_tiles + max(0, hi / KT - first + 1);
    uint4 kr[N], vr[N];
    const auto at = [&](int t) { return (t < sink_tiles ? t : first + t - sink_tiles) * KT; };
    const auto load = [&](int j0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * kThreads, j = j0 + c / PPR;
            kr[i] = vr[i] = make_uint4(0, 0, 0, 0);
            if (j <= hi && (j >= lo || j < a.sinks)) {
                kr[i] = *(const uint4 *)(kp + (int64_t)j * a.lk.stride_n + (c % PPR) * M::VEC);
                vr[i] = *(const uint4 *)(vp + (int64_t)j * a.lv.stride_n + (c % PPR) * M::VEC);
            }
        }
    };
    const auto store = [&](int t) {
        if (!sees_all(a, keys, a.start_pos + i0, a.start_pos + last, at(t), at(t) + KT - 1)) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < N; ++i) bad |= make_finite<T>(kr[i]);
            if (bad) infinite[t & 1] = t;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * kThreads, at = (c / PPR) * LD + (c % PPR) * M::VEC;
            *(uint4 *)(tile[t & 1][0] + at) = kr[i];
            *(uint4 *)(tile[t & 1][1] + at) = vr[i];
        }
    };
    if (threadIdx.x < 2) infinite[threadIdx.x] = -1;
    if (tiles > 0) load(at(0));
    __syncthreads();
    if (tiles > 0) store(0);
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
        const int j0 = at(t);
        if (t + 1 < tiles) load(at(t + 1));
        if (!sees_none(a, keys, p0, p1, j0, j0 + KT - 1)) {
            const T *kt = tile[t & 1][0], *vt = tile[t & 1][1];
            const bool all = sees_all(a, keys, p0, p1, j0, j0 + KT - 1);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                f32x16 s = zeros16(), dp = zeros16();
#pragma unroll
                for (int f = 0; f < NF; ++f) s = M::mma(M::row(kt + (kb * 32 + col) * LD, f, half), q[f], s);
#pragma unroll
                for (int f = 0; f < NF; ++f) dp = M::mma(M::row(vt + (kb * 32 + col) * LD, f, half), g[f], dp);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(s[i], scale2, -lse2)) * (dp[i] - delta);
                    s[i] = all || sees(a, keys, p, j0 + kb * 32 + block_row(i, half)) ? x : 0.f;
                }
#pragma unroll
                for (int gr = 0; gr < M::GROUPS; ++gr) {
                    const F ds = M::pack(s, gr);
#pragma unroll
                    for (int d = 0; d < DB; ++d) acc[d] = M::mma(M::column(kt + kb * 32 * LD, LD, d * 32, gr, lane), ds, acc[d]);
                }
            }
            if (infinite[t & 1] == t) {                  // (a seen key that is not finite: so is the row's gradient)
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
        if (t + 1 < tiles) store(t + 1);
        __syncthreads();
    }
    if (iq >= a.n) return;
    O *dq = (O *)a.dq + (int64_t)b * a.ldq.stride_b + (int64_t)iq * a.ldq.stride_n + (int64_t)h * a.ldq.stride_h;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            store4(dq + d * 32 + 8 * r + 4 * half, acc[d][4 * r] * a.scale, acc[d][4 * r + 1] * a.scale, acc[d][4 * r + 2] * a.scale,
                   acc[d][4 * r + 3] * a.scale);
}

// Workgroups: first the sinks' key tiles, part after part, then the others.
template <typename T, typename O, int D>
__global__ void __launch_bounds__(kThreads)
window_dkv_kernel(WindowArgs a)
{
    typedef Mat<T> M;
    typedef typename M::F F;
    constexpr int QT = sizeof(T) == 2 ? 64 : 32, LD = D + M::PAD, QB = QT / 32, DB = D / 32, NF = D / M::KF;
    constexpr int N = QT * D / M::VEC / kThreads, PPR = D / M::VEC;
    __shared__ __align__(16) T tile[2][2][QT * LD];
    __shared__ int infinite[2];                          // number of the last step in this half whose rows are not all finite
    __shared__ __align__(16) float stat[2][2][QT];       // lse (in powers of two) and delta of a tile's queries

    const int kt = (a.m + kTile - 1) / kTile;
    const int units = a.sink_tiles * a.sink_parts + kt - a.sink_tiles;      // workgroups of a key head
    const int64_t id = xcd_run(blockIdx.x, (int64_t)units * a.B * a.Hk);
    if (id >= (int64_t)units * a.B * a.Hk) return;
    const int unit = (int)(id % units), bh = (int)(id / units), b = bh / a.Hk, hk = bh % a.Hk, G = a.Hq / a.Hk;
    const bool sink = unit < a.sink_tiles * a.sink_parts;
    const int kti = sink ? unit / a.sink_parts : unit - a.sink_tiles * a.sink_parts + a.sink_tiles;
    const int part = sink ? unit % a.sink_parts : 0, parts = sink ? a.sink_parts : 1;
    const int j0 = kti * kTile;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
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
    int i_next = 0, h_next = 0;                          // tile (of the share) and head that are loaded next
    const auto load = [&]() {
        const int i0 = (t_first + i_next) * QT;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * kThreads, iq = i0 + c / PPR;
            qr[i] = gr[i] = make_uint4(0, 0, 0, 0);
            if (iq < a.n) {
                qr[i] = *(const uint4 *)(qp + (int64_t)iq * a.lq.stride_n + h_next * a.lq.stride_h + (c % PPR) * M::VEC);
                gr[i] = *(const uint4 *)(gp + (int64_t)iq * a.ldo.stride_n + h_next * a.ldo.stride_h + (c % PPR) * M::VEC);
            }
        }
        if (threadIdx.x < 2 * QT) {
            const int iq = i0 + threadIdx.x % QT;
            const float *x = threadIdx.x < QT ? a.lse : a.delta;
            sr = iq < a.n ? x[stat0 + (int64_t)h_next * a.n + iq] : threadIdx.x < QT ? INFINITY : 0.f;
        }
        if (++i_next == t_count) { i_next = 0; ++h_next; }
    };
    const auto store = [&](int t) {                      // step t, whose loads came last
        const int buf = t & 1, p0 = a.start_pos + (t_first + t % t_count) * QT;
        if (!sees_all(a, keys, p0, p0 + QT - 1, j0, j0 + kTile - 1)) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                bad |= make_finite<T>(qr[i]);
                bad |= make_finite<T>(gr[i]);
            }
            if (bad) infinite[buf] = t;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * kThreads, at = (c / PPR) * LD + (c % PPR) * M::VEC;
            *(uint4 *)(tile[buf][0] + at) = qr[i];
            *(uint4 *)(tile[buf][1] + at) = gr[i];
        }
        if (threadIdx.x < 2 * QT) stat[buf][threadIdx.x / QT][threadIdx.x % QT] = threadIdx.x < QT ? sr * kLog2e : sr;
    };
    if (threadIdx.x < 2) infinite[threadIdx.x] = -1;
    if (steps > 0) load();
    __syncthreads();
    if (steps > 0) store(0);
    __syncthreads();
    int ti = 0, hi = 0;                                  // tile and head of the present step
    for (int t = 0; t < steps; ++t) {
        const int p0 = a.start_pos + (t_first + ti) * QT, p1 = p0 + QT - 1;
        if (t + 1 < steps) load();
        if (!sees_none(a, keys, p0, p1, w0, w1)) {
            const T *qt = tile[t & 1][0], *gt = tile[t & 1][1];
            const bool all = sees_all(a, keys, p0, p1, w0, w1);
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                f32x16 s = zeros16(), dp = zeros16();
#pragma unroll
                for (int f = 0; f < NF; ++f) s = M::mma(M::row(qt + (qb * 32 + col) * LD, f, half), k[f], s);
#pragma unroll
                for (int f = 0; f < NF; ++f) dp = M::mma(M::row(gt + (qb * 32 + col) * LD, f, half), v[f], dp);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float4 ls = *(const float4 *)(stat[t & 1][0] + qb * 32 + 8 * r + 4 * half);
                    const float4 de = *(const float4 *)(stat[t & 1][1] + qb * 32 + 8 * r + 4 * half);
                    const float lsx[4] = {ls.x, ls.y, ls.z, ls.w}, dex[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = 4 * r + e;
                        const bool on = all || sees(a, keys, p0 + qb * 32 + block_row(i, half), jk);
                        const float pr = on ? __builtin_amdgcn_exp2f(fmaf(s[i], scale2, -lsx[e])) : 0.f;
                        dp[i] = on ? pr * (dp[i] - dex[e]) : 0.f;
                        s[i] = pr;
                    }
                }
#pragma unroll
                for (int g = 0; g < M::GROUPS; ++g) {
                    const F pf = M::pack(s, g), df = M::pack(dp, g);
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        dv[d] = M::mma(M::column(gt + qb * 32 * LD, LD, d * 32, g, lane), pf, dv[d]);
                        dk[d] = M::mma(M::column(qt + qb * 32 * LD, LD, d * 32, g, lane), df, dk[d]);
                    }
                }
            }
            if (infinite[t & 1] == t) {                  // (a query that is not finite: so are the gradients of all keys it sees)
                for (int p = p0; p < min(p0 + QT, a.start_pos + a.n); ++p) {
                    const int64_t iq = p - a.start_pos;
                    const bool on = sees(a, keys, p, jk), bad = row_infinite<T, D>(qp + iq * a.lq.stride_n + hi * a.lq.stride_h, lane);
                    add_infinite<T, DB>(gp + iq * a.ldo.stride_n + hi * a.ldo.stride_h, on, half, dv);
                    if (bad && on) {
#pragma unroll
                        for (int d = 0; d < DB; ++d)
#pragma unroll
                            for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = NAN;
                    }
                }
            }
        }
        if (++ti == t_count) { ti = 0; ++hi; }
        if (t + 1 < steps) store(t + 1);
        __syncthreads();
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
    O *dkp = (O *)a.dk + (int64_t)b * a.ldk.stride_b + (int64_t)jk * a.ldk.stride_n + (int64_t)hk * a.ldk.stride_h;
    O *dvp = (O *)a.dv + (int64_t)b * a.ldv.stride_b + (int64_t)jk * a.ldv.stride_n + (int64_t)hk * a.ldv.stride_h;
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
    const int64_t total = (int64_t)a.B * a.Hk * a.sink_tiles * 2 * kTile * q;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (id >= total) return;
    const int c = (int)(id % q) * 4;
    const int row = (int)(id / q % kTile), which = (int)(id / q / kTile % 2);
    const int64_t tile = id / q / kTile / 2;             // (b, hk, sink tile)
    const int j = (int)(tile % a.sink_tiles) * kTile + row;
    if (j >= a.m) return;
    const int bh = (int)(tile / a.sink_tiles), b = bh / a.Hk, hk = bh % a.Hk;
    const float *p = a.parts + (tile * a.sink_parts * 2 + which) * kTile * a.d + (int64_t)row * a.d + c;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < a.sink_parts; ++i) {
        const float4 x = *(const float4 *)(p + (int64_t)i * 2 * kTile * a.d);
        s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
    }
    const lasad_layout_t &l = which ? a.ldv : a.ldk;
    const float f = which ? 1.f : a.scale;
    O *out = (O *)(which ? a.dv : a.dk) + (int64_t)b * l.stride_b + (int64_t)j * l.stride_n + (int64_t)hk * l.stride_h + c;
    store4(out, s.x * f, s.y * f, s.z * f, s.w * f);
}

// Key tiles with sinks and the parts they are cut into: a part walks about as many queries as an ordinary tile has.
// (None where the sinks' tiles alone are workgroups enough: at most 1024 parts in all, which bounds the workspace.)
void plan(int64_t heads, int n, int m, int window, int sinks, int &tiles, int &parts)
{
    const int64_t ordinary = (int64_t)window + kTile;
    tiles = (int)(((int64_t)(sinks < m ? sinks : m) + kTile - 1) / kTile);
    const int64_t want = (n + ordinary - 1) / ordinary, most = tiles > 0 ? 1024 / (heads * tiles) : 1;
    parts = (int)(want > most ? most : want);
    parts = parts < 1 ? 1 : parts > 64 ? 64 : parts;
}

size_t delta_bytes(int B, int Hq, int n) { return ((size_t)B * Hq * n * sizeof(float) + 255) / 256 * 256; }

}  // namespace

size_t window_backward_bytes(int B, int Hq, int Hk, int d, int n, int m, int window, int sinks)
{
    int tiles, parts;
    plan((int64_t)B * Hk, n, m, window, sinks, tiles, parts);
    return delta_bytes(B, Hq, n) + (parts > 1 ? (size_t)B * Hk * tiles * parts * 2 * kTile * d * sizeof(float) : 0);
}

hipError_t launch_window_backward(WindowArgs &a, void *workspace, hipStream_t s)
{
    a.delta = (float *)workspace;
    a.parts = (float *)((char *)workspace + delta_bytes(a.B, a.Hq, a.n));
    plan((int64_t)a.B * a.Hk, a.n, a.m, a.window, a.sinks, a.sink_tiles, a.sink_parts);
    const int64_t q_total = (int64_t)((a.n + kTile - 1) / kTile) * a.B * a.Hq;
    if (q_total > 0) {
#define LASAD_WQ(T, O, D) window_dq_kernel<T, O, D><<<dim3(xcd_grid(q_total)), dim3(kThreads), 0, s>>>(a)
        LASAD_WINDOW_DISPATCH(LASAD_WQ);
#undef LASAD_WQ
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int units = a.sink_tiles * a.sink_parts + (a.m + kTile - 1) / kTile - a.sink_tiles;
    const int64_t k_total = (int64_t)units * a.B * a.Hk;
    if (k_total == 0) return hipSuccess;
#define LASAD_WK(T, O, D) window_dkv_kernel<T, O, D><<<dim3(xcd_grid(k_total)), dim3(kThreads), 0, s>>>(a)
    LASAD_WINDOW_DISPATCH(LASAD_WK);
#undef LASAD_WK
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.sink_tiles > 0 && a.sink_parts > 1) {
        const int64_t total = (int64_t)a.B * a.Hk * a.sink_tiles * 2 * kTile * (a.d / 4);
        const dim3 grid((unsigned)((total + kThreads - 1) / kThreads));
        if (a.out_dtype == LASAD_BF16) window_sink_sum_kernel<uint16_t><<<grid, dim3(kThreads), 0, s>>>(a);
        else window_sink_sum_kernel<float><<<grid, dim3(kThreads), 0, s>>>(a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace lasad
