// The key pass of the window attention's backward, bf16 (lasad_window_backward.hip has the formulas and the order of the work).
//
// A wavefront has 16 keys and takes 32 queries at a time, in products of 16 x 16: k, v, the sums of dk and dv and a block's P and dS are
// 48 registers of d = 64 where 32 keys in products of 32 x 32 have 96, so that four wavefronts fit a SIMD instead of two and hide each
// other's chains of products, exponentials and products.  Queries and d_o are then read from LDS twice as often, which has room for it once
// no two lanes meet in a bank (`first_row`).
//
// Measured, bf16, d = 64: 512 heads of 576 tokens, window 144 75 us (32 keys a wavefront 104); 2 x 8 key heads, each shared by three, of
// 4096 tokens, window 1024, 16 sinks 150 us, 610 TFLOP/s of the pairs that are seen (155), matrix cores busy for 30 % of the time, LDS
// for 39, vector units for 43; d = 128, 60 x 6 key heads of 48 tokens 15 us (29).  Bank conflicts cost 3 to 5 %, a rolled loop over a
// tile's blocks 3, eight wavefronts to a workgroup (128 keys) 10 % in the first case.
#include "lasad_window.h"

namespace lasad {

namespace {

constexpr int kThreads = 256, kTile = kWindowKeyTile;    // keys of a workgroup
static_assert(kTile == 16 * (kThreads / 64), "16 keys to a wavefront");

// x of lane L of each 16
template <int L>
__device__ inline float of_row(int x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0x150 + L, 0xf, 0xf, true));
}

// One block of 32 queries (positions from pb on, rows of qt and gt, their -lse / scale and -delta) for a wavefront's 16 keys.
template <int D>
__device__ inline void dkv_block(const WindowArgs &a, const Frag (&k)[D / 32], const Frag (&v)[D / 32], const uint16_t *qt, const uint16_t *gt,
                                   const float *shift, const float *delta, int pb, int keys, int w0, const Edge &edge, float scale2, int lane,
                                   f32x4v (&dk)[D / 16], f32x4v (&dv)[D / 16])
{
    typedef Mat<uint16_t> M;
    constexpr int LD = D + M::PAD, NF = D / 32, NC = D / 16;
    const int quad = lane >> 4, col = lane & 15;
    const int own = first_row(quad), row = first_row(col >> 2) + 4 * (col & 3);
    // (lanes 0 .. 7 of 16 have -lse / scale of the 16 lanes' eight queries, 8 .. 15 -delta; one read instead of four)
    const int held = __float_as_int(((col < 8 ? shift : delta))[16 * ((col >> 2) & 1) + own + 4 * (col & 3)]);
    f32x4v s[2], dp[2];
    s[0] = f32x4v{of_row<0>(held), of_row<1>(held), of_row<2>(held), of_row<3>(held)};
    s[1] = f32x4v{of_row<4>(held), of_row<5>(held), of_row<6>(held), of_row<7>(held)};
    dp[0] = f32x4v{of_row<8>(held), of_row<9>(held), of_row<10>(held), of_row<11>(held)};
    dp[1] = f32x4v{of_row<12>(held), of_row<13>(held), of_row<14>(held), of_row<15>(held)};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            s[t] = mfma16(M::piece(qt + (16 * t + row) * LD + channel<D>(f, quad)), k[f], s[t]);
            dp[t] = mfma16(M::piece(gt + (16 * t + row) * LD + channel<D>(f, quad)), v[f], dp[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[t][i] = __builtin_amdgcn_exp2f(s[t][i] * scale2);
            dp[t][i] *= s[t][i];
        }
    if (pb < w0 + 15 || w0 + 15 >= keys || pb + 31 - w0 >= a.window) {
        const int hi = edge.hi - pb - own, lo = edge.lo - pb - own;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (16 * t + 4 * i > hi || 16 * t + 4 * i < lo) s[t][i] = dp[t][i] = 0.f;
    }
    Frag pf, df;
    pf.u = make_uint4(pack2(s[0][0], s[0][1]), pack2(s[0][2], s[0][3]), pack2(s[1][0], s[1][1]), pack2(s[1][2], s[1][3]));
    df.u = make_uint4(pack2(dp[0][0], dp[0][1]), pack2(dp[0][2], dp[0][3]), pack2(dp[1][0], dp[1][1]), pack2(dp[1][2], dp[1][3]));
    const int at = (own + 4 * (col >> 2)) * LD + 4 * (col & 3);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        Frag x, y;
        x.h[0] = tr_read(gt + at + 16 * c);
        x.h[1] = tr_read(gt + at + 16 * LD + 16 * c);
        dv[c] = mfma16(x, pf, dv[c]);
        y.h[0] = tr_read(qt + at + 16 * c);
        y.h[1] = tr_read(qt + at + 16 * LD + 16 * c);
        dk[c] = mfma16(y, df, dk[c]);
    }
}

// Workgroups: first the sinks' key tiles, part after part, then the others.
template <typename O, int D>
__global__ void __launch_bounds__(kThreads, D <= 64 ? 4 : 2)
window_dkv_bf16_kernel(WindowArgs a)
{
    typedef uint16_t T;
    typedef Mat<T> M;
    typedef Frag F;
    constexpr int QT = 64, LD = D + M::PAD, QB = QT / 32, NC = D / 16, NF = D / 32;
    constexpr int PPR = D / 8, RPP = kThreads / PPR, N = QT / RPP;
    __shared__ __align__(16) T tile[2][2][QT * LD];
    __shared__ __align__(16) float stat[2][2][QT];       // -lse / scale and -delta of a tile's queries
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
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, quad = lane >> 4, col = lane & 15;
    const int jk = j0 + 16 * wave + col;                             // this lane's key
    const int w0 = j0 + 16 * wave, w1 = w0 + 15;                     // the wavefront's
    // (keys behind the last query are nobody's; a tile's rows behind it have lse = inf, so that P is 0 for every finite key)
    const int keys = min(valid_keys(a, b), a.start_pos + a.n);

    F k[NF], v[NF];
    {
        const T *kp = (const T *)a.k + (int64_t)b * a.lk.stride_b + (int64_t)jk * a.lk.stride_n + (int64_t)hk * a.lk.stride_h;
        const T *vp = (const T *)a.v + (int64_t)b * a.lv.stride_b + (int64_t)jk * a.lv.stride_n + (int64_t)hk * a.lv.stride_h;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            k[f] = jk < keys ? M::piece(kp + channel<D>(f, quad)) : M::zero();
            v[f] = jk < keys ? M::piece(vp + channel<D>(f, quad)) : M::zero();
        }
    }
    f32x4v dk[NC], dv[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) dk[c] = dv[c] = f32x4v{0.f, 0.f, 0.f, 0.f};
    const float scale2 = a.scale * kLog2e, inv_scale = 1.0f / a.scale;
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
        if (threadIdx.x < 2 * QT) stat[buf][threadIdx.x / QT][threadIdx.x % QT] = threadIdx.x < QT ? -sr * inv_scale : -sr;
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
                    const T *row = gp + iq * a.ldo.stride_n + h * a.ldo.stride_h;
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float x = as_float<T>(row[16 * c + 4 * quad + i]);
                            if (on && !(fabsf(x) < INFINITY)) dv[c][i] += x;
                            if (on && bad) dk[c][i] = dv[c][i] = NAN;
                        }
                }
            }
    }
    if (parts > 1) {                                     // (whole tiles, rows past the last key included)
        float *out = a.parts + (((int64_t)bh * a.sink_tiles * a.sink_parts + unit) * 2 * kTile + 16 * wave + col) * D + 4 * quad;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            store4(out + 16 * c, dk[c][0], dk[c][1], dk[c][2], dk[c][3]);
            store4(out + (int64_t)kTile * D + 16 * c, dv[c][0], dv[c][1], dv[c][2], dv[c][3]);
        }
        return;
    }
    if (jk >= a.m) return;
    O *dkp = (O *)a.dk + (int64_t)b * a.ldk.stride_b + (int64_t)jk * a.ldk.stride_n + (int64_t)hk * a.ldk.stride_h + 4 * quad;
    O *dvp = (O *)a.dv + (int64_t)b * a.ldv.stride_b + (int64_t)jk * a.ldv.stride_n + (int64_t)hk * a.ldv.stride_h + 4 * quad;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        store4(dkp + 16 * c, dk[c][0] * a.scale, dk[c][1] * a.scale, dk[c][2] * a.scale, dk[c][3] * a.scale);
        store4(dvp + 16 * c, dv[c][0], dv[c][1], dv[c][2], dv[c][3]);
    }
}

}  // namespace

hipError_t launch_window_dkv_bf16(const WindowArgs &a, hipStream_t s)
{
    const dim3 grid(launch_grid((int64_t)a.B * a.Hk, a.sink_tiles * a.sink_parts + (a.m + kTile - 1) / kTile - a.sink_tiles));
#define LASAD_WK(O, D) window_dkv_bf16_kernel<O, D><<<grid, dim3(kThreads), 0, s>>>(a)
    if (a.out_dtype == LASAD_BF16) {
        if (a.d == 32) LASAD_WK(uint16_t, 32); else if (a.d == 64) LASAD_WK(uint16_t, 64); else LASAD_WK(uint16_t, 128);
    } else {
        if (a.d == 32) LASAD_WK(float, 32); else if (a.d == 64) LASAD_WK(float, 64); else LASAD_WK(float, 128);
    }
#undef LASAD_WK
    return hipGetLastError();
}

}  // namespace lasad
