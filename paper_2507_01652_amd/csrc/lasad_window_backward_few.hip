// The backward of the window attention for few queries or keys (lasad_window_backward.hip has the formulas, the choice and what is for many):
// a workgroup has 32 queries (keys) of one head, and its four wavefronts take the blocks of keys (queries) in turn, each with sums of
// its own, which are added up at the end.  A block's rows go from memory to the first products' operands and, from the same registers,
// to the wavefront's own LDS, whose columns the last products read; no barrier before the end.
//
// Bound by latency: a call is one chain of loads and products a wavefront.  Measured, bf16, d = 64, query and key pass, us: 6 heads of 2048
// tokens, all seen, 26 and 28 (workgroups of 64: 33 and 51), 4 heads, window 256, 9.2 and 11.9 (10.6 and 12.9); fp32, 16 over 8 heads of
// 229 tokens, bound by its matrix rate: 16 and 30.
#include "lasad_window.h"

namespace lasad {

namespace {

constexpr int kThreads = 256, W = kThreads / 64;

// A wavefront's 32 x D sums to its part of `join`: row (query or key) col, fp32.
template <int D>
__device__ inline void put_sums(float *join, int wave, int col, int half, const f32x16 (&acc)[D / 32])
{
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(float4 *)(join + (wave * 32 + col) * (D + 4) + d * 32 + 8 * g + 4 * half) =
                make_float4(acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]);
}
// The wavefronts' sums of row `row` from channel `ch` on, in their order.
template <int D>
__device__ inline float4 added(const float *join, int row, int ch)
{
    float4 s = *(const float4 *)(join + row * (D + 4) + ch);
#pragma unroll
    for (int w = 1; w < W; ++w) {
        const float4 x = *(const float4 *)(join + (w * 32 + row) * (D + 4) + ch);
        s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
    }
    return s;
}

template <typename T, typename O, int D>
__global__ void __launch_bounds__(kThreads, D == 32 ? 3 : sizeof(T) == 2 && D == 64 ? 2 : 1)
window_dq_few_kernel(WindowArgs a)
{
    typedef Mat<T> M;
    typedef typename M::F F;
    constexpr int LD = D + M::PAD, DB = D / 32, NF = D / M::KF;
    constexpr int ROWS = W * 32 * LD * (int)sizeof(T), JOIN = W * 32 * (D + 4) * 4;
    __shared__ __align__(16) char lds[ROWS > JOIN ? ROWS : JOIN];
    __shared__ int infinite;

    const int qt = (a.n + 31) / 32;
    const Place place = launch_place(blockIdx.x, a.B * a.Hq, qt);
    if (place.head < 0) return;
    const int i0 = (qt - 1 - place.unit) * 32, bh = place.head, b = bh / a.Hq, h = bh % a.Hq, hk = h / (a.Hq / a.Hk);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int iq = i0 + col, p = a.start_pos + iq, p0 = a.start_pos + i0, p1 = a.start_pos + min(i0 + 32, a.n) - 1;
    const int keys = valid_keys(a, b);
    const int hi = min(p1, keys - 1), lo = max(0, p0 - a.window + 1);
    const T *kp = (const T *)a.k + (int64_t)b * a.lk.stride_b + (int64_t)hk * a.lk.stride_h;
    const T *vp = (const T *)a.v + (int64_t)b * a.lv.stride_b + (int64_t)hk * a.lv.stride_h;
    const float scale2 = a.scale * kLog2e;
    const Edge edge = query_edge(a, keys, p);
    const Range range(a, keys, p0, p1);
    const int first = lo / 32, sink_blocks = min((min(a.sinks, hi + 1) + 31) / 32, first);
    const int blocks = hi < 0 ? 0 : sink_blocks + max(0, hi / 32 - first + 1);
    const auto at = [&](int t) { return (t < sink_blocks ? t : first + t - sink_blocks) * 32; };
    F kr[NF], vr[NF];
    const auto load = [&](int t) {                       // (rows behind the last one that is seen: that one)
        const int64_t j = min(at(t) + col, hi);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            kr[f] = M::row(kp + j * a.lk.stride_n, f, half);
            vr[f] = M::row(vp + j * a.lv.stride_n, f, half);
        }
    };
    const int turn = (wave + blockIdx.x) % W;            // (as in the forward)
    if (turn < blocks) load(turn);
    F q[NF], g[NF];
    float delta = 0.f, lse2 = INFINITY;
    {
        const int64_t i = min(iq, a.n - 1);
        const T *qp = (const T *)a.q + (int64_t)b * a.lq.stride_b + i * a.lq.stride_n + (int64_t)h * a.lq.stride_h;
        const T *gp = (const T *)a.d_o + (int64_t)b * a.ldo.stride_b + i * a.ldo.stride_n + (int64_t)h * a.ldo.stride_h;
        const T *op = (const T *)a.o + (int64_t)b * a.lo.stride_b + i * a.lo.stride_n + (int64_t)h * a.lo.stride_h;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            q[f] = M::row(qp, f, half);
            g[f] = M::row(gp, f, half);
            delta += M::dot(g[f], M::row(op, f, half));
        }
        delta = both_halves_sum(delta);
        lse2 = a.lse[(int64_t)bh * a.n + i] * kLog2e;
        if (threadIdx.x < 32 && iq < a.n) a.delta[(int64_t)bh * a.n + iq] = delta;
    }
    if (threadIdx.x == 0) infinite = 0;
    __syncthreads();
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zeros16();
    T *kt = (T *)lds + wave * 32 * LD;
    for (int t = turn; t < blocks; t += W) {
        const int j0 = at(t);
        if (!range.all(j0, j0 + 31)) {
            bool bad = false;
            const int j = j0 + col;
            const bool unseen = j > hi || (j < lo && j >= a.sinks);
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                uint4 x = __builtin_bit_cast(uint4, kr[f]);
                if (unseen) x = make_uint4(0, 0, 0, 0);
                bad |= make_finite<T>(x);
                kr[f] = __builtin_bit_cast(F, x);
            }
            if (bad) infinite = 1;
        }
#pragma unroll
        for (int f = 0; f < NF; ++f) *(uint4 *)(kt + col * LD + f * M::KF + M::VEC * half) = __builtin_bit_cast(uint4, kr[f]);
        f32x16 s = zeros16(), dp = zeros16();
#pragma unroll
        for (int f = 0; f < NF; ++f) { s = M::mma(kr[f], q[f], s); dp = M::mma(vr[f], g[f], dp); }
        if (t + W < blocks) load(t + W);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale2, -lse2)) * (dp[i] - delta);
        const bool top_edge = range.top_edge(j0 + 31), bottom_edge = range.bottom_edge(j0);
        if (top_edge || bottom_edge) hide(s, edge, j0, half, top_edge, bottom_edge, 0.f);
        wave_lds_order();
#pragma unroll
        for (int r = 0; r < M::GROUPS; ++r) {
            const F ds = M::pack(s, r);
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[d] = M::mma(M::column(kt, LD, d * 32, r, lane), ds, acc[d]);
        }
        wave_lds_order();
    }
    __syncthreads();
    if (infinite && wave == 0) {                         // (a seen key that is not finite: so is the row's gradient)
        for (int t = 0; t < blocks; ++t) {
            if (range.all(at(t), at(t) + 31)) continue;  // (as it was)
            for (int j = at(t); j < min(at(t) + 32, keys); ++j) {
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
    put_sums<D>((float *)lds, wave, col, half, acc);
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * D / 4; c += kThreads) {
        const int row = c / (D / 4), ch = c % (D / 4) * 4;
        if (i0 + row >= a.n) break;
        const float4 s = added<D>((const float *)lds, row, ch);
        store4((O *)a.dq + (int64_t)b * a.ldq.stride_b + (int64_t)(i0 + row) * a.ldq.stride_n + (int64_t)h * a.ldq.stride_h + ch,
               s.x * a.scale, s.y * a.scale, s.z * a.scale, s.w * a.scale);
    }
}

template <typename T, typename O, int D>
__global__ void __launch_bounds__(kThreads, D == 32 ? 3 : sizeof(T) == 2 && D == 64 ? 2 : 1)
window_dkv_few_kernel(WindowArgs a)
{
    typedef Mat<T> M;
    typedef typename M::F F;
    constexpr int LD = D + M::PAD, DB = D / 32, NF = D / M::KF;
    constexpr int ROWS = W * 64 * LD * (int)sizeof(T), JOIN = W * 32 * (D + 4) * 4;
    __shared__ __align__(16) char lds[ROWS > JOIN ? ROWS : JOIN];
    __shared__ __align__(16) float stat[W][2][32];
    __shared__ int infinite;

    const int units = a.sink_tiles * a.sink_parts + (a.m + 31) / 32 - a.sink_tiles;
    const Place place = launch_place(blockIdx.x, a.B * a.Hk, units);
    if (place.head < 0) return;
    const int unit = place.unit, bh = place.head, b = bh / a.Hk, hk = bh % a.Hk, G = a.Hq / a.Hk;
    const bool sink = unit < a.sink_tiles * a.sink_parts;
    const int kti = sink ? unit / a.sink_parts : unit - a.sink_tiles * a.sink_parts + a.sink_tiles;
    const int part = sink ? unit % a.sink_parts : 0, parts = sink ? a.sink_parts : 1;
    const int j0 = kti * 32;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int jk = j0 + col, keys = min(valid_keys(a, b), a.start_pos + a.n);
    // (what lse is in the place where it enters: fp32 the exponential's multiply-add, bf16 the sums that the scores start from)
    const float scale2 = a.scale * kLog2e, lse_unit = sizeof(T) == 4 ? kLog2e : -1.0f / a.scale;
    const Edge edge = key_edge(a, keys, jk);

    // blocks of 32 queries that see any of the keys, and this part's share of them
    const int j1 = min(j0 + 32, keys) - 1;
    int q_lo = max(0, j0 - a.start_pos), q_hi = a.n - 1;
    if (j0 >= a.sinks) q_hi = (int)min((int64_t)q_hi, (int64_t)j1 + a.window - 1 - a.start_pos);
    const int t_lo = q_lo / 32;
    const int t_all = j1 < j0 || q_hi < q_lo ? 0 : q_hi / 32 - t_lo + 1;
    const int share = (t_all + parts - 1) / parts, t_first = t_lo + part * share;
    const int t_count = max(0, min(share, t_all - part * share)), steps = t_count * G;

    const T *qp = (const T *)a.q + (int64_t)b * a.lq.stride_b + (int64_t)hk * G * a.lq.stride_h;
    const T *gp = (const T *)a.d_o + (int64_t)b * a.ldo.stride_b + (int64_t)hk * G * a.ldo.stride_h;
    const float *statp = (half ? a.delta : a.lse) + ((int64_t)b * a.Hq + hk * G) * a.n;
    F qr[NF], gr[NF];
    float sr = 0.f;
    const auto load = [&](int t) {                       // step t: block t mod t_count of head t / t_count
        const int hd = t / t_count;
        const int64_t i = min((t_first + t - hd * t_count) * 32 + col, a.n - 1);
        const T *q0 = qp + i * a.lq.stride_n + (int64_t)hd * a.lq.stride_h, *g0 = gp + i * a.ldo.stride_n + (int64_t)hd * a.ldo.stride_h;
#pragma unroll
        for (int f = 0; f < NF; ++f) { qr[f] = M::row(q0, f, half); gr[f] = M::row(g0, f, half); }
        sr = statp[(int64_t)hd * a.n + i];
    };
    const int turn = (wave + blockIdx.x) % W;
    if (turn < steps) load(turn);
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
    if (threadIdx.x == 0) infinite = 0;
    __syncthreads();
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = dv[d] = zeros16();
    T *qt = (T *)lds + wave * 64 * LD, *gt = qt + 32 * LD;
    const auto whole = [&](int i0) { return i0 + 32 <= a.n && sees_all(a, keys, a.start_pos + i0, a.start_pos + i0 + 31, j0, j0 + 31); };
    for (int t = turn; t < steps; t += W) {
        const int i0 = (t_first + t % t_count) * 32, pb = a.start_pos + i0;
        if (!whole(i0)) {
            bool bad = false;
            const bool behind = i0 + col >= a.n;
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                uint4 x = __builtin_bit_cast(uint4, qr[f]), y = __builtin_bit_cast(uint4, gr[f]);
                if (behind) x = y = make_uint4(0, 0, 0, 0);
                bad |= make_finite<T>(x);
                bad |= make_finite<T>(y);
                qr[f] = __builtin_bit_cast(F, x);
                gr[f] = __builtin_bit_cast(F, y);
            }
            if (bad) infinite = 1;
            if (behind) sr = half ? 0.f : INFINITY;
        }
        stat[wave][half][col] = half ? -sr : sr * lse_unit;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            *(uint4 *)(qt + col * LD + f * M::KF + M::VEC * half) = __builtin_bit_cast(uint4, qr[f]);
            *(uint4 *)(gt + col * LD + f * M::KF + M::VEC * half) = __builtin_bit_cast(uint4, gr[f]);
        }
        wave_lds_order();
        f32x16 s = zeros16(), dp;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float4 y = *(const float4 *)(stat[wave][1] + 8 * r + 4 * half);
            dp[4 * r] = y.x; dp[4 * r + 1] = y.y; dp[4 * r + 2] = y.z; dp[4 * r + 3] = y.w;
            if constexpr (sizeof(T) == 2) {
                const float4 x = *(const float4 *)(stat[wave][0] + 8 * r + 4 * half);
                s[4 * r] = x.x; s[4 * r + 1] = x.y; s[4 * r + 2] = x.z; s[4 * r + 3] = x.w;
            }
        }
#pragma unroll
        for (int f = 0; f < NF; ++f) { s = M::mma(qr[f], k[f], s); dp = M::mma(gr[f], v[f], dp); }
        if (t + W < steps) load(t + W);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float lse2[4] = {};
            if constexpr (sizeof(T) == 4) {
                const float4 x = *(const float4 *)(stat[wave][0] + 8 * r + 4 * half);
                lse2[0] = x.x; lse2[1] = x.y; lse2[2] = x.z; lse2[3] = x.w;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = s[4 * r + i];
                s[4 * r + i] = __builtin_amdgcn_exp2f(sizeof(T) == 4 ? fmaf(x, scale2, -lse2[i]) : x * scale2);
                dp[4 * r + i] *= s[4 * r + i];
            }
        }
        const bool first_edge = pb < j0 + 31 || j0 + 31 >= keys, last_edge = pb + 31 - j0 >= a.window;
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
        wave_lds_order();
    }
    __syncthreads();
    if (infinite && wave == 0) {                         // (a query that is not finite: so are the gradients of all keys it sees)
        for (int t = 0; t < steps; ++t) {
            const int hd = t / t_count, i0 = (t_first + t - hd * t_count) * 32;
            if (whole(i0)) continue;                     // (as they were)
            for (int iq = i0; iq < min(i0 + 32, a.n); ++iq) {
                const bool on = sees(a, keys, a.start_pos + iq, jk);
                const bool bad = row_infinite<T, D>(qp + (int64_t)iq * a.lq.stride_n + (int64_t)hd * a.lq.stride_h, lane);
                add_infinite<T, DB>(gp + (int64_t)iq * a.ldo.stride_n + (int64_t)hd * a.ldo.stride_h, on, half, dv);
                if (bad && on) {
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = NAN;
                }
            }
        }
    }
    for (int which = 0; which < 2; ++which) {
        put_sums<D>((float *)lds, wave, col, half, which ? dv : dk);
        __syncthreads();
        const lasad_layout_t &l = which ? a.ldv : a.ldk;
        const float f = which ? 1.f : a.scale;
        for (int c = threadIdx.x; c < 32 * D / 4; c += kThreads) {
            const int row = c / (D / 4), ch = c % (D / 4) * 4;
            const float4 s = added<D>((const float *)lds, row, ch);
            if (parts > 1)                               // (whole tiles, rows past the last key included)
                *(float4 *)(a.parts + ((((int64_t)bh * a.sink_tiles * a.sink_parts + unit) * 2 + which) * 32 + row) * D + ch) = s;
            else if (j0 + row < a.m)
                store4((O *)(which ? a.dv : a.dk) + (int64_t)b * l.stride_b + (int64_t)(j0 + row) * l.stride_n + (int64_t)hk * l.stride_h + ch,
                       s.x * f, s.y * f, s.z * f, s.w * f);
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_window_dq_few(const WindowArgs &a, hipStream_t s)
{
    const dim3 grid(launch_grid((int64_t)a.B * a.Hq, (a.n + 31) / 32));
#define LASAD_WQ(T, O, D) window_dq_few_kernel<T, O, D><<<grid, dim3(kThreads), 0, s>>>(a)
    LASAD_WINDOW_DISPATCH(LASAD_WQ);
#undef LASAD_WQ
    return hipGetLastError();
}

hipError_t launch_window_dkv_few(const WindowArgs &a, hipStream_t s)
{
    const dim3 grid(launch_grid((int64_t)a.B * a.Hk, a.sink_tiles * a.sink_parts + (a.m + 31) / 32 - a.sink_tiles));
#define LASAD_WK(T, O, D) window_dkv_few_kernel<T, O, D><<<grid, dim3(kThreads), 0, s>>>(a)
    LASAD_WINDOW_DISPATCH(LASAD_WK);
#undef LASAD_WK
    return hipGetLastError();
}

}  // namespace lasad
