// The query pass of the window attention's backward, bf16 (lasad_window_backward.hip has the formulas).
//
// A wavefront has 16 queries and takes 32 keys at a time, in products of 16 x 16, as the key pass does and for the same reasons: four
// wavefronts a SIMD instead of three, no two lanes in a bank, and 64 queries a workgroup, which leaves fewer units without one.
//
// Measured, bf16, d = 64: 512 heads of 576 tokens, window 144 70 us (32 queries a wavefront, 128 a workgroup: 75): 424 MB, half of it
// k and v again for the next tile, at 6.1 TB/s; all of a head's queries launched together 65, but 111 in the next; 2 x 24 heads over 8 of 4096 tokens, window 1024, 16 sinks 105 us, 650 TFLOP/s of the pairs that are seen (104);
// 12 heads of 2048 tokens, window 256 14 us (18), d = 128 22 (29).
#include "lasad_window.h"

namespace lasad {

namespace {

constexpr int kThreads = 256, kTile = 64;                // queries of a workgroup, 16 to a wavefront

// One block of 32 keys (from j0 on, rows of kt and vt) for a wavefront's 16 queries: dS, and its product with k.  s0, d0: -lse / scale
// and -delta.
template <int D>
__device__ inline void dq_block(const Frag (&q)[D / 32], const Frag (&g)[D / 32], const uint16_t *kt, const uint16_t *vt, int j0, const Range &range,
                                const Edge &edge, float scale2, const f32x4v &s0, const f32x4v &d0, int lane, f32x4v (&acc)[D / 16])
{
    typedef Mat<uint16_t> M;
    constexpr int LD = D + M::PAD, NF = D / 32, NC = D / 16;
    const int quad = lane >> 4, col = lane & 15;
    const int own = first_row(quad), row = first_row(col >> 2) + 4 * (col & 3);
    f32x4v s[2], dp[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            s[t] = mfma16(M::piece(kt + (16 * t + row) * LD + channel<D>(f, quad)), q[f], f ? s[t] : s0);
            dp[t] = mfma16(M::piece(vt + (16 * t + row) * LD + channel<D>(f, quad)), g[f], f ? dp[t] : d0);
        }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) dp[t][i] *= __builtin_amdgcn_exp2f(s[t][i] * scale2);
    if (range.top_edge(j0 + 31) || range.bottom_edge(j0)) {
        const int hi = edge.hi - j0 - own, lo = edge.lo - j0 - own, first = edge.first - j0 - own;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (16 * t + 4 * i > hi || (16 * t + 4 * i < lo && 16 * t + 4 * i >= first)) dp[t][i] = 0.f;
    }
    Frag ds;
    ds.u = make_uint4(pack2(dp[0][0], dp[0][1]), pack2(dp[0][2], dp[0][3]), pack2(dp[1][0], dp[1][1]), pack2(dp[1][2], dp[1][3]));
    const int at = (own + 4 * (col >> 2)) * LD + 4 * (col & 3);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        Frag x;
        x.h[0] = tr_read(kt + at + 16 * c);
        x.h[1] = tr_read(kt + at + 16 * LD + 16 * c);
        acc[c] = mfma16(x, ds, acc[c]);
    }
}

template <typename O, int D>
__global__ void __launch_bounds__(kThreads, D <= 64 ? 4 : 2)
window_dq_bf16_kernel(WindowArgs a)
{
    typedef uint16_t T;
    typedef Mat<T> M;
    typedef Frag F;
    constexpr int KT = 64, LD = D + M::PAD, NC = D / 16, NF = D / 32;
    constexpr int PPR = D / 8, RPP = kThreads / PPR, N = KT / RPP;
    __shared__ __align__(16) T tile[2][2][KT * LD];
    __shared__ int infinite;                             // whether a key that was taken out of a tile was not finite

    const int qt = (a.n + kTile - 1) / kTile;
    const Place place = launch_place(blockIdx.x, a.B * a.Hq, qt);
    if (place.head < 0) return;
    const int i0 = (qt - 1 - place.unit) * kTile;        // (the first queries see the fewest keys: last)
    const int bh = place.head, b = bh / a.Hq, h = bh % a.Hq, hk = h / (a.Hq / a.Hk);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, quad = lane >> 4, col = lane & 15;
    const int iq = i0 + 16 * wave + col, p = a.start_pos + iq;
    const int p0 = a.start_pos + i0 + 16 * wave, p1 = p0 + 15;
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
            q[f] = on ? M::piece(qp + channel<D>(f, quad)) : M::zero();
            g[f] = on ? M::piece(gp + channel<D>(f, quad)) : M::zero();
            if (on) delta += M::dot(g[f], M::piece(op + channel<D>(f, quad)));
        }
        delta += __shfl_xor(delta, 16);
        delta = both_halves_sum(delta);
        if (on) {
            lse2 = a.lse[(int64_t)bh * a.n + iq] * kLog2e;
            if (quad == 0) a.delta[(int64_t)bh * a.n + iq] = delta;
        }
    }
    f32x4v acc[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] = f32x4v{0.f, 0.f, 0.f, 0.f};
    const float shift = -lse2 / scale2;
    const f32x4v s0 = {shift, shift, shift, shift}, d0 = {-delta, -delta, -delta, -delta};
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
                dq_block<D>(q, g, kt + b * LD, vt + b * LD, j0 + b, mine, edge, scale2, s0, d0, lane, acc);
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
                    for (int c = 0; c < NC; ++c) acc[c] = f32x4v{NAN, NAN, NAN, NAN};
                }
            }
        }
    }
    if (iq >= a.n) return;
    O *dq = (O *)a.dq + (int64_t)b * a.ldq.stride_b + (int64_t)iq * a.ldq.stride_n + (int64_t)h * a.ldq.stride_h + 4 * quad;
#pragma unroll
    for (int c = 0; c < NC; ++c) store4(dq + 16 * c, acc[c][0] * a.scale, acc[c][1] * a.scale, acc[c][2] * a.scale, acc[c][3] * a.scale);
}

}  // namespace

hipError_t launch_window_dq_bf16(const WindowArgs &a, hipStream_t s)
{
    const dim3 grid(launch_grid((int64_t)a.B * a.Hq, (a.n + kTile - 1) / kTile));
#define LASAD_WQ(O, D) window_dq_bf16_kernel<O, D><<<grid, dim3(kThreads), 0, s>>>(a)
    if (a.out_dtype == LASAD_BF16) {
        if (a.d == 32) LASAD_WQ(uint16_t, 32); else if (a.d == 64) LASAD_WQ(uint16_t, 64); else LASAD_WQ(uint16_t, 128);
    } else {
        if (a.d == 32) LASAD_WQ(float, 32); else if (a.d == 64) LASAD_WQ(float, 64); else LASAD_WQ(float, 128);
    }
#undef LASAD_WQ
    return hipGetLastError();
}

}  // namespace lasad
