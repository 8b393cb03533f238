// Attention with a window and sinks, forward: o = softmax(scale q k^T over the seen keys) v, and the logarithm of the sum.
//
// One pass over the keys with the running maximum m and sum l of every query (in powers of two: exp(x) = 2^(x log2 e)):
//     m' = max(m, max_j s_j),  l' = l 2^(m - m') + sum_j 2^(s_j - m'),  o' = o 2^(m - m') + sum_j 2^(s_j - m') v_j.
// A wavefront has 32 queries, a workgroup 128 of one head; it walks the key tiles that any of them sees (the sinks' first,
// then those of the window), staged in LDS twice, the next tile's loads in flight over the products of the present one.
// Sums are fp32; the only rounding between q, k, v and o is that of 2^(s - m) to the storage type as the second product's
// operand (bf16: half a step of 2^-8, of terms of one sign; l is added up from the unrounded ones).
#include "lasad_window.h"

namespace lasad {

namespace {

constexpr int kThreads = 256, kQueries = 128;

// Rows j0 .. j0 + KT - 1 of one head's keys or values, a thread's 16-byte pieces; what no query of the workgroup may see is 0
// (so that what lies there cannot reach a sum as 0 * NaN).
template <typename T, int D, int KT, int N>
__device__ inline void load_tile(uint4 (&r)[N], const T *base, int64_t stride_n, int j0, int lo, int hi, int sinks)
{
    constexpr int PPR = D / Mat<T>::VEC;                 // pieces of a row
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = threadIdx.x + i * kThreads, j = j0 + c / PPR;
        r[i] = make_uint4(0, 0, 0, 0);
        if (j <= hi && (j >= lo || j < sinks)) r[i] = *(const uint4 *)(base + (int64_t)j * stride_n + (c % PPR) * Mat<T>::VEC);
    }
}

template <typename T, int D, int KT, int N>
__device__ inline void store_tile(const uint4 (&r)[N], T *lds)
{
    constexpr int PPR = D / Mat<T>::VEC, LD = D + Mat<T>::PAD;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = threadIdx.x + i * kThreads;
        *(uint4 *)(lds + (c / PPR) * LD + (c % PPR) * Mat<T>::VEC) = r[i];
    }
}

template <typename T, typename O, int D>
__global__ void __launch_bounds__(kThreads)
window_forward_kernel(WindowArgs a)
{
    typedef Mat<T> M;
    typedef typename M::F F;
    constexpr int KT = sizeof(T) == 2 ? 64 : 32, LD = D + M::PAD, KB = KT / 32, DB = D / 32, NF = D / M::KF;
    constexpr int N = KT * D / M::VEC / kThreads;        // a thread's pieces of a tile
    static_assert(N >= 1, "a tile has at least one piece for every thread");
    __shared__ __align__(16) T tile[2][2][KT * LD];
    __shared__ int infinite[2];                          // number of the last tile in this half whose values are not all finite

    const int qt = (a.n + kQueries - 1) / kQueries;
    const int64_t id = xcd_run(blockIdx.x, (int64_t)qt * a.B * a.Hq);
    if (id >= (int64_t)qt * a.B * a.Hq) return;
    const int i0 = (int)(id % qt) * kQueries;
    const int bh = (int)(id / qt), b = bh / a.Hq, h = bh % a.Hq, hk = h / (a.Hq / a.Hk);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int iq = i0 + 32 * wave + col, p = a.start_pos + iq;       // this lane's query
    const int p0 = a.start_pos + i0 + 32 * wave, p1 = p0 + 31;       // the wavefront's
    const int last = min(i0 + kQueries, a.n) - 1;                    // the workgroup's last query
    const int keys = valid_keys(a, b);
    const int hi = min(a.start_pos + last, keys - 1), lo = max(0, a.start_pos + i0 - a.window + 1);
    const T *kp = (const T *)a.k + (int64_t)b * a.lk.stride_b + (int64_t)hk * a.lk.stride_h;
    const T *vp = (const T *)a.v + (int64_t)b * a.lv.stride_b + (int64_t)hk * a.lv.stride_h;

    F q[NF];
    {
        const T *qp = (const T *)a.q + (int64_t)b * a.lq.stride_b + (int64_t)iq * a.lq.stride_n + (int64_t)h * a.lq.stride_h;
#pragma unroll
        for (int f = 0; f < NF; ++f) q[f] = iq < a.n ? M::row(qp, f, half) : M::zero();
    }
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zeros16();
    float m = -INFINITY, l = 0.f;
    const float scale2 = a.scale * kLog2e;

    // key tiles: those of the sinks before the window's, then the window's
    const int first = lo / KT, sink_tiles = min((min(a.sinks, hi + 1) + KT - 1) / KT, first);
    const int tiles = hi < 0 ? 0 : sink_tiles + max(0, hi / KT - first + 1);
    uint4 kr[N], vr[N];
    const auto at = [&](int t) { return (t < sink_tiles ? t : first + t - sink_tiles) * KT; };
    const auto load = [&](int t) {
        load_tile<T, D, KT>(kr, kp, a.lk.stride_n, at(t), lo, hi, a.sinks);
        load_tile<T, D, KT>(vr, vp, a.lv.stride_n, at(t), lo, hi, a.sinks);
    };
    const auto store = [&](int t) {
        if (!sees_all(a, keys, a.start_pos + i0, a.start_pos + last, at(t), at(t) + KT - 1)) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < N; ++i) bad |= make_finite<T>(vr[i]);
            if (bad) infinite[t & 1] = t;
        }
        store_tile<T, D, KT>(kr, tile[t & 1][0]);
        store_tile<T, D, KT>(vr, tile[t & 1][1]);
    };
    if (threadIdx.x < 2) infinite[threadIdx.x] = -1;
    if (tiles > 0) load(0);
    __syncthreads();
    if (tiles > 0) store(0);
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
        const int j0 = at(t);
        const T *kt = tile[t & 1][0], *vt = tile[t & 1][1];
        if (t + 1 < tiles) load(t + 1);
        if (!sees_none(a, keys, p0, p1, j0, j0 + KT - 1)) {
            f32x16 s[KB];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                s[kb] = zeros16();
#pragma unroll
                for (int f = 0; f < NF; ++f) s[kb] = M::mma(M::row(kt + (kb * 32 + col) * LD, f, half), q[f], s[kb]);
            }
            if (!sees_all(a, keys, p0, p1, j0, j0 + KT - 1)) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[kb][i] = sees(a, keys, p, j0 + kb * 32 + block_row(i, half)) ? s[kb][i] : -INFINITY;
            }
            float top = s[0][0];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m1 = fmaxf(m, top * scale2);
            const float use = m1 == -INFINITY ? 0.f : m1;            // (nothing seen yet: every term is 2^-inf)
            const float fade = __builtin_amdgcn_exp2f(m - use);
            m = m1;
            float sum = 0.f;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[kb][i] = __builtin_amdgcn_exp2f(fmaf(s[kb][i], scale2, -use));
                    sum += s[kb][i];
                }
            l = fmaf(l, fade, sum);
            if (__any(fade != 1.f)) {
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[d][i] *= fade;
            }
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int g = 0; g < M::GROUPS; ++g) {
                    const F pf = M::pack(s[kb], g);
#pragma unroll
                    for (int d = 0; d < DB; ++d) acc[d] = M::mma(M::column(vt + kb * 32 * LD, LD, d * 32, g, lane), pf, acc[d]);
                }
            if (infinite[t & 1] == t) {
                for (int j = j0; j < min(j0 + KT, keys); ++j) add_infinite<T, DB>(vp + (int64_t)j * a.lv.stride_n, sees(a, keys, p, j), half, acc);
            }
        }
        if (t + 1 < tiles) store(t + 1);
        __syncthreads();
    }
    l += __shfl_xor(l, 32);                              // (each half of the wavefront added up its own rows)
    if (iq >= a.n) return;
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    O *op = (O *)a.o + (int64_t)b * a.lo.stride_b + (int64_t)iq * a.lo.stride_n + (int64_t)h * a.lo.stride_h;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            store4(op + d * 32 + 8 * g + 4 * half, acc[d][4 * g] * inv, acc[d][4 * g + 1] * inv, acc[d][4 * g + 2] * inv, acc[d][4 * g + 3] * inv);
    if (a.lse && half == 0) a.lse[(int64_t)bh * a.n + iq] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace

hipError_t launch_window_forward(const WindowArgs &a, hipStream_t s)
{
    const int64_t total = (int64_t)((a.n + kQueries - 1) / kQueries) * a.B * a.Hq;
    if (total == 0) return hipSuccess;
#define LASAD_WF(T, O, D) window_forward_kernel<T, O, D><<<dim3(xcd_grid(total)), dim3(kThreads), 0, s>>>(a)
    LASAD_WINDOW_DISPATCH(LASAD_WF);
#undef LASAD_WF
    return hipGetLastError();
}

}  // namespace lasad
