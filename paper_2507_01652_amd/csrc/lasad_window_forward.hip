// Attention with a window and sinks, forward: o = softmax(scale q k^T over the seen keys) v, and the logarithm of the sum.
//
// One pass over the keys with the running maximum m and sum l of every query (in powers of two: exp(x) = 2^(x log2 e)):
//     m' = max(m, max_j s_j),  l' = l 2^(m - m') + sum_j 2^(s_j - m'),  o' = o 2^(m - m') + sum_j 2^(s_j - m') v_j.
// A wavefront has 32 queries, a workgroup 128 of one head; it walks the key tiles that any of them sees (the sinks' first,
// then those of the window), staged in LDS twice, the next tile's loads in flight over the products of the present one.
// Sums are fp32; the only rounding between q, k, v and o is that of 2^(s - m) to the storage type as the second product's
// operand (bf16: half a step of 2^-8, of terms of one sign; l is added up from the unrounded ones).
//
// Measured, bf16, d = 64, 4 x 24 heads of 4096 tokens, window 1024, 16 sinks: 142 us, 640 TFLOP/s of the pairs that are seen (91.4
// GFLOP; a product of 8192^3 reaches 1221).  No unit is full there: the vector units issue 62 % of the time (16 exponentials,
// 16 multiply-adds, 16 additions, 9 maxima, 8 conversions a block of 32 x 32, some 110 with the edges and addresses), the matrix cores
// are busy for 31 %, LDS for 32 %; a block is one chain of products, maximum, exponentials and products, 0.6 us for a wavefront
// alone, and four wavefronts a SIMD hide 60 % of it.  Timed without a part (us): tile loads and stores 114, exponentials 126,
// the second product 120.  512 heads of 576 tokens, window 144: 49 us for 260 MB, 5.2 TB/s, near the memory's rate.
// Took longer, in the first case's us: 64 queries a wavefront 181, eight wavefronts to a tile 155, all of a head's queries launched
// together 151, priorities of wavefronts 143 to 151.  Tiles loaded straight into LDS came to 138 before the rearrangement they need.
#include "lasad_window.h"

namespace lasad {

namespace {

constexpr int kThreads = 256, kQueries = 128;

// One block of 32 keys (from j0 on, scores s, values in the rows of vt) for a wavefront's queries: exponentials, products with v.
// Blocks are taken one after the other, not two at a time: with 16 scores a lane (and not 32) four wavefronts fit a SIMD, which hide
// each other's waits better than a longer run of independent operations does (4 x 4096 tokens of 24 heads: 156 us with two blocks and
// three wavefronts, 148 so; two tiles in a wavefront's registers, products beside exponentials: 245).
template <typename T, int D>
__device__ inline void forward_block(f32x16 s, const T *vt, int j0, const Range &range, const Edge &edge, float scale2, int lane, float &m, float &l,
                                     f32x16 (&acc)[D / 32])
{
    typedef Mat<T> M;
    constexpr int LD = D + M::PAD, DB = D / 32;
    const int half = lane >> 5;
    const bool top_edge = range.top_edge(j0 + 31), bottom_edge = range.bottom_edge(j0);
    if (top_edge || bottom_edge) hide(s, edge, j0, half, top_edge, bottom_edge, -INFINITY);
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    // m need not be the maximum, only near it: it is raised (and what was summed up rescaled) where a score passes it by 2^8,
    // which some query of 32 does in every tile when every new maximum counts, and hardly ever so
    top = both_halves_max(top) * scale2;
    if (__any(top > m + kSlack)) {
        const float m1 = top > m + kSlack ? top : m;
        const float fade = m == m1 ? 1.f : __builtin_amdgcn_exp2f(m - m1);
        m = m1;
        l *= fade;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] *= fade;
    }
    const float use = m == -INFINITY ? 0.f : m;          // (nothing seen yet: every term is 2^-inf)
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale2, -use));
        sum += s[i];
    }
    l += sum;
#pragma unroll
    for (int g = 0; g < M::GROUPS; ++g) {
        const typename M::F pf = M::pack(s, g);
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[d] = M::mma(M::column(vt, LD, d * 32, g, lane), pf, acc[d]);
    }
}

template <typename T, typename O, int D>
__global__ void __launch_bounds__(kThreads, D > 64 ? 2 : sizeof(T) == 2 ? 4 : 3)
window_forward_kernel(WindowArgs a)
{
    typedef Mat<T> M;
    typedef typename M::F F;
    constexpr int KT = sizeof(T) == 2 ? 64 : 32, LD = D + M::PAD, DB = D / 32, NF = D / M::KF;
    constexpr int PPR = D / M::VEC, RPP = kThreads / PPR, N = KT / RPP;
    static_assert(N >= 1, "a tile has at least one piece for every thread");
    __shared__ __align__(16) T tile[2][2][KT * LD];
    __shared__ int infinite;                             // whether a value that was taken out of a tile was not finite

    const int qt = (a.n + kQueries - 1) / kQueries;
    const Place place = launch_place(blockIdx.x, a.B * a.Hq, qt);
    if (place.head < 0) return;
    const int i0 = (qt - 1 - place.unit) * kQueries;     // (the first queries see the fewest keys: last)
    const int bh = place.head, b = bh / a.Hq, h = bh % a.Hq, hk = h / (a.Hq / a.Hk);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int iq = i0 + 32 * wave + col, p = a.start_pos + iq;       // this lane's query
    const int p0 = a.start_pos + i0 + 32 * wave, p1 = p0 + 31;       // the wavefront's
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
        for (int f = 0; f < NF; ++f) q[f] = iq < a.n ? M::row(qp, f, half) : M::zero();
    }
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zeros16();
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
            if (mine.some(j0 + b, j0 + b + 31)) {
                f32x16 s = zeros16();
#pragma unroll
                for (int f = 0; f < NF; ++f) s = M::mma(M::row(kt + (b + col) * LD, f, half), q[f], s);
                forward_block<T, D>(s, vt + b * LD, j0 + b, mine, edge, scale2, lane, m, l, acc);
            }
        if (t + 1 < tiles) store(j1, (t + 1) & 1);
        __syncthreads();
        j0 = j1;
    }
    l = both_halves_sum(l);                              // (each half of the wavefront added up its own rows)
    if (iq >= a.n) return;
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] *= inv;
    if (infinite) {
        int j0 = begin;
        for (int t = 0; t < tiles; ++t, j0 = next(j0)) {
            if (all.all(j0, j0 + KT - 1)) continue;      // (as it was)
            for (int j = j0; j < min(j0 + KT, keys); ++j) add_infinite<T, DB>(vp + (int64_t)j * a.lv.stride_n, sees(a, keys, p, j), half, acc);
        }
    }
    O *op = (O *)a.o + (int64_t)b * a.lo.stride_b + (int64_t)iq * a.lo.stride_n + (int64_t)h * a.lo.stride_h;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            store4(op + d * 32 + 8 * g + 4 * half, acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]);
    if (a.lse && half == 0) a.lse[(int64_t)bh * a.n + iq] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// For few queries: a workgroup has 32 of one head, and its four wavefronts take the blocks of keys in turn, each with its own
// maximum, sum and output, which are joined at the end.  Nothing is shared on the way: keys go from memory to the products' operands,
// values through the wavefront's own rows of LDS, without a barrier.
template <typename T, typename O, int D>
__global__ void __launch_bounds__(kThreads, D <= 64 ? 3 : 1)
window_forward_few_kernel(WindowArgs a)
{
    typedef Mat<T> M;
    typedef typename M::F F;
    constexpr int LD = D + M::PAD, DB = D / 32, NF = D / M::KF, PPR = D / M::VEC, RPW = 64 / PPR, N = 32 / RPW, W = kThreads / 64;
    constexpr int V_BYTES = W * 32 * LD * (int)sizeof(T), JOIN_BYTES = W * 32 * (D + 4) * 4;
    __shared__ __align__(16) char lds[V_BYTES > JOIN_BYTES ? V_BYTES : JOIN_BYTES];
    __shared__ float tops[W][32], sums[W][32];
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

    // blocks of keys: those of the sinks before the window's, then the window's
    const int first = lo / 32, sink_blocks = min((min(a.sinks, hi + 1) + 31) / 32, first);
    const int blocks = hi < 0 ? 0 : sink_blocks + max(0, hi / 32 - first + 1);
    const auto at = [&](int t) { return (t < sink_blocks ? t : first + t - sink_blocks) * 32; };
    T *vt = (T *)lds + wave * 32 * LD;
    F kr[NF];
    uint4 vr[N];
    const int row0 = lane / PPR, col0 = (lane % PPR) * M::VEC;
    const auto load = [&](int t) {                       // (rows behind the last one that is seen: that one)
        const int j0 = at(t);
        const T *kq = kp + (int64_t)min(j0 + col, hi) * a.lk.stride_n;
#pragma unroll
        for (int f = 0; f < NF; ++f) kr[f] = M::row(kq, f, half);
#pragma unroll
        for (int i = 0; i < N; ++i) vr[i] = *(const uint4 *)(vp + (int64_t)min(j0 + row0 + i * RPW, hi) * a.lv.stride_n + col0);
    };
    // (wavefronts with the same number share a SIMD: the first block, and with it an odd one, goes to another of them each time)
    const int turn = (wave + blockIdx.x) % W;
    if (turn < blocks) load(turn);
    F q[NF];
    {
        const T *qp = (const T *)a.q + (int64_t)b * a.lq.stride_b + (int64_t)min(iq, a.n - 1) * a.lq.stride_n + (int64_t)h * a.lq.stride_h;
#pragma unroll
        for (int f = 0; f < NF; ++f) q[f] = M::row(qp, f, half);
    }
    if (threadIdx.x == 0) infinite = 0;
    __syncthreads();
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zeros16();
    float m = -INFINITY, l = 0.f;
    for (int t = turn; t < blocks; t += W) {
        const int j0 = at(t);
        if (!range.all(j0, j0 + 31)) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int j = j0 + row0 + i * RPW;
                if (j > hi || (j < lo && j >= a.sinks)) vr[i] = make_uint4(0, 0, 0, 0);
                bad |= make_finite<T>(vr[i]);
            }
            if (bad) infinite = 1;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) *(uint4 *)(vt + (row0 + i * RPW) * LD + col0) = vr[i];
        f32x16 s = zeros16();
#pragma unroll
        for (int f = 0; f < NF; ++f) s = M::mma(kr[f], q[f], s);
        if (t + W < blocks) load(t + W);
        wave_lds_order();
        forward_block<T, D>(s, vt, j0, range, edge, scale2, lane, m, l, acc);
        wave_lds_order();
    }
    l = both_halves_sum(l);
    if (half == 0) { tops[wave][col] = m; sums[wave][col] = l; }
    __syncthreads();
    float top = tops[0][col];
#pragma unroll
    for (int w = 1; w < W; ++w) top = fmaxf(top, tops[w][col]);
    const float use = top == -INFINITY ? 0.f : top;
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) total = fmaf(sums[w][col], __builtin_amdgcn_exp2f(tops[w][col] - use), total);
    const float f = total == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - use) / total;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] *= f;
    if (infinite && wave == 0) {
        for (int t = 0; t < blocks; ++t) {
            if (range.all(at(t), at(t) + 31)) continue;  // (as it was)
            for (int j = at(t); j < min(at(t) + 32, keys); ++j) add_infinite<T, DB>(vp + (int64_t)j * a.lv.stride_n, sees(a, keys, p, j), half, acc);
        }
    }
    float *join = (float *)lds;                          // (all values have been read: the barrier above)
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(float4 *)(join + (wave * 32 + col) * (D + 4) + d * 32 + 8 * g + 4 * half) =
                make_float4(acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]);
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * D / 4; c += kThreads) {
        const int row = c / (D / 4), ch = c % (D / 4) * 4;
        if (i0 + row >= a.n) break;
        float4 s = *(const float4 *)(join + row * (D + 4) + ch);
#pragma unroll
        for (int w = 1; w < W; ++w) {
            const float4 x = *(const float4 *)(join + (w * 32 + row) * (D + 4) + ch);
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        store4((O *)a.o + (int64_t)b * a.lo.stride_b + (int64_t)(i0 + row) * a.lo.stride_n + (int64_t)h * a.lo.stride_h + ch, s.x, s.y, s.z, s.w);
    }
    if (a.lse && threadIdx.x < 32 && iq < a.n)
        a.lse[(int64_t)bh * a.n + iq] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
}

// Which kernel, by the number of workgroups that 128 queries each would make, heads counted in eights as they are dealt out.  Few: one
// of 32, whose wavefronts share out the keys, fills the chip's 256 units sooner, and pays for longer where the walk over the keys is long.
// us, few, 16 queries a wavefront, 32 and 128 a workgroup.  d = 64, window 256 of 2048 tokens: 96 workgroups 9.8 10.2 13.9, 256 16.1 13.1
// 14.7, 384 20.6 16.0 18.4, 640 29 22.9 23.4, 1024 43 31 28; all seen: 256 30 36 41, 384 39 38 44, 1024 92 68 54; window 32 of 256: 192 8.1 8.8
// 10.5, 256 10.4 9.1 10.6.  d = 32, window 256: 256 9.4 10.5 12.0, 384 13.0 12.5 14.3, 1024 24 22 21; all seen: 640 35 34 39.  d = 128, window
// 256: 64 12.3 13.8 19.4, 96 22 14 20, 384 63 23 27, 4096 643 207 201; all seen: 96 29 46 60, 192 70 51 59.  fp32, bound by its matrix rate:
// window 128 of 256 tokens, 12 heads, batch 4 (96) 16.7 and 27.5, 16 (384) 38.7 and 37.4.
enum Kernel { FEW, MIDDLING, MANY };
Kernel choose(const WindowArgs &a)
{
    const int64_t heads = (int64_t)a.B * a.Hq, groups = (heads < 8 ? heads : (heads + 7) / 8 * 8) * ((a.n + kQueries - 1) / kQueries);
    if (a.io_dtype == LASAD_F32) return groups < 384 ? FEW : MANY;
    const int64_t last = (int64_t)a.start_pos + a.n, seen = (int64_t)a.window + 64 < last ? (int64_t)a.window + 64 : last;
    const bool far = seen >= 1024;
    const int few = a.d == 32 ? (far ? 640 : 384) : a.d == 64 ? (far ? 320 : 200) : (far ? 128 : 72);
    return groups < few ? FEW : a.d == 128 || groups < 768 ? MIDDLING : MANY;
}

}  // namespace

int64_t window_forward_groups(const WindowArgs &a)
{
    const Kernel kernel = choose(a);
    const int64_t queries = kernel == FEW ? 32 : kernel == MIDDLING ? 64 : kQueries;
    return launch_groups((int64_t)a.B * a.Hq, (a.n + queries - 1) / queries);
}

hipError_t launch_window_forward(const WindowArgs &a, hipStream_t s)
{
    if (a.n == 0) return hipSuccess;
    const int64_t heads = (int64_t)a.B * a.Hq;
    const Kernel kernel = choose(a);
    if (kernel == FEW) {
        const dim3 grid(launch_grid(heads, (a.n + 31) / 32));
#define LASAD_WF(T, O, D) window_forward_few_kernel<T, O, D><<<grid, dim3(kThreads), 0, s>>>(a)
        LASAD_WINDOW_DISPATCH(LASAD_WF);
#undef LASAD_WF
        return hipGetLastError();
    }
    if (kernel == MIDDLING) return launch_window_forward_16(a, s);
    const dim3 grid(launch_grid(heads, (a.n + kQueries - 1) / kQueries));
#define LASAD_WF(T, O, D) window_forward_kernel<T, O, D><<<grid, dim3(kThreads), 0, s>>>(a)
    if (a.io_dtype == LASAD_F32) {
        if (a.d == 32) LASAD_WF(float, float, 32); else if (a.d == 64) LASAD_WF(float, float, 64); else LASAD_WF(float, float, 128);
    } else if (a.out_dtype == LASAD_BF16) {
        if (a.d == 32) LASAD_WF(uint16_t, uint16_t, 32); else LASAD_WF(uint16_t, uint16_t, 64);
    } else {
        if (a.d == 32) LASAD_WF(uint16_t, float, 32); else LASAD_WF(uint16_t, float, 64);
    }
#undef LASAD_WF
    return hipGetLastError();
}

}  // namespace lasad
