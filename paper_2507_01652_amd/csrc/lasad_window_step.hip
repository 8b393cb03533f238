// Attention with a window and sinks for one token of every batch row, against a cache that goes round:
//     o = sum over the seen keys j of softmax_j(scale q . k_j) v_j,   seen: j <= pos, pos - j < window or j < sinks.
// Key j lies in cache row j < sinks ? j : sinks + (j - sinks) mod (cap - sinks); the call's own key and value come from its
// arguments and are written to their row by the same launch.
//
// Bound by memory: the seen rows of k and v are read once for up to four query heads that share them; more than four are dealt out over
// workgroups of four, each of which reads them (64 rows, 8 key heads, 1040 keys: 24 query heads 23.6 us, 32 25.8, 40 48.4, 64 47.9).  A row is
// read by d / 8 lanes (fp32: d / 4) with one 16-byte load, so a wavefront takes 64 / lanes rows at a time, four such steps of k and v in flight.
// A group of lanes keeps maximum, sum and output of its rows for every query head of the group; they are joined over the
// groups by cross-lane exchange, over the wavefronts in LDS, and, where few heads have many rows, over `splits` workgroups
// by a second kernel.
//
// Measured, bf16, d = 64: 64 rows, 24 heads over 8, 1040 keys (116 MB) 23 us, 5.0 TB/s; 2 rows of 16 heads, 16448 keys (135 MB)
// 22 us, 6.1 TB/s (part of it cached), and 3.8 for the join; one row of 12 heads, 129 keys 4.1 us, which is a launch and two
// memory latencies.  A large copy reaches 4.94 TB/s.
#include "lasad_attention.h"
#include "lasad_mfma_util.h"

namespace lasad {

namespace {

constexpr int kThreads = 256, kWaves = 4;                // of the join
constexpr float kLog2e = 1.4426950408889634f;

template <int BF16, int VEC>
__device__ inline void unpack(const uint4 w, float (&f)[VEC])
{
    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (BF16) {
            f[2 * e] = __uint_as_float(ww[e] << 16);
            f[(2 * e + 1) % VEC] = __uint_as_float(ww[e] & 0xffff0000u);
        } else {
            f[e] = __uint_as_float(ww[e]);
        }
    }
}

template <int CTRL>
__device__ inline float dpp_add(float x)
{
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
// Sum over the LPT lanes (4 to 32, aligned) of a row, in every one of them.
template <int LPT>
__device__ inline float row_sum(float x)
{
    x = dpp_add<0xB1>(x);
    x = dpp_add<0x4E>(x);
    if (LPT >= 8) x = dpp_add<0x141>(x);
    if (LPT >= 16) x = dpp_add<0x140>(x);
    if (LPT >= 32) x += __shfl_xor(x, 16);
    return x;
}

// x of the lanes that hold the same channels (lane % LPT) combined, in every one of them.  The rotations by 4 and 8 lanes are inside 16.
template <int LPT, typename Op>
__device__ inline float over_slots(float x, Op op)
{
    if (LPT <= 4) x = op(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x124, 0xf, 0xf, true)));
    if (LPT <= 8) x = op(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xf, 0xf, true)));
    if (LPT <= 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// What a batch row at position `pos` sees: keys 0 .. far - 1, then near .. pos; false: the row is inactive.
struct Seen {
    int far, near, count;              // count: both together
    int near_row, ring;                // cache row (counted behind the sinks) of the first near key that is no sink
    int own_row;                       // cache row of the call's own key
};
__device__ inline bool seen_rows(const WindowStepArgs &a, int pos, Seen &s)
{
    s.ring = a.cap - a.sinks;
    if (pos < 0 || (pos >= a.cap && s.ring < a.window)) return false;
    s.near = max(0, pos - a.window + 1);
    s.far = min(a.sinks, s.near);
    s.count = s.far + pos - s.near + 1;
    s.near_row = (max(s.near, a.sinks) - a.sinks) % s.ring;
    s.own_row = pos < a.sinks ? pos : a.sinks + (pos - a.sinks) % s.ring;
    return true;
}
// cache row of seen key t (0 .. count - 1)
__device__ inline int cache_row(const WindowStepArgs &a, const Seen &s, int t)
{
    const int j = t < s.far ? t : s.near + t - s.far;
    int r = s.near_row + j - max(s.near, a.sinks);
    if (r >= s.ring) r -= s.ring;
    return j < a.sinks ? j : a.sinks + r;
}

// Workgroup: one key head of one batch row (blockIdx.x), one chunk of at most GC of its query heads (y), one split (z).
template <int BF16, int OBF16, int D, int GC, int WAVES>
__global__ void __launch_bounds__(WAVES * 64)
window_step_kernel(WindowStepArgs a)
{
    constexpr int VEC = BF16 ? 8 : 4, LPT = D / VEC, TPW = 64 / LPT, UNROLL = 4, ELT = BF16 ? 2 : 4;
    const int bh = blockIdx.x, b = bh / a.Hk, hk = bh - b * a.Hk, G = a.Hq / a.Hk, g0 = blockIdx.y * GC;
    const int pos = a.pos_rows ? a.pos_rows[b] : a.pos;
    Seen s;
    if (!seen_rows(a, pos, s)) return;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, piece = lane % LPT, slot = lane / LPT;

    const char *k_row = (const char *)a.k + ((int64_t)bh * D + piece * VEC) * ELT;
    const char *v_row = (const char *)a.v + ((int64_t)bh * D + piece * VEC) * ELT;
    const int64_t cache = ((int64_t)bh * a.cap * D + piece * VEC) * ELT;
    const char *kc = (const char *)a.k_cache + cache, *vc = (const char *)a.v_cache + cache;
    float q[GC][VEC];
#pragma unroll
    for (int g = 0; g < GC; ++g) {
        const int h = hk * G + min(g0 + g, G - 1);
        unpack<BF16, VEC>(*(const uint4 *)((const char *)a.q + (((int64_t)b * a.Hq + h) * D + piece * VEC) * ELT), q[g]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) q[g][e] *= a.scale * kLog2e;
    }
    // this split's keys; its share in whole steps of the workgroup
    constexpr int STEP = WAVES * UNROLL * TPW;
    const int share = ((s.count + a.splits - 1) / a.splits + STEP - 1) / STEP * STEP;
    const int t0 = min(s.count, (int)blockIdx.z * share), t1 = min(s.count, t0 + share);
    // (the own row's old contents are not read by this call: its key comes from the arguments)
    if (blockIdx.z == 0 && blockIdx.y == 0 && wave == 0 && slot < 2) {
        char *dst = (char *)(slot ? a.v_cache : a.k_cache) + cache + (int64_t)s.own_row * D * ELT;
        *(uint4 *)dst = *(const uint4 *)(slot ? v_row : k_row);
    }

    float m[GC], l[GC], acc[GC][VEC];
#pragma unroll
    for (int g = 0; g < GC; ++g) {
        m[g] = -INFINITY;
        l[g] = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[g][e] = 0.f;
    }
    for (int base = t0 + wave * UNROLL * TPW; base < t1; base += STEP) {
        uint4 kw[UNROLL], vw[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int t = min(base + u * TPW + slot, t1 - 1);
            const int64_t off = (int64_t)cache_row(a, s, t) * D * ELT;
            const bool own = t == s.count - 1;
            kw[u] = *(const uint4 *)(own ? k_row : kc + off);
            vw[u] = *(const uint4 *)(own ? v_row : vc + off);
        }
        float x[UNROLL][GC];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float kf[VEC];
            unpack<BF16, VEC>(kw[u], kf);
            const bool on = base + u * TPW + slot < t1;
#pragma unroll
            for (int g = 0; g < GC; ++g) {
                float d = 0.f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) d = fmaf(q[g][e], kf[e], d);
                d = row_sum<LPT>(d);
                x[u][g] = on ? d : -INFINITY;
            }
        }
#pragma unroll
        for (int g = 0; g < GC; ++g) {
            float top = m[g];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) top = fmaxf(top, x[u][g]);
            const float use = top == -INFINITY ? 0.f : top;
            const float fade = __builtin_amdgcn_exp2f(m[g] - use);
            m[g] = top;
            l[g] *= fade;
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[g][e] *= fade;
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                x[u][g] = __builtin_amdgcn_exp2f(x[u][g] - use);
                l[g] += x[u][g];
            }
        }
        // (lanes behind the last key hold that key's value once more; their weight is 0, and 0 times an infinity would be NaN)
        if (base + UNROLL * TPW > t1) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
                if (base + u * TPW + slot >= t1) vw[u] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float vf[VEC];
            unpack<BF16, VEC>(vw[u], vf);
#pragma unroll
            for (int g = 0; g < GC; ++g)
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[g][e] = fmaf(x[u][g], vf[e], acc[g][e]);
        }
    }

    // join the groups of lanes, then the wavefronts
    __shared__ float red[WAVES][GC][D + 2];
#pragma unroll
    for (int g = 0; g < GC; ++g) {
        const auto add = [](float x, float y) { return x + y; };
        const float top = over_slots<LPT>(m[g], [](float x, float y) { return fmaxf(x, y); });
        const float f = __builtin_amdgcn_exp2f(m[g] - (top == -INFINITY ? 0.f : top));
        l[g] = over_slots<LPT>(l[g] * f, add);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float x = over_slots<LPT>(acc[g][e] * f, add);
            if (slot == 0) red[wave][g][piece * VEC + e] = x;
        }
        if (lane == 0) {
            red[wave][g][D] = top;
            red[wave][g][D + 1] = l[g];
        }
    }
    __syncthreads();
    for (int i = tid; i < GC * D; i += WAVES * 64) {
        const int g = i / D, c = i % D;
        if (g0 + g >= G) continue;
        float top = red[0][g][D];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, red[w][g][D]);
        const float use = top == -INFINITY ? 0.f : top;
        float sum = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(red[w][g][D] - use);
            sum = fmaf(red[w][g][D + 1], f, sum);
            o = fmaf(red[w][g][c], f, o);
        }
        const int64_t row = (int64_t)b * a.Hq + hk * G + g0 + g;
        if (a.splits > 1) {
            float *p = a.parts + (row * a.splits + blockIdx.z) * (D + 2);
            p[c] = o;
            if (c == 0) { p[D] = top; p[D + 1] = sum; }
        } else if (OBF16) {
            ((uint16_t *)a.o)[row * D + c] = float_to_bf16_bits(o / sum);
        } else {
            ((float *)a.o)[row * D + c] = o / sum;
        }
    }
}

// The splits (at most 64) of a query head joined: a wavefront takes every fourth of them, a lane one channel (two of 128).
template <int OBF16, int D>
__global__ void __launch_bounds__(kThreads)
window_join_kernel(WindowStepArgs a)
{
    constexpr int C = D < 64 ? 1 : D / 64, UNROLL = 4;
    __shared__ float factor[64], part[kWaves][D];
    const int64_t row = blockIdx.x;
    const int b = (int)(row / a.Hq), wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    Seen s;
    if (!seen_rows(a, a.pos_rows ? a.pos_rows[b] : a.pos, s)) return;
    const float *p = a.parts + row * a.splits * (D + 2);
    const int ch = lane % (D < 64 ? D : 64);
    // (every wavefront forms the splits' factors for itself: no wait before the sums' loads)
    const float m = lane < a.splits ? p[lane * (D + 2) + D] : -INFINITY, l = lane < a.splits ? p[lane * (D + 2) + D + 1] : 0.f;
    float top = m;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) top = fmaxf(top, __shfl_xor(top, off));
    const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
    float sum = l * f;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) sum += __shfl_xor(sum, off);
    if (wave == 0) factor[lane] = f;
    float o[C] = {};
    __syncthreads();
    for (int i = wave; i < a.splits; i += kWaves * UNROLL) {
        float x[UNROLL][C];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int c = 0; c < C; ++c) x[u][c] = p[min(i + u * kWaves, a.splits - 1) * (D + 2) + c * 64 + ch];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int c = 0; c < C; ++c) o[c] = i + u * kWaves < a.splits ? fmaf(x[u][c], factor[i + u * kWaves], o[c]) : o[c];
    }
#pragma unroll
    for (int c = 0; c < C; ++c) part[wave][c * 64 + ch] = o[c];
    __syncthreads();
    if (threadIdx.x >= D) return;
    const int e = threadIdx.x;
    const float r = ((part[0][e] + part[1][e]) + (part[2][e] + part[3][e])) / sum;
    if (OBF16) ((uint16_t *)a.o)[row * D + e] = float_to_bf16_bits(r);
    else ((float *)a.o)[row * D + e] = r;
}

template <int BF16, int OBF16, int D, int WAVES>
void launch_step(const WindowStepArgs &a, hipStream_t s)
{
    const int G = a.Hq / a.Hk;
    const unsigned x = (unsigned)(a.B * a.Hk), z = (unsigned)a.splits;
#define LASAD_WS(GC) window_step_kernel<BF16, OBF16, D, GC, WAVES><<<dim3(x, (G + GC - 1) / GC, z), dim3(WAVES * 64), 0, s>>>(a)
    if (G == 1) LASAD_WS(1);
    else if (G == 2) LASAD_WS(2);
    else if (G == 3) LASAD_WS(3);
    else LASAD_WS(4);
#undef LASAD_WS
}

template <int BF16, int OBF16, int D>
hipError_t launch(const WindowStepArgs &a, hipStream_t s)
{
    if ((int64_t)a.B * a.Hk * a.splits <= 256) launch_step<BF16, OBF16, D, 8>(a, s);
    else launch_step<BF16, OBF16, D, 4>(a, s);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) {
        window_join_kernel<OBF16, D><<<dim3((unsigned)(a.B * a.Hq)), dim3(kThreads), 0, s>>>(a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

// Splits of a call whose rows see up to `seen` keys: enough workgroups for the chip's 256 units twice, planned with at least 256 keys each.
// (A workgroup takes whole steps of 128 to 512 keys of bf16, so that the last splits may have none: 43 of 64 have some for 8 heads of 16448
// keys.)  The join's launch costs as much as 700 keys more in a workgroup (12 heads, us without and with: 1024 keys 7.1 and 8.0, 2048 10.5 and
// 8.1, 16384 73 and 13), and two splits of many heads gain nothing (256 heads of 4096 keys 40 and 43).
int window_step_splits(int B, int Hk, int64_t seen)
{
    const int64_t heads = (int64_t)B * Hk;
    int64_t n = 512 / heads;
    if (seen < 1536 || n < 4) return 1;
    if (n > seen / 256) n = seen / 256;
    return (int)(n > 64 ? 64 : n);
}

size_t window_step_bytes(int B, int Hq, int d, int splits)
{
    return splits > 1 ? (size_t)B * Hq * splits * (d + 2) * sizeof(float) : 0;
}

hipError_t launch_window_step(const WindowStepArgs &a, hipStream_t s)
{
    if (a.io_dtype == LASAD_BF16) {
        if (a.out_dtype == LASAD_BF16) return a.d == 32 ? launch<1, 1, 32>(a, s) : a.d == 64 ? launch<1, 1, 64>(a, s) : launch<1, 1, 128>(a, s);
        return a.d == 32 ? launch<1, 0, 32>(a, s) : a.d == 64 ? launch<1, 0, 64>(a, s) : launch<1, 0, 128>(a, s);
    }
    return a.d == 32 ? launch<0, 0, 32>(a, s) : a.d == 64 ? launch<0, 0, 64>(a, s) : launch<0, 0, 128>(a, s);
}

}  // namespace lasad
