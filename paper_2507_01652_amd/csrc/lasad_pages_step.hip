// One token of every row over the paged 8-bit cache, in one launch: norms and rotation of its query heads and its key, key and value into their
// page, attention (lasad_pages_append.hip and lasad_pages_attend.hip have the formulas).
//
// A workgroup has a key head of a row, 16 of its query heads at a time, and all of its pages or a split of them; its wavefronts take pages in turn.
// A head's channels lie over the lanes as the first product wants them, so that every wavefront forms its queries for itself: sums over a head are
// sums over four lanes, the table of angles is the workgroup's.  The wavefront that has the last page forms the new key's and value's codes, which in
// that layout are just the bytes that it has to put into its registers of the page; it writes them to memory and goes on without reading them
// again, unless the page's scale had to grow.
//
// bf16 queries are two bf16 parts and so is P: what a step adds to o's error is far below o's own rounding.  Bound by memory where there is enough:
// 128 rows of 20 heads that see 24 to 4001 keys (767 MB) 151 us, 5.1 TB/s; 64 rows of 24 heads over 8, 1040 keys (58 MB) 15.2 us, 3.9; two rows of
// 16 heads, 16448 keys (67 MB) 14 in 16 parts and 4 for their join; one row of 12 heads 6.7, of which the launch, position and table take 2.3: the
// chain position, page, codes, norms, products, join.  With up to eight query heads a key head a tile holds copies of them (Columns): 16 columns for 3 heads would
// raise four times as many scores to powers (64 rows of 8 key heads, 1040 keys, in a graph: one to four heads each 16.6 us, without copies 17.0 to 17.2, with
// two 16.6; five to eight 16.7, without copies 17.1).
#include "lasad_heads.h"
#include "lasad_pages_codes.h"
#include "lasad_pages_tile.h"

namespace lasad {

namespace {

// A head's channels in a wavefront as they are loaded: page_channel(f, quad) .. + 7 of a lane.
template <typename T, int D>
struct RawHead {
    static constexpr int NF = D / 32, EACH = sizeof(T) / 2;
    uint4 w[NF][EACH];
    __device__ inline void load(const T *p, int quad)
    {
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < EACH; ++i) w[f][i] = ((const uint4 *)(p + page_channel<D>(f, quad)))[i];
    }
    __device__ inline void unpack(float (&y)[NF][8]) const
    {
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const uint32_t x[4] = {w[f][i].x, w[f][i].y, w[f][i].z, w[f][i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (sizeof(T) == 2) {
                        y[f][2 * e] = __uint_as_float(x[e] << 16);
                        y[f][2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
                    } else {
                        y[f][4 * i + e] = __uint_as_float(x[e]);
                    }
                }
            }
    }
};

// Its norm, weights (read where `weighted`) and rotation by the table cs.
template <int D>
__device__ inline void norm_and_turn(const AppendArgs &a, bool weighted, const RawHead<float, D> &w, const float2 *cs, int quad, float (&y)[D / 32][8])
{
    constexpr int NF = D / 32;
    if (a.norm) {
        float ss = 0.f;
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(y[f][e], y[f][e], ss);
        const float rstd = rsqrtf(quads_sum(ss) * (1.0f / D) + a.eps);
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[f][e] *= rstd;
        if (weighted) {
            float x[NF][8];
            w.unpack(x);
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int e = 0; e < 8; ++e) y[f][e] *= x[f][e];
        }
    }
    if (a.rope == LASAD_ROPE_NONE) return;
    if (a.pairing == LASAD_PAIR_ADJACENT) {
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 c = cs[page_channel<D>(f, quad) / 2 + i];
                const float p = y[f][2 * i], q = y[f][2 * i + 1];
                y[f][2 * i] = p * c.x - q * c.y;
                y[f][2 * i + 1] = p * c.y + q * c.x;
            }
        return;
    }
    // the other member of a channel's pair is `half` channels away: in a lane of another quad, or in another piece of this one
    const int span = a.rope == LASAD_ROPE_2D ? D / 2 : D, half = span / 2;
    float other[NF][8];
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (D == 128 && half == 64) other[f][e] = y[f ^ (NF / 2)][e];
            else other[f][e] = __shfl_xor(y[f][e], D == 32 ? 2 * half : half);
        }
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        const int ch = page_channel<D>(f, quad), in = ch % span;
        const float2 *c = cs + ch / span * half + in % half;
        const float sign = in < half ? -1.f : 1.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[f][e] = y[f][e] * c[e].x + other[f][e] * (sign * c[e].y);
    }
}

// The new key and value as they lie in a wavefront's registers of their page.
template <int D>
struct NewKey {
    uint32_t k[D / 16];                                  // codes of the lane's channels
    uint32_t v[D / 16];                                  // code of channel 16 c + lane % 16
    float k_scale, v_scale;
    bool grown;                                          // the page's earlier codes have changed

    // rk, rv: the key's channels and channel 16 c + lane % 16 of the value; w: the key's weights; k_old, v_old: the page's scales before
    template <typename T>
    __device__ inline void append(const AppendArgs &a, const float2 *cs, const RawHead<T, D> &rk, const T (&rv)[D / 16], const RawHead<float, D> &w, float k_old,
                                  float v_old, int hk, int pos, int page, int lane)
    {
        constexpr int NF = D / 32, NC = D / 16;
        const int quad = lane >> 4, col = lane & 15, slot = pos % kPage;
        const int64_t ph = (int64_t)page * a.pages.heads + hk;
        float y[NF][8], x[NC];
        rk.unpack(y);
#pragma unroll
        for (int c = 0; c < NC; ++c) x[c] = as_float<T>(rv[c]);
        norm_and_turn<D>(a, a.w[1] != nullptr, w, cs, quad, y);
        float k_most = 0.f, v_most = 0.f;
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int e = 0; e < 8; ++e) k_most = fmaxf(k_most, finite_size(y[f][e]));
#pragma unroll
        for (int c = 0; c < NC; ++c) v_most = fmaxf(v_most, finite_size(x[c]));
        v_most = fmaxf(v_most, dpp_move<0xB1>(v_most));
        v_most = fmaxf(v_most, dpp_move<0x4E>(v_most));
        v_most = fmaxf(v_most, dpp_move<0x141>(v_most));
        v_most = fmaxf(v_most, dpp_move<0x140>(v_most));
        uint8_t *kp = a.pages.k + ph * kPage * D, *vp = a.pages.v + ph * kPage * D;
        float k_less, v_less;
        k_scale = page_scale(quads_max(k_most), slot, k_old, k_less);
        v_scale = page_scale(v_most, slot, v_old, v_less);
        if (k_less < 1.f) shrink_page<D, false>(kp, slot, k_less, lane);
        if (v_less < 1.f) shrink_page<D, true>(vp, slot, v_less, lane);
        if (lane == 0) {
            a.pages.k_scale[ph] = k_scale;
            a.pages.v_scale[ph] = v_scale;
        }
        grown = k_less < 1.f || v_less < 1.f;
        const Divide k_by(k_scale), v_by(v_scale);
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < 2; ++i) k[2 * f + i] = code4(k_by(y[f][4 * i]), k_by(y[f][4 * i + 1]), k_by(y[f][4 * i + 2]), k_by(y[f][4 * i + 3]));
#pragma unroll
        for (int c = 0; c < NC; ++c) v[c] = code2(v_by(x[c]), 0.f, 0, false) & 0xffu;
        if (col == slot % 16) {
#pragma unroll
            for (int f = 0; f < NF; ++f) *(uint2 *)(kp + slot * D + page_channel<D>(f, quad)) = make_uint2(k[2 * f], k[2 * f + 1]);
        }
        if (quad == slot / 4 % 4) {
#pragma unroll
            for (int c = 0; c < NC; ++c) vp[(16 * c + col) * kPage + 16 * quad + slot / 16 * 4 + slot % 4] = (uint8_t)v[c];
        }
        if (grown) __threadfence_block();
    }

    // Into a page as it was before (or after).
    __device__ inline void put(PagePart<D> &t, int slot, int lane) const
    {
        const int quad = lane >> 4, col = lane & 15;
        const uint32_t shift = 8 * (slot % 4), keep = quad == slot / 4 % 4 ? ~(0xffu << shift) : ~0u;
        const int block = slot / 16;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int w = 0; w < D / 16; ++w) {
                constexpr int EACH = D == 32 ? 2 : 4;
                t.k[b][w / EACH][w % EACH] = b == block && col == slot % 16 ? k[w] : t.k[b][w / EACH][w % EACH];
            }
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int b = 0; b < 4; ++b) t.v[c][b] = b == block ? (t.v[c][b] & keep) | (v[c] << shift & ~keep) : t.v[c][b];
        t.k_scale = k_scale;
        t.v_scale = v_scale;
    }
};

// T: type of q, k and v.  NQ, NP: bf16 parts of a query and of P.  SHARE: copies of the query heads in a tile of 16 columns.
template <typename T, typename O, int D, int NQ, int NP, int SHARE, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, D == 128 ? 1 : D == 64 && (SHARE == 1 || sizeof(T) == 4) ? 2 : 3)
step_pages_kernel(AppendArgs a, AttendArgs g)
{
    constexpr int NF = D / 32, NC = D / 16, P = D / 2, EACH = 16 / SHARE;
    __shared__ __align__(16) float2 cs[P];
    __shared__ __align__(16) float red[WAVES][16][D + 4];
    const int heads = a.pages.heads, G = a.Hq / heads, hk = blockIdx.x % heads, split = blockIdx.y;
    PageRow row;
    if (!find_row(a.rows, a.pages, blockIdx.x / heads, 1, 1, 1, row)) return;
    const int b = row.b, pos = row.pos;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, quad = lane >> 4, col = lane & 15;
    const PageList list(pos, pos, g.window, g.sinks);
    const int step = g.splits * WAVES, begin = split * WAVES + wave;
    // Everything that the first page, the queries and the new key need is on its way before anything is waited for, what is needed first in front:
    // their norms and codes are formed while the page's codes come (weights and old scales loaded where they are used: 15.8 us for 64 rows, 15.2 so).
    Walk walk;
    walk.fill(a.pages, list, b, begin, step);
    RawHead<T, D> rq, rk;
    RawHead<float, D> wq, wk;
    T rv[NC];
    const T *queries = (const T *)a.q + ((int64_t)b * a.Hq + hk * G) * D;
    const bool owner = (list.count - 1) % step == begin;               // the wavefront that has the row's last page
    const auto load_queries = [&](int g0) {
        const int h = min(g0 + col % EACH, G - 1);
        rq.load(queries + h * D, quad);
        if (a.w[0]) wq.load(a.w[0] + (a.shared ? 0 : (hk * G + h) * D), quad);
    };
    int last = -1;
    float k_old = 0.f, v_old = 0.f;
    if (owner) {
        const int64_t at = ((int64_t)b * heads + hk) * D;
        rk.load((const T *)a.k + at, quad);
        if (a.w[1]) wk.load(a.w[1] + (a.shared ? 0 : hk * D), quad);
#pragma unroll
        for (int c = 0; c < NC; ++c) rv[c] = ((const T *)a.v)[at + 16 * c + col];
        const int entry = scalar_load(a.pages.table + b * a.pages.table_stride + list.number(list.count - 1));
        last = entry < a.pages.n_pages ? max(entry, -1) : -1;
        k_old = scalar_load(a.pages.k_scale + (int64_t)max(last, 0) * heads + hk);
        v_old = scalar_load(a.pages.v_scale + (int64_t)max(last, 0) * heads + hk);
    }
    load_queries(0);
    int page = walk.next(a.pages, list, b, begin, step);
    PagePart<D> t;
    const auto load_k = [&](int page) { t.load_k(a.pages, max(page, 0), hk, lane); };
    const auto load_v = [&](int page) { t.load_v(a.pages, max(page, 0), hk, lane); };
    __builtin_amdgcn_sched_barrier(0);
    load_k(page);
    __builtin_amdgcn_sched_barrier(0);
    load_v(page);
    if (a.rope != LASAD_ROPE_NONE && threadIdx.x < P)
        cs[threadIdx.x] = pair_angle<D, true>(a.rope, threadIdx.x, pos, a.grid_w, pair_turns<D>(a.rope, threadIdx.x, a.log2_base));
    __syncthreads();
    NewKey<D> fresh;
    if (last >= 0) fresh.template append<T>(a, cs, rk, rv, wk, k_old, v_old, hk, pos, last, lane);
    for (int g0 = 0; g0 < (SHARE > 1 ? 1 : G); g0 += EACH) {               // (copies: all of the heads at once)
        if (g0 > 0) {
            __syncthreads();                             // (the sums of the heads before are out of LDS)
            load_queries(g0);
            walk.fill(a.pages, list, b, begin, step);
            page = walk.next(a.pages, list, b, begin, step);
            load_k(page);
            __builtin_amdgcn_sched_barrier(0);
            load_v(page);
        }
        Columns<D, NQ, NP, 1, SHARE> x;
        {
            float y[NF][8];
            rq.unpack(y);
            norm_and_turn<D>(a, a.w[0] != nullptr, wq, cs, quad, y);
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                uint32_t part[4][NQ];
#pragma unroll
                for (int i = 0; i < 4; ++i) split_pair<NQ>(y[f][2 * i], y[f][2 * i + 1], part[i]);
#pragma unroll
                for (int i = 0; i < NQ; ++i) x.q[0][f][i].u = make_uint4(part[0][i], part[1][i], part[2][i], part[3][i]);
            }
        }
        x.p[0] = x.p0 = x.p1 = pos;
        x.m[0] = -INFINITY;
        x.l[0] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) x.acc[0][c] = f32x4v{0.f, 0.f, 0.f, 0.f};
        const auto put_new = [&]() __attribute__((always_inline)) {
            if (fresh.grown) {
                load_k(last);
                load_v(last);
            }
            fresh.put(t, pos % kPage, lane);
        };
        x.template run<true>(t, list, begin, step, page, g.scale * kLog2e, g.window, g.sinks, lane, [&](int i) { return walk.next(a.pages, list, b, i, step); },
                             load_k, load_v, put_new);
        join_waves<O, D, WAVES, SHARE>(red, x.acc[0], x.m[0], x.total(0), wave, lane, min(EACH, G - g0), g.splits, split, [&](int c, int ch) {
            const int64_t at = (int64_t)b * a.Hq + hk * G + g0 + c;
            return Result<O>{g.parts + at * g.splits * (D + 4), (O *)g.o + at * D + ch};
        });
    }
}

template <typename T, typename O, int D, int NP, int SHARE>
void launch_shared(const AppendArgs &a, const AttendArgs &t, hipStream_t s)
{
    const dim3 grid((unsigned)((int64_t)a.rows.B * a.pages.heads), (unsigned)t.splits);
    step_pages_kernel<T, O, D, NP, NP, SHARE, 4><<<grid, dim3(256), 0, s>>>(a, t);
}

template <typename T, typename O, int D, int NP>
hipError_t launch(const AppendArgs &a, const AttendArgs &t, hipStream_t s)
{
    const int G = t.Hq / t.pages.heads;
    if (G <= 4) launch_shared<T, O, D, NP, 4>(a, t, s);
    else if (G <= 8) launch_shared<T, O, D, NP, 2>(a, t, s);
    else launch_shared<T, O, D, NP, 1>(a, t, s);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && t.splits > 1) e = launch_join_pages(t, s);
    return e;
}

}  // namespace

int64_t step_pages_groups(const AttendArgs &t) { return (int64_t)t.rows.B * t.pages.heads * t.splits; }

// Splits of a step whose rows see up to `seen` keys.  us, d = 64, as many query heads as key heads; a join costs some 4:
//   512 workgroups in all: two rows of 16 heads, 16448 keys 17.9; 256 19.0, 1024 19.5.
//   from 1536 keys on: two rows of 16 heads 1100 keys 9.8, split 11.0; 1600 11.1 and 11.1 split, 2000 11.8 and 10.3, 4000 17.9 and 12.7.
//   four at least: 8 rows of 16 heads 4000 keys 18.3, in four 17.6; 9 rows 18.6, in three 19.5; 16 rows 30.0, in two 32.9.  (At 16000 keys 68 and 55,
//     71 and 62, 95 and 100: with so many three are worth their join, which the rule leaves out.)
//   512 keys each: one row of 16 heads, 4000 keys 11.0; 256 10.4, 1024 13.0; 8000 keys 12.8; 13.2, 13.6; 2000 keys 10.3; 9.3, 11.7.
//   64 at most: one row of 4 heads, 65000 keys 14.5; 32 15.9, 128 15.8; 40000 13.3; 13.6, 14.0.
int step_pages_splits(int64_t B, int Hq, int Hk, int64_t seen)
{
    int64_t n = 512 / (B * Hk);
    if (seen < 1536 || n < 4) return 1;
    if (n > seen / 512) n = seen / 512;
    return (int)(n > 64 ? 64 : n < 1 ? 1 : n);
}

hipError_t launch_step_pages(const AppendArgs &a, const AttendArgs &t, hipStream_t s)
{
#define LASAD_SP(T, O, NP) (a.d == 32 ? launch<T, O, 32, NP>(a, t, s) : a.d == 64 ? launch<T, O, 64, NP>(a, t, s) : launch<T, O, 128, NP>(a, t, s))
    if (a.io_dtype == LASAD_F32) return LASAD_SP(float, float, 3);
    return t.out_dtype == LASAD_BF16 ? LASAD_SP(uint16_t, uint16_t, 2) : LASAD_SP(uint16_t, float, 2);
#undef LASAD_SP
}

}  // namespace lasad
