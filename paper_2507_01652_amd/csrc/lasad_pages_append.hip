// New tokens of rows into the paged 8-bit cache, with the norm of query and key heads and their rotation on the way (lasad_qk.hip has
// those formulas).  Of every page of a row that gets tokens, and of every key head, with y the call's tokens in it:
//     A = max |y| (of the finite ones);   s = A / 448 if the page has no earlier token, or its scale is 0;
//     otherwise s = s_old 2^j, j >= 0 the smallest with 448 s >= A, and the earlier codes are divided by 2^j;
//     code = e4m3(y / s).
// A power of two keeps the earlier codes exact but for the smallest binades, so that a page filled token by token is not rounded again and
// again; and the first scale as it comes leaves no border at which a rounding of A would change a page by a factor of two.
//
// A wavefront has one head of one page: all of its numbers are in registers (a lane has 8 channels of up to 64 / (512 / d) tokens in a row), so
// that A is known before the first code is formed, with no wait for others.  Bound by memory: every number is read once, codes are written once.
#include "lasad_heads.h"
#include "lasad_pages_codes.h"

namespace lasad {

namespace {

constexpr int kThreads = 256, kWaves = 4;

// the largest of a wavefront's lanes, in every one of them
__device__ inline float wave_max(float x)
{
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) x = fmaxf(x, __shfl_xor(x, off));
    return x;
}

template <int BF16, int OBF16, int D>
__global__ void __launch_bounds__(kThreads)
append_pages_kernel(AppendArgs a, int groups)
{
    constexpr int LPR = D / 8, P = D / 2, TPL = kPage * LPR / 64;          // lanes of a token, pairs, tokens of a lane
    constexpr int ELT = BF16 ? 2 : 4, OELT = OBF16 ? 2 : 4;
    __shared__ __align__(16) float2 cs[kPage * P];
    const int group = blockIdx.x % groups;
    PageRow row;
    if (!find_row(a.rows, a.pages, blockIdx.x / groups, 1, kPage, 2, row)) return;
    const int j = row.pos / kPage + row.unit;
    if (j * kPage >= row.pos + row.n) return;
    const int begin = max(row.pos - j * kPage, 0), end = min(row.pos + row.n - j * kPage, kPage);      // the call's positions in the page
    const int64_t token0 = (int64_t)row.first + j * kPage - row.pos;                                  // token of the page's position 0
    const int page = page_of(a.pages, row.b, j);

    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, piece = lane % LPR, slot0 = lane / LPR * TPL;
    if (a.rope != LASAD_ROPE_NONE) {
        const int pair = tid % P;
        const double f = pair_turns<D>(a.rope, pair, a.log2_base);
        for (int t = begin + tid / P; t < end; t += kThreads / P) cs[t * P + pair] = pair_angle<D>(a.rope, pair, j * kPage + t, a.grid_w, f);
    }
    __syncthreads();
    const Turn turn = lane_turn<D>(a.rope, a.pairing, piece);
    const auto here = [&](int u) { return slot0 + u >= begin && slot0 + u < end; };

    const int q_heads = a.q ? a.Hq : 0, units = q_heads + a.pages.heads;
    for (int unit = group * kWaves + wave; unit < units; unit += groups * kWaves) {
        const bool key = unit >= q_heads;
        const int h = key ? unit - q_heads : unit;
        if (key && page < 0) continue;
        const lasad_layout_t &l = key ? a.lk : a.lq;
        const char *in = (const char *)(key ? a.k : a.q) + ((token0 + slot0) * l.stride_n + h * l.stride_h + piece * 8) * ELT;
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = 1.f;
        if (a.w[key]) load8<0>((const char *)(a.w[key] + (a.shared ? 0 : (int64_t)h * D) + piece * 8), w);
        float y[TPL][8];
#pragma unroll
        for (int u = 0; u < TPL; ++u) {
            if (here(u)) {
                load8<BF16>(in + u * l.stride_n * ELT, y[u]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[u][e] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < TPL; ++u) {
            if (!here(u)) continue;
            if (a.norm) {
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(y[u][e], y[u][e], ss);
                const float rstd = rsqrtf(row_sum<LPR>(ss) * (1.0f / D) + a.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[u][e] = y[u][e] * rstd * w[e];
            }
            if (a.rope != LASAD_ROPE_NONE) turn8(cs + (slot0 + u) * P, turn, false, y[u]);
        }
        if (!key) {
            char *out = (char *)a.q_out + ((token0 + slot0) * a.lo.stride_n + h * a.lo.stride_h + piece * 8) * OELT;
#pragma unroll
            for (int u = 0; u < TPL; ++u)
                if (here(u)) store8<OBF16>(out + u * a.lo.stride_n * OELT, y[u]);
            continue;
        }
        const int64_t ph = (int64_t)page * a.pages.heads + h;
        bool grown;
        {
            float most = 0.f;
#pragma unroll
            for (int u = 0; u < TPL; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, finite_size(y[u][e]));
            uint8_t *codes = a.pages.k + ph * kPage * D;
            const Divide by(page_scale<D, false>(wave_max(most), begin, a.pages.k_scale[ph], a.pages.k_scale + ph, codes, lane, grown));
#pragma unroll
            for (int u = 0; u < TPL; ++u)
                if (here(u))
                    *(uint2 *)(codes + (slot0 + u) * D + piece * 8) =
                        make_uint2(code4(by(y[u][0]), by(y[u][1]), by(y[u][2]), by(y[u][3])), code4(by(y[u][4]), by(y[u][5]), by(y[u][6]), by(y[u][7])));
        }
        in = (const char *)a.v + ((token0 + slot0) * a.lv.stride_n + h * a.lv.stride_h + piece * 8) * ELT;
        float most = 0.f;
#pragma unroll
        for (int u = 0; u < TPL; ++u) {
            if (here(u)) {
                load8<BF16>(in + u * a.lv.stride_n * ELT, y[u]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[u][e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, finite_size(y[u][e]));
        }
        uint8_t *codes = a.pages.v + ph * kPage * D;
        const Divide by(page_scale<D, true>(wave_max(most), begin, a.pages.v_scale[ph], a.pages.v_scale + ph, codes, lane, grown));
#pragma unroll
        for (int u = 0; u < TPL; u += 4) {
            const int t = slot0 + u, at = 16 * (t / 4 % 4) + 4 * (t / 16);         // place of four positions in a channel's 64
            const bool whole = t >= begin && t + 4 <= end;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t c = code4(by(y[u][e]), by(y[u + 1][e]), by(y[u + 2][e]), by(y[u + 3][e]));
                uint8_t *p = codes + (piece * 8 + e) * kPage + at;
                if (whole) {
                    *(uint32_t *)p = c;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (here(u + i)) p[i] = (uint8_t)(c >> 8 * i);
                }
            }
        }
    }
}

// Workgroups of a page's heads: one for each four of them, fewer where the pages fill the chip four times over, as each forms the table of
// angles for itself.
int64_t slots_of(const AppendArgs &a) { return row_slots(a.rows, 1, kPage, 2); }

int head_groups(const AppendArgs &a)
{
    const int units = (a.q ? a.Hq : 0) + a.pages.heads, most = (units + kWaves - 1) / kWaves;
    const int64_t want = (1024 + slots_of(a) - 1) / slots_of(a);
    return (int)(want < 1 ? 1 : want > most ? most : want);
}

}  // namespace

int64_t append_pages_groups(const AppendArgs &a) { return slots_of(a) * head_groups(a); }

hipError_t launch_append_pages(const AppendArgs &a, hipStream_t s)
{
    const int groups = head_groups(a);
    const dim3 grid((unsigned)append_pages_groups(a)), block(kThreads);
#define LASAD_AP(I, O, D) append_pages_kernel<I, O, D><<<grid, block, 0, s>>>(a, groups)
#define LASAD_AP_D(I, O) (a.d == 32 ? (void)(LASAD_AP(I, O, 32)) : a.d == 64 ? (void)(LASAD_AP(I, O, 64)) : (void)(LASAD_AP(I, O, 128)))
    if (a.io_dtype == LASAD_BF16) { if (a.out_dtype == LASAD_BF16) LASAD_AP_D(1, 1); else LASAD_AP_D(1, 0); }
    else LASAD_AP_D(0, 0);
#undef LASAD_AP_D
#undef LASAD_AP
    return hipGetLastError();
}

}  // namespace lasad
