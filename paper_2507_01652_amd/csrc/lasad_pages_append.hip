// New tokens of rows into the paged 8-bit cache, with the norm of query and key heads and their rotation on the way (lasad_qk.hip has
// those formulas).  Of every page of a row that gets tokens, and of every key head, with y the call's tokens in it:
//     A = max |y| (of the finite ones);   s = A / 448 if the page has no earlier token, or its scale is 0;
//     otherwise s = s_old 2^j, j >= 0 the smallest with 448 s >= A, and the earlier codes are divided by 2^j;
//     code = e4m3(y / s).
// A power of two keeps the earlier codes exact but for the smallest binades, so that a page filled token by token is not rounded again and
// again; and the first scale as it comes leaves no border at which a rounding of A would change a page by a factor of two.
//
// A wavefront has one head of one page, queries, keys or values: all of its numbers are in registers, so that A is known before the first code is
// formed, with no wait for others.  Of queries and keys a lane has 8 channels of up to 64 / (512 / d) tokens in a row, of values d / 16 channels
// of the 16 tokens whose codes are 16 bytes in a row of a channel.  Bound by memory: every number is read once, codes are written once.  What the
// next head needs is on its way while one is worked on, and the first one's before the table of angles is formed.
#include "lasad_heads.h"
#include "lasad_pages_codes.h"

namespace lasad {

namespace {

constexpr int kThreads = 256, kWaves = 4;

// the largest of a wavefront's lanes, in every one of them
__device__ inline float wave_max(float x)
{
    x = fmaxf(x, dpp_move<0xB1>(x));
    x = fmaxf(x, dpp_move<0x4E>(x));
    x = fmaxf(x, dpp_move<0x141>(x));
    x = fmaxf(x, dpp_move<0x140>(x));
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return both_halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

// n words from p on.
template <int N>
__device__ inline void load_words(const char *p, uint32_t *w)
{
    if constexpr (N == 1) {
        w[0] = *(const uint32_t *)p;
    } else if constexpr (N == 2) {
        const uint2 x = *(const uint2 *)p;
        w[0] = x.x; w[1] = x.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 x = *(const uint4 *)(p + 4 * i);
            w[i] = x.x; w[i + 1] = x.y; w[i + 2] = x.z; w[i + 3] = x.w;
        }
    }
}
template <int BF16>
__device__ inline float word_float(const uint32_t *w, int e)
{
    if (BF16) return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    return __uint_as_float(w[e]);
}

enum { kNone, kAdjacent, kHalves };

template <int BF16, int OBF16, int D, int TURN>
__global__ void __launch_bounds__(kThreads, D == 128 ? 2 : 3)
append_pages_kernel(AppendArgs a, int groups)
{
    constexpr int LPR = D / 8, P = D / 2, TPL = kPage * LPR / 64;          // lanes of a token, pairs, tokens of a lane
    constexpr int ELT = BF16 ? 2 : 4, OELT = OBF16 ? 2 : 4;
    constexpr int CH = D / 16, VW = CH * ELT / 4;                          // values: channels and words of a lane and token
    constexpr bool AHEAD = BF16 || D < 128;                                // (fp32 of 128 channels would not fit in registers twice)
    __shared__ __align__(16) float2 cs[kPage * P];
    const int group = blockIdx.x % groups;
    PageRow row;
    if (!find_row(a.rows, a.pages, blockIdx.x / groups, 1, kPage, 2, row)) return;
    const int j = row.pos / kPage + row.unit;
    if (j * kPage >= row.pos + row.n) return;
    const int begin = max(row.pos - j * kPage, 0), end = min(row.pos + row.n - j * kPage, kPage);      // the call's positions in the page
    const int64_t token0 = (int64_t)row.first + j * kPage - row.pos;                                  // token of the page's position 0
    const int page = __builtin_amdgcn_readfirstlane(page_of(a.pages, row.b, j));

    // A lane's place is formed anew for each head: kept, all the offsets that follow from it would fill the registers.
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    struct Place {
        int lane, piece, slot0;                          // queries and keys: 8 channels from 8 piece on, TPL positions from slot0 on
        int quad, ch0;                                   // values: CH channels from ch0 on, positions 16 b + 4 quad + i
        __device__ inline Place()
        {
            lane = threadIdx.x & 63;
            asm volatile("" : "+v"(lane));
            piece = lane % LPR; slot0 = lane / LPR * TPL;
            quad = lane % 4; ch0 = lane / 4 * CH;
        }
    };
    const auto here = [&](int t) { return t >= begin && t < end; };
    const auto near = [&](int t) -> int64_t { return min(max(t, begin), end - 1); };          // (other positions: one of the call's once more)

    const int q_heads = a.q ? a.Hq : 0, heads = a.pages.heads, units = q_heads + (page < 0 ? 0 : 2 * heads), step = groups * kWaves;
    uint32_t raw[D * ELT / 4];
    float w[8], old = 0.f;
    const auto load = [&](int unit) {
        const Place at;
        if (unit < q_heads + heads) {
            const bool key = unit >= q_heads;
            const int h = key ? unit - q_heads : unit;
            const lasad_layout_t &l = key ? a.lk : a.lq;
            const int64_t stride = l.stride_n;
            const char *in = (const char *)(key ? a.k : a.q) + (token0 * stride + h * l.stride_h + at.piece * 8) * ELT;
#pragma unroll
            for (int u = 0; u < TPL; ++u)
                load_words<2 * ELT>(in + near(at.slot0 + u) * stride * ELT, raw + u * 2 * ELT);
            if (a.w[key]) load8<0>((const char *)(a.w[key] + (a.shared ? 0 : (int64_t)h * D) + at.piece * 8), w);
            if (key) old = a.pages.k_scale[(int64_t)page * heads + h];
        } else {
            const int h = unit - q_heads - heads;
            const int64_t stride = a.lv.stride_n;
            const char *in = (const char *)a.v + (token0 * stride + h * a.lv.stride_h + at.ch0) * ELT;
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                load_words<VW>(in + near(u / 4 * 16 + 4 * at.quad + u % 4) * stride * ELT, raw + u * VW);
                if (u % 4 == 3) __builtin_amdgcn_sched_barrier(0);           // (addresses of a few at a time)
            }
            old = a.pages.v_scale[(int64_t)page * heads + h];
        }
    };
    int unit = group * kWaves + wave;
    if (AHEAD && unit < units) load(unit);
    if (TURN != kNone) {
        const int pair = tid % P;
        const double f = pair_turns<D>(a.rope, pair, a.log2_base);
        for (int t = begin + tid / P; t < end; t += kThreads / P) cs[t * P + pair] = pair_angle<D>(a.rope, pair, j * kPage + t, a.grid_w, f);
    }
    __syncthreads();

    for (; unit < units; unit += step) {
        if (!AHEAD) load(unit);
        const Place at;
        const bool value = unit >= q_heads + heads, key = !value && unit >= q_heads;
        const int h = value ? unit - q_heads - heads : key ? unit - q_heads : unit;
        const int64_t ph = (int64_t)page * heads + h;
        const float was = old;
        if (value) {
            uint8_t *codes = a.pages.v + ph * kPage * D;
            uint4 before[CH] = {};
            bool all = true;
#pragma unroll
            for (int b = 0; b < 4; ++b) all &= here(16 * b + 4 * at.quad) && here(16 * b + 4 * at.quad + 3);
            if (!all) {
#pragma unroll
                for (int e = 0; e < CH; ++e) before[e] = *(const uint4 *)(codes + (at.ch0 + e) * kPage + 16 * at.quad);
            }
            float y[16][CH], most = 0.f;
#pragma unroll
            for (int u = 0; u < 16; ++u)
#pragma unroll
                for (int e = 0; e < CH; ++e) {
                    y[u][e] = word_float<BF16>(raw + u * VW, e);
                    most = fmaxf(most, finite_size(y[u][e]));
                }
            if (AHEAD && unit + step < units) load(unit + step);
            float less;
            const float s = page_scale(wave_max(most), begin, was, less);
            if (at.lane == 0) a.pages.v_scale[ph] = s;
            const Divide by(s);
#pragma unroll
            for (int e = 0; e < CH; ++e) {
                uint32_t c[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) c[b] = code4(by(y[4 * b][e]), by(y[4 * b + 1][e]), by(y[4 * b + 2][e]), by(y[4 * b + 3][e]));
                if (!all) {
                    const uint32_t o[4] = {before[e].x, before[e].y, before[e].z, before[e].w};
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const int t = 16 * b + 4 * at.quad;
                        const uint32_t earlier = first_bytes(begin - t), mine = first_bytes(end - t) & ~earlier;
                        c[b] = (c[b] & mine) | ((less < 1.f ? shrink(o[b], less, earlier) : o[b]) & ~mine);
                    }
                }
                *(uint4 *)(codes + (at.ch0 + e) * kPage + 16 * at.quad) = make_uint4(c[0], c[1], c[2], c[3]);
            }
            continue;
        }
        const Turn turn = lane_turn<D>(a.rope, TURN == kHalves ? LASAD_PAIR_HALVES : LASAD_PAIR_ADJACENT, at.piece);
        float y[TPL][8], x[8];
#pragma unroll
        for (int u = 0; u < TPL; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[u][e] = word_float<BF16>(raw + u * 2 * ELT, e);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = a.w[key] ? w[e] : 1.f;
        if (AHEAD && unit + step < units) load(unit + step);
        // (one run of code with no branches: values that branches change would be held twice)
#pragma unroll
        for (int u = 0; u < TPL; ++u) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(y[u][e], y[u][e], ss);
            const float r = rsqrtf(row_sum<LPR>(ss) * (1.0f / D) + a.eps), rstd = a.norm ? r : 1.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[u][e] = y[u][e] * rstd * x[e];
            if constexpr (TURN != kNone) turn8(cs + near(at.slot0 + u) * P, turn, false, y[u]);
            if (u % 2) __builtin_amdgcn_sched_barrier(0);               // (all tokens' angles at once would need registers)
        }
        if (!key) {
            const int64_t stride = a.lo.stride_n;
            char *out = (char *)a.q_out + ((token0 + at.slot0) * stride + h * a.lo.stride_h + at.piece * 8) * OELT;
#pragma unroll
            for (int u = 0; u < TPL; ++u)
                if (here(at.slot0 + u)) store8<OBF16>(out + u * stride * OELT, y[u]);
            continue;
        }
        float most = 0.f, less;
#pragma unroll
        for (int u = 0; u < TPL; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, finite_size(y[u][e]));
        const float s = page_scale(wave_max(most), begin, was, less);
        if (at.lane == 0) a.pages.k_scale[ph] = s;
        const Divide by(s);
        uint8_t *codes = a.pages.k + ph * kPage * D + at.slot0 * D + at.piece * 8;
        if (less < 1.f) {
            uint2 o[TPL] = {};
#pragma unroll
            for (int u = 0; u < TPL; ++u)
                if (at.slot0 + u < begin) o[u] = *(const uint2 *)(codes + u * D);
#pragma unroll
            for (int u = 0; u < TPL; ++u)
                if (at.slot0 + u < begin) *(uint2 *)(codes + u * D) = make_uint2(shrink(o[u].x, less, 0xffffffffu), shrink(o[u].y, less, 0xffffffffu));
        }
#pragma unroll
        for (int u = 0; u < TPL; ++u)
            if (here(at.slot0 + u))
                *(uint2 *)(codes + u * D) =
                    make_uint2(code4(by(y[u][0]), by(y[u][1]), by(y[u][2]), by(y[u][3])), code4(by(y[u][4]), by(y[u][5]), by(y[u][6]), by(y[u][7])));
    }
}

// Workgroups of a page's heads: one for each four of them, fewer where the pages fill the chip four times over, as each forms the table of
// angles for itself.
int64_t slots_of(const AppendArgs &a) { return row_slots(a.rows, 1, kPage, 2); }

int head_groups(const AppendArgs &a)
{
    const int units = (a.q ? a.Hq : 0) + 2 * a.pages.heads, most = (units + kWaves - 1) / kWaves;
    const int64_t want = (1024 + slots_of(a) - 1) / slots_of(a);
    return (int)(want < 1 ? 1 : want > most ? most : want);
}

}  // namespace

int64_t append_pages_groups(const AppendArgs &a) { return slots_of(a) * head_groups(a); }

hipError_t launch_append_pages(const AppendArgs &a, hipStream_t s)
{
    const int groups = head_groups(a);
    const dim3 grid((unsigned)append_pages_groups(a)), block(kThreads);
    const int turn = a.rope == LASAD_ROPE_NONE ? kNone : a.pairing == LASAD_PAIR_ADJACENT ? kAdjacent : kHalves;
#define LASAD_AP_T(I, O, D, T) append_pages_kernel<I, O, D, T><<<grid, block, 0, s>>>(a, groups)
#define LASAD_AP(I, O, D) (turn == kNone ? (void)(LASAD_AP_T(I, O, D, kNone)) : turn == kAdjacent ? (void)(LASAD_AP_T(I, O, D, kAdjacent)) : (void)(LASAD_AP_T(I, O, D, kHalves)))
#define LASAD_AP_D(I, O) (a.d == 32 ? LASAD_AP(I, O, 32) : a.d == 64 ? LASAD_AP(I, O, 64) : LASAD_AP(I, O, 128))
    if (a.io_dtype == LASAD_BF16) { if (a.out_dtype == LASAD_BF16) LASAD_AP_D(1, 1); else LASAD_AP_D(1, 0); }
    else LASAD_AP_D(0, 0);
#undef LASAD_AP_D
#undef LASAD_AP
#undef LASAD_AP_T
    return hipGetLastError();
}

}  // namespace lasad
