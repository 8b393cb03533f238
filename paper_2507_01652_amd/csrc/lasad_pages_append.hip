// New tokens of rows into the paged 8-bit cache, with the norm of query and key heads and their rotation on the way (lasad_qk.hip has
// those formulas).  Of every page of a row that gets tokens, and of every key head, with y the call's tokens in it:
//     A = max |y| (of the finite ones);   s = A / 448 if the page has no earlier token, or its scale is 0;
//     otherwise s = s_old 2^j, j >= 0 the smallest with 448 s >= A, and the earlier codes are divided by 2^j;
//     code = e4m3(y / s).
// A power of two keeps the earlier codes exact but for the smallest binades, so that a page filled token by token is not rounded again and
// again; and the first scale as it comes leaves no border at which a rounding of A would change a page by a factor of two.
//
// A wavefront has 2048 numbers of one head of one page (queries, keys or values), in registers, so that A is known before the first code is formed:
// of queries and keys 2048 / d tokens, a lane 8 channels of four of them in a row; of values 32 channels, a lane two of the 16 tokens whose
// codes are 16 bytes in a row of a channel.  d / 32 wavefronts share a head and tell each other their maxima.  Twice as many numbers a lane
// (no sharing at d = 64) took registers for two or three wavefronts a SIMD instead of four: 66 us for the 252 MB below, where this took 60 then.  Values in
// the same wavefront as their keys, in the keys' order and with codes of 4 bytes, before that: 98.  What the next head needs is on its way while one is worked on, and
// the first one's before the table of angles is formed.
//
// Bound by memory: every number is read once, codes are written once.  4 x 4096 tokens of 72 heads in bf16, d = 64 (252 MB): 54 us by itself, 4.6 TB/s where
// a copy of 1 GiB reaches 5.0; 58 a pass in a stream.  32 rows of 22 to 200 tokens of 36 heads (27 MB): 15, two rounds of latencies (row, page, numbers) and of
// workgroups on partly filled pages; one token of 36 heads 5.6, a launch and those latencies.
#include <type_traits>

#include "lasad_heads.h"
#include "lasad_pages_codes.h"

namespace lasad {

namespace {

constexpr int kThreads = 512, kWaves = 8;

// the largest of a wavefront's lanes, in every one of them
__device__ inline uint32_t wave_max(uint32_t x)
{
    x = max(x, __float_as_uint(dpp_move<0xB1>(__uint_as_float(x))));
    x = max(x, __float_as_uint(dpp_move<0x4E>(__uint_as_float(x))));
    x = max(x, __float_as_uint(dpp_move<0x141>(__uint_as_float(x))));
    x = max(x, __float_as_uint(dpp_move<0x140>(__uint_as_float(x))));
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(r[0], r[1]);
    const auto t = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max(t[0], t[1]);
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

template <int N>
using Int = std::integral_constant<int, N>;

enum { kNone, kAdjacent, kHalves };

template <int BF16, int OBF16, int D, int TURN>
__global__ void __launch_bounds__(kThreads, 4)
append_pages_kernel(AppendArgs a, int groups)
{
    constexpr int LPR = D / 8, P = D / 2, PARTS = D / 32, ABREAST = kWaves / PARTS;      // lanes of a token, pairs, wavefronts of a head, heads at once
    constexpr int ELT = BF16 ? 2 : 4, OELT = OBF16 ? 2 : 4, RW = 2 * ELT, VW = ELT / 2;  // words of 8 channels, of 2
    __shared__ __align__(16) float2 cs[TURN == kNone ? 1 : kPage * P];
    __shared__ uint32_t tops[2][kWaves];
    const int group = blockIdx.x % groups;
    PageRow row;
    if (!find_row(a.rows, a.pages, blockIdx.x / groups, 1, kPage, 2, row)) return;
    if (row.unit > (row.pos % kPage + row.n - 1) / kPage) return;
    const int j = row.pos / kPage + row.unit;
    const int begin = max(row.pos - j * kPage, 0), end = min(row.pos + row.n - j * kPage, kPage);      // the call's positions in the page
    const int64_t token0 = (int64_t)row.first + j * kPage - row.pos;                                  // token of the page's position 0
    const int entry = page_of(a.pages, row.b, j);

    // A lane's place is formed anew for each head: kept, all the offsets that follow from it would fill the registers.
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = wave % PARTS;
    struct Place {
        int lane, piece, slot;                           // queries and keys: 8 channels from 8 piece on, four positions from slot on
        int quad, ch;                                    // values: two channels from ch on, positions 16 b + 4 quad + i
        __device__ inline explicit Place(int part)
        {
            lane = threadIdx.x & 63;
            asm volatile("" : "+v"(lane));
            piece = lane % LPR; slot = part * (kPage / PARTS) + lane / LPR * 4;
            quad = lane % 4; ch = part * 32 + lane / 4 * 2;
        }
    };
    const auto here = [&](int t) { return t >= begin && t < end; };
    const auto near = [&](int t) { return min(max(t, begin), end - 1); };          // (other positions: one of the call's once more)
    // words of N positions' numbers, from the token of position 0 on: offsets in 32 bits where the stride allows it (16 MB a token)
    const auto load_tokens = [&](auto words, auto count, const char *in, uint32_t lane_bytes, int64_t stride, uint32_t *to, auto position) {
        constexpr int W = decltype(words)::value, N = decltype(count)::value;
        if (stride < 1 << 24) {
            if (begin == 0 && end == kPage) {
                const uint32_t at = (uint32_t)position(0) * (uint32_t)stride + lane_bytes;
#pragma unroll
                for (int u = 0; u < N; ++u) load_words<W>(in + (position(u) - position(0)) * stride + at, to + u * W);
            } else {
#pragma unroll
                for (int u = 0; u < N; ++u) load_words<W>(in + (__umul24(near(position(u)), (uint32_t)stride) + lane_bytes), to + u * W);
            }
        } else {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                load_words<W>(in + near(position(u)) * stride + lane_bytes, to + u * W);
                __builtin_amdgcn_sched_barrier(0);                             // (one address at a time)
            }
        }
    };

    const int q_heads = a.q ? a.Hq : 0, heads = a.pages.heads, step = groups * ABREAST;
    uint32_t raw[16 * VW];
    float w[8];
    const auto load = [&](int unit) {
        const Place at(part);
        if (unit < q_heads + heads) {
            const bool key = unit >= q_heads;
            const int h = key ? unit - q_heads : unit;
            const lasad_layout_t &l = key ? a.lk : a.lq;
            const char *in = (const char *)(key ? a.k : a.q) + (token0 * l.stride_n + h * l.stride_h) * ELT;
            load_tokens(Int<RW>(), Int<4>(), in, at.piece * 8 * ELT, l.stride_n * ELT, raw, [&](int u) { return at.slot + u; });
            if (a.w[key]) load8<0>((const char *)(a.w[key] + (a.shared ? 0 : (int64_t)h * D) + at.piece * 8), w);
        } else {
            const int h = unit - q_heads - heads;
            const char *in = (const char *)a.v + (token0 * a.lv.stride_n + h * a.lv.stride_h) * ELT;
            load_tokens(Int<VW>(), Int<16>(), in, at.ch * ELT, a.lv.stride_n * ELT, raw, [&](int u) { return u / 4 * 16 + 4 * at.quad + u % 4; });
        }
    };
    int unit = group * ABREAST + wave / PARTS;
    if (unit < q_heads + 2 * heads) load(unit);
    if constexpr (TURN != kNone) {
        const int pair = tid % P;
        const double f = pair_turns<D>(a.rope, pair, a.log2_base);
        for (int t = begin + tid / P; t < end; t += kThreads / P) cs[t * P + pair] = pair_angle<D, true>(a.rope, pair, j * kPage + t, a.grid_w, f);
        __syncthreads();
    }
    const int page = __builtin_amdgcn_readfirstlane(entry), units = q_heads + (page < 0 ? 0 : 2 * heads);

    // What the pages held: the scale, and the old bytes beside the call's in a lane's 16 of a value.
    float next_old = 0.f;
    uint4 next_before[2] = {};
    const auto load_old = [&](int unit) {
        if (unit < q_heads || unit >= units) return;
        const Place at(part);
        const bool value = unit >= q_heads + heads;
        const int64_t ph = (int64_t)page * heads + (value ? unit - q_heads - heads : unit - q_heads);
        next_old = (value ? a.pages.v_scale : a.pages.k_scale)[ph];
        if (value && (begin > 0 || end < kPage)) {
            const uint8_t *codes = a.pages.v + ph * kPage * D + at.ch * kPage + 16 * at.quad;
            next_before[0] = *(const uint4 *)codes;
            next_before[1] = *(const uint4 *)(codes + kPage);
        }
    };
    load_old(unit);
    for (int first = group * ABREAST, turn_of = 0; first < units; first += step, unit += step, turn_of ^= 1) {        // (as often in all wavefronts)
        const Place at(part);
        if (!BF16 && first != group * ABREAST) {         // (a second set would not fit in registers)
            if (unit < units) load(unit);
            load_old(unit);
        }
        const bool on = unit < units, value = unit >= q_heads + heads, key = !value && unit >= q_heads;
        const int h = value ? unit - q_heads - heads : key ? unit - q_heads : unit;
        const int64_t ph = (int64_t)page * heads + h;
        uint8_t *codes = value ? a.pages.v + ph * kPage * D + at.ch * kPage + 16 * at.quad : a.pages.k + ph * kPage * D + at.slot * D + at.piece * 8;
        float *scale = (value ? a.pages.v_scale : a.pages.k_scale) + ph;
        const float old = next_old;
        const uint4 before[2] = {next_before[0], next_before[1]};
        float y[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) y[i] = word_float<BF16>(raw + i / 2 * VW, i % 2);          // (four tokens' 8 channels, or 16 tokens' two)
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = a.w[key] ? w[e] : 1.f;
        if constexpr (BF16) {
            if (unit + step < units) load(unit + step);
            load_old(unit + step);
        }
        if (!value) {
            const Turn turn = lane_turn<D>(a.rope, TURN == kHalves ? LASAD_PAIR_HALVES : LASAD_PAIR_ADJACENT, at.piece);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float (&z)[8] = *(float (*)[8])(y + 8 * u);
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(z[e], z[e], ss);
                const float r = rsqrtf(row_sum<LPR>(ss) * (1.0f / D) + a.eps), rstd = a.norm ? r : 1.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = z[e] * rstd * x[e];
                if constexpr (TURN != kNone) turn8(cs + near(at.slot + u) * P, turn, false, z);
                if (!BF16) __builtin_amdgcn_sched_barrier(0);
            }
            if (!key && on) {
                char *out = (char *)a.q_out + ((token0 + at.slot) * a.lo.stride_n + h * a.lo.stride_h + at.piece * 8) * OELT;
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (here(at.slot + u)) store8<OBF16>(out + u * a.lo.stride_n * OELT, *(const float (*)[8])(y + 8 * u));
            }
        }
        // The bits of magnitudes are in their order, what is not finite behind: a second look where there is any.
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) most = max(most, __float_as_uint(y[i]) & 0x7fffffffu);
        most = wave_max(most);
        if (most >= 0x7f800000u) {
            most = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) most = max(most, __float_as_uint(finite_size(y[i])));
            most = wave_max(most);
        }
        if constexpr (PARTS > 1) {
            if (at.lane == 0) tops[turn_of][wave] = most;
            __syncthreads();                             // (the other half of `tops` is read by then)
#pragma unroll
            for (int i = 0; i < PARTS; ++i) most = max(most, tops[turn_of][wave - part + i]);
        }
        if (!on || !(value || key)) continue;
        float less;
        const float s = page_scale(__uint_as_float(most), begin, old, less);
        if (part == 0 && at.lane == 0) *scale = s;
        const Divide by(s);
        if (value) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                uint32_t c[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) c[b] = code4(by(y[8 * b + e]), by(y[8 * b + 2 + e]), by(y[8 * b + 4 + e]), by(y[8 * b + 6 + e]));
                if (begin > 0 || end < kPage) {
                    const uint32_t o[4] = {before[e].x, before[e].y, before[e].z, before[e].w};
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const int t = 16 * b + 4 * at.quad;
                        const uint32_t earlier = first_bytes(begin - t), mine = first_bytes(end - t) & ~earlier;
                        c[b] = (c[b] & mine) | ((less < 1.f ? shrink(o[b], less, earlier) : o[b]) & ~mine);
                    }
                }
                *(uint4 *)(codes + e * kPage) = make_uint4(c[0], c[1], c[2], c[3]);
            }
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                uint2 c = make_uint2(code4(by(y[8 * u]), by(y[8 * u + 1]), by(y[8 * u + 2]), by(y[8 * u + 3])),
                                     code4(by(y[8 * u + 4]), by(y[8 * u + 5]), by(y[8 * u + 6]), by(y[8 * u + 7])));
                const bool earlier = less < 1.f && at.slot + u < begin;
                if (earlier) {
                    c = *(const uint2 *)(codes + u * D);
                    c = make_uint2(shrink(c.x, less, 0xffffffffu), shrink(c.y, less, 0xffffffffu));
                }
                if (earlier || here(at.slot + u)) *(uint2 *)(codes + u * D) = c;
            }
        }
    }
}

// Workgroups of a page's heads: as many as its heads can have, fewer where the pages alone fill the chip twice over, as each forms the table of
// angles for itself (want 512 of them: 252 MB as above 57.9 us, 1024 63.0, 256 87; 27 MB 14.9, 16.7, 17.6).
int64_t slots_of(const AppendArgs &a) { return row_slots(a.rows, 1, kPage, 2); }

int head_groups(const AppendArgs &a)
{
    const int units = (a.q ? a.Hq : 0) + 2 * a.pages.heads, abreast = kWaves * 32 / a.d, most = (units + abreast - 1) / abreast;
    const int64_t want = (512 + slots_of(a) - 1) / slots_of(a);
    return (int)(want < 1 ? 1 : want > most ? most : want);
}

}  // namespace

int64_t append_pages_groups(const AppendArgs &a) { return slots_of(a) * head_groups(a) * (kThreads / 256); }

hipError_t launch_append_pages(const AppendArgs &a, hipStream_t s)
{
    const int groups = head_groups(a);
    const dim3 grid((unsigned)(slots_of(a) * groups)), block(kThreads);
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
