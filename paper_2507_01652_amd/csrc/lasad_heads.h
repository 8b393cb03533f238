// What the kernels that normalise and turn heads share: a head's channels over lanes, eight to a lane, sums over a head, and the rotation of
// its pairs by a table of cosines and sines.
#pragma once

#include "lasad_attention.h"
#include "lasad_mfma_util.h"

namespace lasad {

template <int BF16>
__device__ inline void load8(const char *p, float (&f)[8])
{
    if (BF16) {
        const uint4 w = *(const uint4 *)p;
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[2 * e] = __uint_as_float(ww[e] << 16);
            f[2 * e + 1] = __uint_as_float(ww[e] & 0xffff0000u);
        }
    } else {
        const float4 lo = *(const float4 *)p, hi = *(const float4 *)(p + 16);
        f[0] = lo.x; f[1] = lo.y; f[2] = lo.z; f[3] = lo.w;
        f[4] = hi.x; f[5] = hi.y; f[6] = hi.z; f[7] = hi.w;
    }
}

template <int BF16>
__device__ inline void store8(char *p, const float (&f)[8])
{
    if (BF16) {
        *(uint4 *)p = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
    } else {
        *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
        *(float4 *)(p + 16) = make_float4(f[4], f[5], f[6], f[7]);
    }
}

template <int CTRL>
__device__ inline float dpp_move(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ inline float dpp_add(float x)
{
    return x + dpp_move<CTRL>(x);
}

// Sum over the LPR lanes (4, 8 or 16, aligned) of a row, in every one of them.
template <int LPR>
__device__ inline float row_sum(float x)
{
    x = dpp_add<0xB1>(x);                        // lane ^ 1
    x = dpp_add<0x4E>(x);                        // lane ^ 2
    if (LPR >= 8) x = dpp_add<0x141>(x);         // mirrored in 8 lanes: the other four (which are equal by now)
    if (LPR >= 16) x = dpp_add<0x140>(x);        // mirrored in 16 lanes
    return x;
}

// What a lane needs to turn its 8 channels with the table of its token.
struct Turn {
    int base;            // first table entry
    int partner;         // halves: lane distance to the other member of the pairs
    float sign;          // halves: -1 where this lane holds the first members
};

template <int D>
__device__ inline Turn lane_turn(int rope, int pairing, int piece)
{
    constexpr int LPR = D / 8;
    Turn t = {4 * piece, 0, 1.f};
    if (pairing == LASAD_PAIR_HALVES) {
        t.partner = rope == LASAD_ROPE_2D ? LPR / 4 : LPR / 2;
        const bool first = (piece & t.partner) == 0;
        t.sign = first ? -1.f : 1.f;
        t.base = rope == LASAD_ROPE_2D ? (piece / (LPR / 2)) * (D / 4) + (piece % (LPR / 4)) * 8 : (piece % (LPR / 2)) * 8;
    }
    return t;
}

// y turned in place; inverse: by the opposite angles.
__device__ inline void turn8(const float2 *cs, const Turn &t, bool inverse, float (&y)[8])
{
    if (t.partner == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 c = cs[t.base + i];
            const float s = inverse ? -c.y : c.y, p = y[2 * i], q = y[2 * i + 1];
            y[2 * i] = p * c.x - q * s;
            y[2 * i + 1] = p * s + q * c.x;
        }
    } else {
        const float sg = inverse ? -t.sign : t.sign;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 c = cs[t.base + i];
            y[i] = y[i] * c.x + __shfl_xor(y[i], t.partner) * (sg * c.y);
        }
    }
}

// Turns a position of a pair: base^(-k / pairs of an axis) / (2 pi), k its number on its axis.
template <int D>
__device__ inline double pair_turns(int rope, int pair, double log2_base)
{
    const int k = rope == LASAD_ROPE_2D ? pair % (D / 4) : pair;
    return rope == LASAD_ROPE_NONE ? 0.0 : exp2(-(double)k * log2_base / (rope == LASAD_ROPE_2D ? D / 4 : D / 2)) * 0.15915494309189533577;
}
// Its cosine and sine at a position.  FINE: with what the rounding of the reduced angle to fp32 leaves out, up to 2^-26 turns, which is three
// times what the cosine's own rounding costs.
template <int D, bool FINE = false>
__device__ inline float2 pair_angle(int rope, int pair, int pos, int grid_w, double turns_each)
{
    int p = pos;
    if (rope == LASAD_ROPE_2D) p = pair < D / 4 ? pos / grid_w : pos % grid_w;
    const double turns = (double)p * turns_each, part = turns - rint(turns);
    const float r = (float)part;                                     // -0.5 .. 0.5
    float s, c;
    sincospif(2.0f * r, &s, &c);
    if (!FINE) return make_float2(c, s);
    const float rest = (float)(part - (double)r) * 6.2831853f;
    return make_float2(fmaf(-s, rest, c), fmaf(c, rest, s));
}

}  // namespace lasad
