// What the kernels of the window attention share: matrix-core fragments of either storage type, tiles in LDS, and which
// keys a query sees.
//
// All products are 32 x 32 blocks with the reduction over k in pieces; a lane of the result holds column lane % 32 and the
// 16 rows 8 (i / 4) + 4 (lane / 32) + i % 4.  Scores are formed with the keys (or, in the key pass of the backward, the
// queries) in the rows, so that a column's numbers lie in two lanes, and the same registers are, group by group of rows, the
// second operand of the next product: its reduction runs over exactly those rows, in the order in which the lane holds them.
// The first operand is then read from the row-major tile by columns in that order: bf16 with the transposing LDS read (four
// rows of one column), fp32 with plain reads.
#pragma once

#include "lasad_attention.h"
#include "lasad_mfma_util.h"

namespace lasad {

template <typename T> struct Mat;

template <> struct Mat<uint16_t> {
    static constexpr int VEC = 8;              // elements of 16 bytes
    static constexpr int KF = 16;              // reduction of one fragment
    static constexpr int PAD = 8;              // of a row in LDS: 36 dwords of 64 channels, so that 16 rows' pieces meet in no bank
    static constexpr int GROUPS = 2;           // fragments of a block's 32 rows
    typedef Frag F;
    static __device__ inline F piece(const uint16_t *p) { F f; f.u = *(const uint4 *)p; return f; }
    static __device__ inline F zero() { F f; f.u = make_uint4(0, 0, 0, 0); return f; }
    // fragment kf of the row that starts at p
    static __device__ inline F row(const uint16_t *p, int kf, int half) { return piece(p + kf * 16 + 8 * half); }
    // columns col0 .. col0 + 31 of the rows of group g of the block that starts at p
    static __device__ inline F column(const uint16_t *p, int ld, int col0, int g, int lane)
    {
        const int half = lane >> 5, col = col0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3), r = 16 * g + 4 * half + ((lane & 15) >> 2);
        F f;
        f.h[0] = tr_read(p + r * ld + col);
        f.h[1] = tr_read(p + (r + 8) * ld + col);
        return f;
    }
    static __device__ inline F pack(const f32x16 &x, int g)
    {
        F f;
        f.u = make_uint4(pack2(x[8 * g], x[8 * g + 1]), pack2(x[8 * g + 2], x[8 * g + 3]), pack2(x[8 * g + 4], x[8 * g + 5]),
                         pack2(x[8 * g + 6], x[8 * g + 7]));
        return f;
    }
    static __device__ inline f32x16 mma(const F &a, const F &b, f32x16 c) { return mfma(a, b, c); }
    static __device__ inline float dot(const F &a, const F &b)
    {
        const uint32_t x[4] = {a.u.x, a.u.y, a.u.z, a.u.w}, y[4] = {b.u.x, b.u.y, b.u.z, b.u.w};
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), s);
            s = fmaf(__uint_as_float(x[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u), s);
        }
        return s;
    }
};

template <> struct Mat<float> {
    static constexpr int VEC = 4, KF = 8, PAD = 4, GROUPS = 4;
    typedef float4 F;
    static __device__ inline F piece(const float *p) { return *(const float4 *)p; }
    static __device__ inline F zero() { return make_float4(0.f, 0.f, 0.f, 0.f); }
    static __device__ inline F row(const float *p, int kf, int half) { return piece(p + kf * 8 + 4 * half); }
    static __device__ inline F column(const float *p, int ld, int col0, int g, int lane)
    {
        const float *q = p + (8 * g + 4 * (lane >> 5)) * ld + col0 + (lane & 31);
        return make_float4(q[0], q[ld], q[2 * ld], q[3 * ld]);
    }
    static __device__ inline F pack(const f32x16 &x, int g) { return make_float4(x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]); }
    static __device__ inline f32x16 mma(const F &a, const F &b, f32x16 c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, b.x, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, b.y, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, b.z, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, b.w, c, 0, 0, 0);
    }
    static __device__ inline float dot(const F &a, const F &b) { return fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, a.w * b.w))); }
};

// Products of 16 x 16 in bf16 (a quad is 16 lanes).  Which rows and which channels a lane has is free, as long as both operands of a
// product agree, and goes by LDS, 64 banks.  Row 4 quad + i of a product of 16 queries (keys) is number 4 i + first_row(quad) of them: lanes
// 0 .. 31 read eight rows by columns, eight dwords of each, and even rows, like odd ones, lie 8 banks apart (36 dwords a row of 64
// channels).  By rows, 16 bytes a lane, lanes 0-3, 12-15 and 20-27 read together, then 4-11, 16-19 and 28-31: with channels 32 apart in
// neighbouring quads the two share no bank (d >= 64).
__device__ inline int first_row(int quad) { return 2 * (quad & 1) + (quad >> 1); }
// first of a lane's eight channels in reduction step f
template <int D>
__device__ inline int channel(int f, int quad)
{
    return D == 32 ? 8 * quad : 32 * (quad & 1) + 8 * (quad >> 1) + 16 * (f & 1) + 64 * (f >> 1);
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;          // by how much (a power of two) a score may pass the forward's running maximum

__device__ inline f32x16 zeros16()
{
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}

// x of this lane and of the one 32 lanes away, joined
__device__ inline float both_halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float both_halves_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Between a wavefront's writes to its own LDS and its other lanes' reads: the hardware keeps a wavefront's LDS operations in order, the
// compiler has to as well.
__device__ inline void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// row of a lane's register i in a 32 x 32 block
__device__ inline int block_row(int i, int half) { return 8 * (i >> 2) + 4 * half + (i & 3); }

// Does position p see key j (of `keys` valid ones)?
__device__ inline bool sees(const WindowArgs &a, int keys, int p, int j)
{
    return j <= p && j < keys && (p - j < a.window || j < a.sinks);
}
// No / every position of p0 .. p1 sees any / all keys of j0 .. j1.
__device__ inline bool sees_none(const WindowArgs &a, int keys, int p0, int p1, int j0, int j1)
{
    return j0 > p1 || j0 >= keys || (p0 - j1 >= a.window && j0 >= a.sinks);
}
__device__ inline bool sees_all(const WindowArgs &a, int keys, int p0, int p1, int j0, int j1)
{
    return j1 <= p0 && j1 < keys && (p1 - j0 < a.window || j1 < a.sinks);
}

// The same for a range of positions, as comparisons with four numbers that a walk over keys keeps.
struct Range {
    int last, before, top, bottom, sinks;
    __device__ inline Range(const WindowArgs &a, int keys, int p0, int p1)
        : last(min(p1, keys - 1)), before(p0 - a.window), top(min(p0, keys - 1)), bottom(p1 - a.window), sinks(a.sinks) {}
    __device__ inline bool some(int j0, int j1) const { return j0 <= last && (j1 > before || j0 < sinks); }
    __device__ inline bool top_edge(int j1) const { return j1 > top; }
    __device__ inline bool bottom_edge(int j0) const { return j0 <= bottom; }                 // (sinks or not)
    __device__ inline bool all(int j0, int j1) const { return j1 <= top && (j0 > bottom || j1 < sinks); }
};

// What a column's query sees of the rows of a block of keys (or a column's key of the rows of a block of queries): rows
// lo .. hi, and those before `first`.  Two comparisons with a constant an entry, and which of them a block needs is the same for
// the whole wavefront, so that a block inside the window pays none.
struct Edge {
    int lo, hi, first;
};
__device__ inline Edge query_edge(const WindowArgs &a, int keys, int p)
{
    const int hi = min(p, keys - 1);
    return {max(0, p - a.window + 1), hi, min(a.sinks, hi + 1)};
}
__device__ inline Edge key_edge(const WindowArgs &a, int keys, int j)
{
    const int far = 0x5fffffff;                          // (behind all positions, and a block's offset may be taken off)
    return {j < keys ? j : far, j < a.sinks ? far : (int)min((int64_t)far, (int64_t)j + a.window - 1), 0};
}
// x in the entries of block rows r0 .. r0 + 31 that are not seen; top, bottom: rows behind hi, before lo are among them
__device__ inline void hide(f32x16 &s, const Edge &e, int r0, int half, bool top, bool bottom, float x)
{
    const int hi = e.hi - r0 - 4 * half, lo = e.lo - r0 - 4 * half, first = e.first - r0 - 4 * half;
    if (top) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 8 * (i >> 2) + (i & 3) <= hi ? s[i] : x;
    }
    if (bottom) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 8 * (i >> 2) + (i & 3) >= lo || 8 * (i >> 2) + (i & 3) < first ? s[i] : x;
    }
}
// valid keys of batch row b
__device__ inline int valid_keys(const WindowArgs &a, int b)
{
    int keys = a.m;
    if (a.lens) {
        const int l = a.lens[b];
        keys = l < 0 ? 0 : l < a.m ? l : a.m;
    }
    return keys;
}

// Infinities and NaN.  A query that does not see a row of a tile has 0 in its place, and 0 * NaN would reach its sums through the
// matrix cores.  Tiles that not every query (key) of a workgroup sees all of are therefore looked over on their way to LDS, and what
// is not finite is kept out of the second product's operand and added for those that do see it: a few operations a tile at the
// borders of what is seen, and a slow loop only where there is such a value.
template <typename T>
__device__ inline bool finite_bits(uint32_t w)           // both bf16 of a word, or one float
{
    const uint32_t e = 0x7f800000u;
    return (w & e) != e && (sizeof(T) == 4 || (w << 16 & e) != e);
}
template <typename T>
__device__ inline uint32_t finite_word(uint32_t w)
{
    if (sizeof(T) == 4) return finite_bits<T>(w) ? w : 0u;
    return ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u) | ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu);
}
// r without what is not finite; whether there was any
template <typename T>
__device__ inline bool make_finite(uint4 &r)
{
    const bool bad = !(finite_bits<T>(r.x) && finite_bits<T>(r.y) && finite_bits<T>(r.z) && finite_bits<T>(r.w));
    if (bad) r = make_uint4(finite_word<T>(r.x), finite_word<T>(r.y), finite_word<T>(r.z), finite_word<T>(r.w));
    return bad;
}
template <typename T>
__device__ inline float as_float(T x)
{
    if constexpr (sizeof(T) == 2) return bf16_bits_to_float(x);
    else return x;
}
// Adds the values of a row that are not finite to a lane's results (32 DB channels of one column), where `on`.
template <typename T, int DB>
__device__ inline void add_infinite(const T *row, bool on, int half, f32x16 (&acc)[DB])
{
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float x = as_float<T>(row[d * 32 + block_row(i, half)]);
            if (on && !(fabsf(x) < INFINITY)) acc[d][i] += x;
        }
}
// Is any of a row's D values not finite?
template <typename T, int D>
__device__ inline bool row_infinite(const T *row, int lane)
{
    bool bad = false;
    for (int c = lane; c < D; c += 64) bad |= !(fabsf(as_float<T>(row[c])) < INFINITY);
    return __any(bad);
}

// The launch order of `units` pieces of work of each of `heads` heads.  Workgroups follow one another over the 8 L2s: with 8 heads
// and more each L2 gets heads of its own, so that what shares keys meets there, and its workgroups take piece after piece of all its
// heads, so that pieces that take long, which come first, do not start last.  Fewer heads are dealt out over all L2s.
// Heads (times batch rows) between two multiples of 8 take what the larger one does, as some dies then have a head less or none: 4096
// tokens, window 1024, forward 28.7 us for 8 heads, 34.7 for 9, 35.1 for 12, 37.0 for 16, 45.5 for 17, 47.4 for 24, backward 72, 92, 93, 95, 126
// and 130.
struct Place {
    int head, unit;                    // (head -1: nothing to do)
};
__device__ inline Place launch_place(unsigned index, int heads, int units)
{
    if (heads < 8) return {(int)(index % (unsigned)heads), (int)(index / (unsigned)heads)};
    const unsigned each = ((unsigned)heads + 7) / 8, slot = index >> 3;
    const int head = (int)((index & 7) * each + slot % each);
    return {head < heads ? head : -1, (int)(slot / each)};
}
inline int64_t launch_groups(int64_t heads, int64_t units) { return heads < 8 ? heads * units : (heads + 7) / 8 * 8 * units; }
inline unsigned launch_grid(int64_t heads, int64_t units) { return (unsigned)launch_groups(heads, units); }     // (kMostGroups at most)

// Four consecutive results of a lane, as they leave the registers.
template <typename O>
__device__ inline void store4(O *p, float x, float y, float z, float w)
{
    if (sizeof(O) == 2) *(uint2 *)p = make_uint2(pack2(x, y), pack2(z, w));
    else *(float4 *)p = make_float4(x, y, z, w);
}

// Launch `kernel<T, O, D>` for the types and head dim of `a`.
#define LASAD_WINDOW_DISPATCH(LAUNCH)                                                     \
    do {                                                                                  \
        if (a.io_dtype == LASAD_BF16 && a.out_dtype == LASAD_BF16) {                      \
            if (a.d == 32) LAUNCH(uint16_t, uint16_t, 32);                                \
            else if (a.d == 64) LAUNCH(uint16_t, uint16_t, 64);                           \
            else LAUNCH(uint16_t, uint16_t, 128);                                         \
        } else if (a.io_dtype == LASAD_BF16) {                                            \
            if (a.d == 32) LAUNCH(uint16_t, float, 32);                                   \
            else if (a.d == 64) LAUNCH(uint16_t, float, 64);                              \
            else LAUNCH(uint16_t, float, 128);                                            \
        } else {                                                                          \
            if (a.d == 32) LAUNCH(float, float, 32);                                      \
            else if (a.d == 64) LAUNCH(float, float, 64);                                 \
            else LAUNCH(float, float, 128);                                               \
        }                                                                                 \
    } while (0)

}  // namespace lasad
