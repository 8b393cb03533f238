// A page's keys and values against tiles of 16 columns, as matrix operands straight from memory (lasad_pages_attend.hip has the formulas): what the
// attention of packed queries and the step share.
#pragma once

#include <type_traits>

#include "lasad_pages.h"

namespace lasad {

// Sum or maximum of a column's four lanes, in each of them.
__device__ inline float quads_max(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return both_halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ inline float quads_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return both_halves_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Four codes as bf16, times a power of two.
__device__ inline uint2 codes_bf16(uint32_t w, float scale)
{
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true)));
}
__device__ inline Frag codes_frag(uint32_t lo, uint32_t hi, float scale = 1.f)
{
    Frag f;
    f.h[0] = codes_bf16(lo, scale);
    f.h[1] = codes_bf16(hi, scale);
    return f;
}

// x in N bf16 parts, each the rounding of what those before it leave.
template <int N>
__device__ inline void split_pair(float x, float y, uint32_t (&part)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        part[i] = pack2(x, y);
        x -= __uint_as_float(part[i] << 16);
        y -= __uint_as_float(part[i] & 0xffff0000u);
    }
}

__device__ inline uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }     // 0x80 where a code is NaN

// A number at an address that is the same in all lanes, through the scalar cache: one more vector load between those of the pages would have
// the next page's keys wait for the values behind it.  The scalar cache does not see what the same launch writes: the step, which writes the
// scales of a row's last page, may find the old ones here, and has to put the new ones in their place (NewKey::put).
template <typename T>
__device__ inline T scalar_load(const T *p) { return *(const __attribute__((address_space(4))) T *)(uintptr_t)p; }

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A lane's share of a page: k of four blocks of 16 positions (its position of each, 16 channels of 64), v of all positions that the second
// product has in its lane (its channel of every 16).
template <int D>
struct PagePart {
    static constexpr int KL = D == 32 ? 1 : D / 64;      // loads of k of a block
    typedef typename std::conditional<D == 32, u32x2, u32x4>::type K;
    K k[4][KL];
    u32x4 v[D / 16];
    float k_scale, v_scale;
    __device__ inline void load_k(const Pages &p, int page, int h, int lane)
    {
        const int64_t at = (int64_t)page * p.heads + h;
        const int col = lane & 15, quad = lane >> 4;
        const uint8_t *kp = p.k + at * kPage * D + col * D + quad * sizeof(K);
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int c = 0; c < KL; ++c) k[b][c] = *(const K *)(kp + b * 16 * D + c * 64);
        k_scale = scalar_load(p.k_scale + at);
    }
    __device__ inline void load_v(const Pages &p, int page, int h, int lane)
    {
        const int64_t at = (int64_t)page * p.heads + h;
        const uint8_t *vp = p.v + at * kPage * D + (lane & 15) * kPage + (lane >> 4) * 16;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) v[c] = *(const u32x4 *)(vp + c * 16 * kPage);
        v_scale = scalar_load(p.v_scale + at);
    }
    // words 2 f and 2 f + 1 of a block's k: the codes of reduction step f
    __device__ inline uint32_t k_word(int b, int f, int i) const
    {
        if constexpr (D == 32) return k[b][0][i];
        else return k[b][f >> 1][2 * (f & 1) + i];
    }
};
// first of a lane's eight channels in reduction step f of the first product
template <int D>
__device__ inline int page_channel(int f, int quad) { return D == 32 ? 8 * quad : 64 * (f >> 1) + 16 * quad + 8 * (f & 1); }

// The pages that positions p0 .. p1 see: those of the sinks before the window's, then the window's.
struct PageList {
    int sink_pages, first, count;
    __device__ inline PageList(int p0, int p1, int window, int sinks)
    {
        first = max(0, p0 - window + 1) / kPage;
        sink_pages = min((int)(((int64_t)sinks + kPage - 1) / kPage), first);
        count = p1 < 0 ? 0 : sink_pages + p1 / kPage - first + 1;
    }
    __device__ inline int number(int i) const { return i < sink_pages ? i : first + i - sink_pages; }
};

// The pages that a wavefront takes, every `step`th from `begin` on: their numbers in the pool are loaded 64 at a time.
struct Walk {
    int ids, used;
    __device__ inline void fill(const Pages &p, const PageList &list, int b, int i, int step)
    {
        const int at = i + (int)(threadIdx.x & 63) * step;
        ids = at < list.count ? page_of(p, b, list.number(at)) : -1;
        used = 0;
    }
    // of item i: begin, then the ones that follow in turn
    __device__ inline int next(const Pages &p, const PageList &list, int b, int i, int step)
    {
        if (used == 64) fill(p, list, b, i, step);
        return __builtin_amdgcn_readlane(ids, used++);
    }
};

// A wavefront's columns: NT tiles of 16, this lane's column of each.  SHARE > 1, for fewer queries than a tile has columns: 16 / SHARE queries
// lie in it SHARE times, and copy i keeps those scores alone whose block of 16 positions is i modulo SHARE.  Its sums are over those, as if it
// were another wavefront's, and a lane has 16 / SHARE scores of a page to raise to a power instead of 16.
template <int D, int NQ, int NP, int NT, int SHARE = 1>
struct Columns {
    static constexpr int NF = D / 32, NC = D / 16, NB = 4 / SHARE;        // NB: blocks of a lane
    static_assert(SHARE == 1 || NT == 1, "copies of one tile");
    Frag q[NT][NF][NQ];
    int p[NT];                                           // position (-1: no column)
    int p0, p1;                                          // first and last position of the wavefront's columns
    float m[NT], l[NT];
    f32x4v acc[NT][NC];

    // Scores of a page, 16 positions x 16 columns a product.
    __device__ inline void scores(const PagePart<D> &t, int copy, f32x4v (&s)[NT][NB]) const
    {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            Frag k[NF];
#pragma unroll
            for (int f = 0; f < NF; ++f) k[f] = codes_frag(t.k_word(b, f, 0), t.k_word(b, f, 1));
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                f32x4v x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = NQ - 1; i >= 0; --i)
#pragma unroll
                    for (int f = 0; f < NF; ++f) x = mfma16(k[f], q[n][f][i], x);
                if (b % SHARE == 0) {
                    s[n][b / SHARE] = x;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[n][b / SHARE][i] = copy == b % SHARE ? x[i] : s[n][b / SHARE][i];
                }
            }
        }
        wait_for_products();
    }

    // P = 2^(s sc - m + log2_more) as the second product's operand, and its sums.  Of a whole tile as it enters the product, by a product with ones,
    // which the matrix cores have more room for than the vector units; of copies, which have fewer terms a lane, by additions (a lane's own).
    __device__ inline void powers(const f32x4v (&s)[NT][NB], float sc, float log2_more, int copy, Frag (&pf)[NT][2][NP], float (&sum)[NT]) const
    {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float use = (m[n] == -INFINITY ? 0.f : m[n]) - log2_more;        // (nothing seen yet: every term is 2^-inf)
            float e[NB][4];
            uint32_t part[NB][2][NP];
#pragma unroll
            for (int r = 0; r < NB; ++r) {
#pragma unroll
                for (int i = 0; i < 4; ++i) e[r][i] = __builtin_amdgcn_exp2f(fmaf(s[n][r][i], sc, -use));
#pragma unroll
                for (int i = 0; i < 2; ++i) split_pair<NP>(e[r][2 * i], e[r][2 * i + 1], part[r][i]);
            }
#pragma unroll
            for (int x = 0; x < NP; ++x) {
                uint2 w[NB];
#pragma unroll
                for (int r = 0; r < NB; ++r) w[r] = make_uint2(part[r][0][x], part[r][1][x]);
                spread(w, copy, pf[n][0][x], pf[n][1][x]);
            }
            if constexpr (SHARE > 1) {
                sum[n] = 0.f;
#pragma unroll
                for (int r = 0; r < NB; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[n] += e[r][i];
            }
        }
        if constexpr (SHARE == 1) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                Frag ones;
                ones.u = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
                f32x4v x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = NP - 1; i >= 0; --i)
#pragma unroll
                    for (int half = 0; half < 2; ++half) x = mfma16(ones, pf[n][half][i], x);
                sum[n] = x[0];
            }
        }
    }

    __device__ inline void add_values(const u32x4 (&values)[NC], const Frag (&pf)[NT][2][NP], float power)
    {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const Frag v = half ? codes_frag(values[c].z, values[c].w, power) : codes_frag(values[c].x, values[c].y, power);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int x = NP - 1; x >= 0; --x) acc[n][c] = mfma16(v, pf[n][half][x], acc[n][c]);
            }
        wait_for_products();
    }

    // Items i, i + step, .. of the list, the first (in `page`) in `t`: what their keys add.  next(i): page of the next item, i (-1: none of the
    // pool's; none of another's keys are seen); load_k(page), load_v(page) load it: once a page's keys are used, and its values, in their
    // place, so that loads are in flight all the time with one set of registers.  finish() puts into the list's last page what is new in it.
    //
    // Most pages are seen whole and raise no maximum by much: their P is formed with the maximum at hand, and the sums, which are needed
    // anyway, tell if a score was beyond 2^kLimit of it.  Then that page, and those that are seen in part, take the long way, which looks for
    // the maximum first.  The short way has a loop of its own, and leaves it with the loads of a next page under way, as it goes round:
    // joined with the long one, every page moved the accumulators twice; left with others, the compiler lets the next keys wait for the values
    // behind them.
    //
    // A page's P adds up to 2^16, that of 2^24 pages to 2^40: from values of 2^72 448 on the sums could pass fp32 although their average
    // does not.  The first page whose scale is 2^72 or more goes the long way, where the maximum is raised by 2^42 for good: P and its sums are
    // less by as much, and what divides them too.  (4 x 24 heads over 8, 4096 tokens: 138.6 us with it and without.)
    template <bool FINISH, typename Next, typename LoadK, typename LoadV, typename Finish>
    __device__ __forceinline__ void run(PagePart<D> &t, const PageList &list, int i, int step, int page, float scale2, int window, int sinks, int lane, Next next,
                                        LoadK load_k, LoadV load_v, Finish finish)
    {
        constexpr int kLimit = 16, kLift = 42;           // (64 keys at 2^kSlack have 2^14)
        constexpr uint32_t kLarge = 0x63800000u;         // 2^72
        int lift = 0;
        bool large;                                      // the first page of such values
        const int quad = lane >> 4;
        const int copy = SHARE > 1 ? (lane & 15) / (16 / SHARE) : 0, own = 4 * quad + 16 * copy;      // (a lane's block r is number SHARE r + copy)
        bool ready = false;                              // every column has a maximum
        f32x4v s[NT][NB];
        Frag pf[NT][2][NP];
        float sum[NT], sc, power, log2_more, less;
        bool there, whole;
        int j0, taken = page;
        const auto go_on = [&]() __attribute__((always_inline)) {
            taken = page;
            i += step;
            if (i < list.count) page = next(i);                      // (behind the last page that one again)
        };
        const auto start = [&]() __attribute__((always_inline)) {
            scores(t, copy, s);
            sc = fmaxf(t.k_scale * scale2, 0x1p-149f);               // (a page of zeros has scale 0, and 0 times -infinity is none)
        };
        const auto load_next_k = [&]() __attribute__((always_inline)) {
            __builtin_amdgcn_sched_barrier(0);                       // (loads moved up over the products, or conversions over the exponentials, would need registers)
            load_k(page);
            // The values' scale is 2^e f, 1 <= f < 2: codes become bf16 with the power of two, and P is raised to P f by its exponent.
            const uint32_t vbits = there && t.v_scale > 0.f ? __float_as_uint(t.v_scale) : 0x3f800000u;
            const float f = __uint_as_float((vbits & 0x007fffffu) | 0x3f800000u);
            power = __uint_as_float(vbits & 0x7f800000u);
            log2_more = __builtin_amdgcn_logf(f);
            less = __builtin_amdgcn_rcpf(f);
            large = vbits >= kLarge && lift == 0;
        };
        enum { kDone, kLong, kAgain };
        int left = i < list.count ? kLong : kDone;
        while (left != kDone) {
            for (;;) {
                j0 = __builtin_amdgcn_readfirstlane(list.number(i)) * kPage;
                there = page >= 0;
                whole = there && j0 + kPage - 1 <= p0 && !(j0 <= p1 - window && j0 + kPage > sinks) && !(FINISH && i == list.count - 1);
                if (!whole || !ready) break;
                start();
                go_on();
                load_next_k();
                powers(s, sc, log2_more, copy, pf, sum);
                bool fine = !large;
                const float limit = __uint_as_float((127 + kLimit - lift) << 23);
#pragma unroll
                for (int n = 0; n < NT; ++n) fine &= sum[n] <= limit;
                if (!__all(fine)) {
                    load_v(page);
                    left = kAgain;
                    break;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) l[n] = fmaf(sum[n], less, l[n]);
                add_values(t.v, pf, power);
                load_v(page);
                if (i >= list.count) {
                    left = kDone;
                    break;
                }
            }
            if (left == kDone) break;
            if (left == kAgain) {
                load_k(taken);
                load_v(taken);
                start();
            } else {
                if (FINISH && there && i == list.count - 1) finish();
                start();
                go_on();
            }
            load_next_k();

            if (!whole) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int hi = there ? p[n] - j0 - own : -1, lo = max(0, p[n] - window + 1) - j0 - own, first = sinks - j0 - own;
#pragma unroll
                    for (int r = 0; r < NB; ++r)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int at = 16 * SHARE * r + i;
                            s[n][r][i] = (at <= hi) & ((at >= lo) | (at < first)) ? s[n][r][i] : -INFINITY;
                        }
                }
            }
            ready = true;
            const float raise = large ? kLift : 0;
            if (large) lift = kLift;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float top = -INFINITY;
#pragma unroll
                for (int r = 0; r < NB; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, s[n][r][i]);
                top = fmaf(quads_max(top), sc, (float)lift);
                const float m0 = m[n] + raise, m1 = top > m0 + kSlack ? top : m0;
                const float fade = m[n] == m1 ? 1.f : __builtin_amdgcn_exp2f(m[n] - m1);
                m[n] = m1;
                ready &= p[n] < 0 || m1 != -INFINITY;
                l[n] *= fade;
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[n][c][i] *= fade;
            }
            ready = __all(ready);
            powers(s, sc, log2_more, copy, pf, sum);
#pragma unroll
            for (int n = 0; n < NT; ++n) l[n] = fmaf(sum[n], less, l[n]);
            // A code that not every column sees may be NaN (what is not yet written is anything), and 0 * NaN would reach the sums: such codes
            // are 0 in the product, and the columns that do see one get their NaN from a product of flags.
            u32x4 v[NC];
#pragma unroll
            for (int c = 0; c < NC; ++c) v[c] = t.v[c];
            if (!whole) {
                uint32_t bad = 0;
#pragma unroll
                for (int c = 0; c < NC; ++c) bad |= nan_bytes(v[c].x) | nan_bytes(v[c].y) | nan_bytes(v[c].z) | nan_bytes(v[c].w);
                if (__any(bad != 0)) take_nan_out(v, j0, there, window, sinks, copy, own);
            }
            add_values(v, pf, power);
            load_v(page);
            left = i < list.count ? kLong : kDone;
        }
    }

    __device__ inline float total(int n) const { return SHARE == 1 ? l[n] : quads_sum(l[n]); }

    // A lane's blocks, four bf16 of each, as the operands of the second product: 0 where a block is another copy's.
    static __device__ inline void spread(const uint2 (&w)[NB], int copy, Frag &low, Frag &high)
    {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const bool mine = SHARE == 1 || copy == b % SHARE;
            (b < 2 ? low : high).h[b & 1] = make_uint2(mine ? w[b / SHARE].x : 0u, mine ? w[b / SHARE].y : 0u);
        }
    }

    __device__ inline void take_nan_out(u32x4 (&v)[NC], int j0, bool there, int window, int sinks, int copy, int own)
    {
        Frag seen[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int hi = there ? p[n] - j0 - own : -1, lo = max(0, p[n] - window + 1) - j0 - own, first = sinks - j0 - own;
            uint2 w[NB];
#pragma unroll
            for (int r = 0; r < NB; ++r) {
                uint32_t on[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = 16 * SHARE * r + i;
                    on[i] = (at <= hi) & ((at >= lo) | (at < first)) ? 0x3f80u : 0u;
                }
                w[r] = make_uint2(on[0] | on[1] << 16, on[2] | on[3] << 16);
            }
            spread(w, copy, seen[n][0], seen[n][1]);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            uint32_t w[4] = {v[c].x, v[c].y, v[c].z, v[c].w}, flag[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t nan = nan_bytes(w[i]) >> 7;
                w[i] &= ~(nan * 0xffu);
                flag[i] = nan * 0x38u;                               // (the code of 1)
            }
            v[c] = u32x4{w[0], w[1], w[2], w[3]};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                f32x4v count = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int half = 0; half < 2; ++half) count = mfma16(codes_frag(flag[2 * half], flag[2 * half + 1]), seen[n][half], count);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (count[i] > 0.f) acc[n][c][i] = __builtin_nanf("");
            }
        }
    }
};

// Eight channels of a query as the parts of a fragment.
template <typename T, int NQ>
__device__ inline void query_parts(const T *p, Frag (&f)[NQ])
{
    if constexpr (sizeof(T) == 2) {
        f[0].u = *(const uint4 *)p;
    } else {
        const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
        uint32_t part[4][NQ];
        split_pair<NQ>(a.x, a.y, part[0]);
        split_pair<NQ>(a.z, a.w, part[1]);
        split_pair<NQ>(b.x, b.y, part[2]);
        split_pair<NQ>(b.z, b.w, part[3]);
#pragma unroll
        for (int i = 0; i < NQ; ++i) f[i].u = make_uint4(part[0][i], part[1][i], part[2][i], part[3][i]);
    }
}

// The sums of KW wavefronts (and of SHARE copies in each) that share columns, joined in `red` and put out: results (of splits: parts) of
// `columns` of them, to where `to` says.
template <typename O>
struct Result {
    float *parts;                                        // of the column's splits
    O *o;                                                // its channels from `ch` on
};
template <typename O, int D, int KW, int SHARE, typename To>
__device__ inline void join_waves(float (&red)[KW][16][D + 4], const f32x4v (&acc)[D / 16], float m, float l, int kw, int lane, int columns, int splits,
                                  int split, To to)
{
    const int quad = lane >> 4;
    float *mine = red[kw][lane & 15];
#pragma unroll
    for (int b = 0; b < D / 16; ++b) *(float4 *)(mine + 16 * b + 4 * quad) = make_float4(acc[b][0], acc[b][1], acc[b][2], acc[b][3]);
    if (quad == 0) { mine[D] = m; mine[D + 1] = l; }
    __syncthreads();
    constexpr int EACH = 16 / SHARE;
    for (int i = threadIdx.x; i < EACH * D / 4; i += KW * 64) {
        const int c = i / (D / 4), ch = i % (D / 4) * 4;
        if (c >= columns) continue;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < KW * SHARE; ++w) top = fmaxf(top, red[w / SHARE][c + w % SHARE * EACH][D]);
        const float use = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < KW * SHARE; ++w) {
            const float *x = red[w / SHARE][c + w % SHARE * EACH];
            const float f = __builtin_amdgcn_exp2f(x[D] - use);
            const float4 r = *(const float4 *)(x + ch);
            sum = fmaf(x[D + 1], f, sum);
            o.x = fmaf(r.x, f, o.x); o.y = fmaf(r.y, f, o.y); o.z = fmaf(r.z, f, o.z); o.w = fmaf(r.w, f, o.w);
        }
        const Result<O> r = to(c, ch);
        if (splits > 1) {
            float *p = r.parts + split * (D + 4);
            *(float4 *)(p + ch) = o;
            if (ch == 0) { p[D] = top; p[D + 1] = sum; }
        } else {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            store4(r.o, o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        }
    }
}

}  // namespace lasad
