// Norms of query and key heads and their rotation by raster position, forward and backward.
//
// A row is one head of one token, x in R^d:
//     y = x rstd w,  rstd = 1 / sqrt(mean(x^2) + eps),
// and the d / 2 pairs of y are turned by the token's angles: (a, b) -> (a cos - b sin, a sin + b cos).  Pair i's angle is
// position * base^(-2i/d), or (two axes) row * base^(-4i/d) for the first d / 4 pairs and column * base^(-4(i - d/4)/d) for
// the others.  With g the output's gradient turned back and xh = x rstd,
//     dx = rstd (g w - xh mean(g w xh)),   dw = sum over tokens of g xh.
//
// Bound by memory: every row is read once and written once.  A row is d / 8 lanes of 8 channels (16-byte loads for bf16),
// sums over a row are cross-lane additions, and nothing else is read twice.  What could keep the lanes from waiting for
// memory alone are the angles: a sine and a cosine cost some 60 operations, four pairs to a lane's 16 bytes.  All heads
// of a token share them, so a workgroup forms the table of its tokens in LDS first, one pair to a thread.  The angle is
// formed in fp64 as turns and reduced there (position 2^30 leaves 2^-23 turns), the sine of the rest in fp32.
//
// Measured, bf16, d = 64: 4 x 4096 tokens of 48 heads (201 MB) 35 us a launch and 45 in a stream of them on inputs that are not
// cached, 4.5 TB/s where a copy of 1 GiB reaches 4.94; backward of 32 x 576 tokens of 32 heads (235 MB with the workgroups' weight
// sums) 40 us, and 4.7 for the second kernel.  One token of 24 heads 3 us.  Stores past the caches take the stream of forwards to
// 39.4 us, but what reads the outputs next then finds none of them in the 256 MB in front of the memory (with the attention after
// it: 96 MB of outputs 96 us and 105 so, 192 MB 192 and 195, 768 MB 747 and 740), so they are ordinary ones.
#include "lasad_heads.h"

namespace lasad {

namespace {

constexpr int kThreads = 256;

// The table of `count` tokens from `first` on: cosines and sines, byte offsets of the tokens (queries, keys), whether the
// token is on the grid.
struct Tokens {
    int64_t in[2], dl[2], out[2];
    int on;
};

template <int D>
__device__ inline void make_tables(const QkArgs &a, int64_t first, int count, int elt, int oelt, float2 *cs, Tokens *tok, bool backward)
{
    constexpr int P = D / 2;
    const int tid = threadIdx.x;
    const int pair = tid % P;
    const double f = pair_turns<D>(a.rope, pair, a.log2_base);
    for (int t = tid / P; t < count; t += kThreads / P) {
        const uint32_t token = (uint32_t)(first + t), b = token / (uint32_t)a.n, i = token - b * (uint32_t)a.n;
        int pos = a.start_pos + (int)i;
        bool on = true;
        if (a.pos_rows) {
            const int row_pos = a.pos_rows[b];
            on = row_pos >= 0 && row_pos < a.last_pos;
            pos = on ? row_pos : 0;
        }
        if (pair == 0) {
            Tokens o;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                o.in[x] = ((int64_t)b * a.in[x].stride_b + (int64_t)i * a.in[x].stride_n) * elt;
                o.out[x] = ((int64_t)b * a.out[x].stride_b + (int64_t)i * a.out[x].stride_n) * oelt;
                o.dl[x] = backward ? ((int64_t)b * a.dl[x].stride_b + (int64_t)i * a.dl[x].stride_n) * elt : 0;
            }
            o.on = on;
            tok[t] = o;
        }
        if (a.rope != LASAD_ROPE_NONE) cs[t * P + pair] = pair_angle<D>(a.rope, pair, pos, a.grid_w, f);
    }
}

// tile: tokens of a workgroup; its rows (token by token, heads in order, queries before keys) are dealt out to the lanes.
template <int BF16, int OBF16, int D>
__global__ void __launch_bounds__(kThreads)
qk_forward_kernel(QkArgs a, int tile)
{
    constexpr int LPR = D / 8, P = D / 2, MAX_TILE = 512 / D, SLOTS = kThreads / LPR;
    constexpr int ELT = BF16 ? 2 : 4, OELT = OBF16 ? 2 : 4;
    __shared__ __align__(16) float2 cs[MAX_TILE * P];
    __shared__ Tokens tok[MAX_TILE];
    const int64_t total = (int64_t)a.B * a.n, first = (int64_t)blockIdx.x * tile;
    const int count = (int)(total - first < tile ? total - first : tile);
    make_tables<D>(a, first, count, ELT, OELT, cs, tok, false);
    __syncthreads();

    const int heads = a.heads[0] + a.heads[1];
    const int piece = threadIdx.x % LPR;
    const Turn turn = lane_turn<D>(a.rope, a.pairing, piece);
    int t = (threadIdx.x / LPR) / heads, h = (threadIdx.x / LPR) % heads;
    const int step_t = SLOTS / heads, step_h = SLOTS % heads;
    while (t < count) {
        const int x = h < a.heads[0] ? 0 : 1, hx = h - (x ? a.heads[0] : 0);
        if (tok[t].on) {
            float y[8];
            load8<BF16>((const char *)a.x[x] + tok[t].in[x] + ((int64_t)hx * a.in[x].stride_h + piece * 8) * ELT, y);
            if (a.norm) {
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(y[e], y[e], ss);
                const float rstd = rsqrtf(row_sum<LPR>(ss) * (1.0f / D) + a.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] *= rstd;
                if (a.w[x]) {
                    float w[8];
                    load8<0>((const char *)(a.w[x] + (a.shared ? 0 : (int64_t)hx * D) + piece * 8), w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] *= w[e];
                }
            }
            if (a.rope != LASAD_ROPE_NONE) turn8(cs + t * P, turn, false, y);
            store8<OBF16>((char *)a.y[x] + tok[t].out[x] + ((int64_t)hx * a.out[x].stride_h + piece * 8) * OELT, y);
        }
        t += step_t;
        h += step_h;
        if (h >= heads) { h -= heads; ++t; }
    }
}

}  // namespace

static int64_t forward_tile(int64_t total, int d)
{
    const int64_t tile = total / 1024, most = 512 / d;
    return tile < 1 ? 1 : tile > most ? most : tile;
}

int64_t qk_forward_groups(int64_t tokens, int d)
{
    const int64_t tile = forward_tile(tokens, d);
    return (tokens + tile - 1) / tile;
}

hipError_t launch_qk_forward(const QkArgs &a, hipStream_t s)
{
    const int64_t total = (int64_t)a.B * a.n, tile = forward_tile(total, a.d);
    if (total == 0) return hipSuccess;
    const dim3 grid((unsigned)qk_forward_groups(total, a.d)), block(kThreads);
#define LASAD_QK(I, O, D) qk_forward_kernel<I, O, D><<<grid, block, 0, s>>>(a, (int)tile)
#define LASAD_QK_D(I, O) (a.d == 32 ? (void)(LASAD_QK(I, O, 32)) : a.d == 64 ? (void)(LASAD_QK(I, O, 64)) : (void)(LASAD_QK(I, O, 128)))
    if (a.io_dtype == LASAD_BF16) { if (a.out_dtype == LASAD_BF16) LASAD_QK_D(1, 1); else LASAD_QK_D(1, 0); }
    else LASAD_QK_D(0, 0);
#undef LASAD_QK_D
#undef LASAD_QK
    return hipGetLastError();
}

namespace {

constexpr int kBackTile = 32;                    // tokens of a workgroup of the backward, at most

int64_t back_tile(int64_t total)
{
    const int64_t t = (total + 1023) / 1024;
    return t < 4 ? 4 : t > kBackTile ? kBackTile : t;
}

// Four wavefronts take the workgroup's tokens in turn, group after group of 64 / LPR of its `share` of the heads, so that a lane's
// head stays the same over its tokens and the weight gradient stays in its registers.  Per head they are added up over the
// wavefronts at the end of a group, shared ones at the end of the workgroup; a second kernel adds the workgroups' sums in their order.
template <int BF16, int OBF16, int D, int SHARED>
__global__ void __launch_bounds__(kThreads)
qk_backward_kernel(QkArgs a, int tile, int share)
{
    constexpr int LPR = D / 8, P = D / 2, RPW = 64 / LPR;
    constexpr int ELT = BF16 ? 2 : 4, OELT = OBF16 ? 2 : 4;
    __shared__ __align__(16) float2 cs[kBackTile * P];
    __shared__ Tokens tok[kBackTile];
    __shared__ float red[4 * 64 * 8 * (SHARED ? 2 : 1)];
    const int64_t total = (int64_t)a.B * a.n, first = (int64_t)blockIdx.x * tile;
    const int count = (int)(total - first < tile ? total - first : tile);
    make_tables<D>(a, first, count, ELT, OELT, cs, tok, true);
    __syncthreads();

    const int heads = a.heads[0] + a.heads[1];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, piece = lane % LPR;
    const Turn turn = lane_turn<D>(a.rope, a.pairing, piece);
    const bool want = a.partial != nullptr;
    float accq[8], acck[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) accq[e] = acck[e] = 0.f;
    const int g_end = min(heads, (int)(blockIdx.y + 1) * share);
    for (int g0 = blockIdx.y * share; g0 < g_end; g0 += RPW) {
        const int h = g0 + lane / LPR;
        const int x = h < a.heads[0] ? 0 : 1, hx = h - (x ? a.heads[0] : 0);
        float w[8], acc[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { w[e] = 1.f; acc[e] = 0.f; }
        if (h < heads) {
            if (a.norm && a.w[x]) load8<0>((const char *)(a.w[x] + (a.shared ? 0 : (int64_t)hx * D) + piece * 8), w);
            const char *xp = (const char *)a.x[x] + ((int64_t)hx * a.in[x].stride_h + piece * 8) * ELT;
            const char *gp = (const char *)a.dy[x] + ((int64_t)hx * a.dl[x].stride_h + piece * 8) * ELT;
            char *yp = (char *)a.y[x] + ((int64_t)hx * a.out[x].stride_h + piece * 8) * OELT;
            for (int t = wave; t < count; t += 4) {
                float v[8], g[8];
                load8<BF16>(xp + tok[t].in[x], v);
                load8<BF16>(gp + tok[t].dl[x], g);
                if (a.rope != LASAD_ROPE_NONE) turn8(cs + t * P, turn, true, g);
                if (a.norm) {
                    float ss = 0.f, sg = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        ss = fmaf(v[e], v[e], ss);
                        sg = fmaf(g[e] * w[e], v[e], sg);
                    }
                    const float rstd = rsqrtf(row_sum<LPR>(ss) * (1.0f / D) + a.eps);
                    const float m = row_sum<LPR>(sg) * (1.0f / D) * rstd;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float xh = v[e] * rstd;
                        acc[e] = fmaf(g[e], xh, acc[e]);
                        g[e] = rstd * (g[e] * w[e] - xh * m);
                    }
                }
                store8<OBF16>(yp + tok[t].out[x], g);
            }
        }
        if (!want) continue;
        if (SHARED) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                accq[e] += x == 0 ? acc[e] : 0.f;
                acck[e] += x == 0 ? 0.f : acc[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) red[(e * 4 + wave) * 64 + lane] = acc[e];
            __syncthreads();
            // (thread: channel e = tid / 32 of lanes tid % 32 and 32 more)
            for (int i = threadIdx.x; i < 64 * 8; i += kThreads) {
                const int e = i >> 6, l = i & 63, hh = g0 + l / LPR;
                if (hh < heads)
                    a.partial[((int64_t)blockIdx.x * heads + hh) * D + (l % LPR) * 8 + e] =
                        (red[(e * 4 + 0) * 64 + l] + red[(e * 4 + 1) * 64 + l]) + (red[(e * 4 + 2) * 64 + l] + red[(e * 4 + 3) * 64 + l]);
            }
            __syncthreads();
        }
    }
    if (SHARED && want) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            red[(e * 4 + wave) * 64 + lane] = accq[e];
            red[2048 + (e * 4 + wave) * 64 + lane] = acck[e];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
            const int x = i / D, c = i % D;
            float sum = 0.f;
            for (int r = 0; r < 4 * RPW; ++r) sum += red[x * 2048 + ((c & 7) * 4 + r / RPW) * 64 + (r % RPW) * LPR + c / 8];
            a.partial[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * D + i] = sum;
        }
    }
}

// Weight gradients: the columns of `rows` partial sums [rows, columns] added up in a fixed order.  A workgroup has 32 columns, a
// thread four of them and every 32nd row, eight rows in flight.  Columns are queries' heads, then keys' (shared: one of each).
__global__ void __launch_bounds__(kThreads)
qk_weight_kernel(const float *partial, int64_t rows, int columns, int q_columns, float *dwq, float *dwk)
{
    __shared__ __align__(16) float red[32][36];
    const int c = (threadIdx.x & 7) * 4, r0 = threadIdx.x >> 3;
    const float *p = partial + blockIdx.x * 32 + c;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int64_t r = r0; r < rows; r += 32 * 8) {
        float4 x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int64_t row = r + 32 * u;
            x[u] = *(const float4 *)(p + (row < rows ? row : r0) * columns);
            if (row >= rows) x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) { s.x += x[u].x; s.y += x[u].y; s.z += x[u].z; s.w += x[u].w; }
    }
    *(float4 *)&red[r0][c] = s;
    __syncthreads();
    if (threadIdx.x < 32) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) sum += red[i][threadIdx.x];
        const int col = blockIdx.x * 32 + threadIdx.x;
        float *dw = col < q_columns ? dwq : dwk;
        if (dw) dw[col < q_columns ? col : col - q_columns] = sum;
    }
}

}  // namespace

// Heads of a workgroup: all of them, or a share in whole groups where the tokens alone do not make 512 workgroups.
static int head_share(int64_t groups, int heads, int d)
{
    const int rows = 512 / d, pieces = (heads + rows - 1) / rows;            // heads of a group, groups
    int64_t parts = groups > 0 ? 512 / groups : 1;
    parts = parts < 1 ? 1 : parts > pieces ? pieces : parts;
    return (int)((pieces + parts - 1) / parts) * rows;
}

int64_t qk_backward_groups(int64_t tokens)
{
    const int64_t tile = back_tile(tokens);
    return (tokens + tile - 1) / tile;
}

size_t qk_partial_bytes(int64_t tokens, int heads, int d, int shared)
{
    const int64_t groups = qk_backward_groups(tokens);
    const int share = head_share(groups, heads, d);
    return (size_t)groups * (shared ? 2 * ((heads + share - 1) / share) : heads) * d * sizeof(float);
}

hipError_t launch_qk_backward(const QkArgs &a, hipStream_t s)
{
    const int64_t total = (int64_t)a.B * a.n, tile = back_tile(total), groups = qk_backward_groups(total);
    const bool want = a.norm && (a.dw[0] || a.dw[1]);
    const int heads = a.heads[0] + a.heads[1], share = head_share(groups, heads, a.d);
    QkArgs b = a;
    if (!want) b.partial = nullptr;
    if (groups > 0) {
        const dim3 grid((unsigned)groups, (unsigned)((heads + share - 1) / share)), block(kThreads);
#define LASAD_QK(I, O, D) (a.shared ? (void)(qk_backward_kernel<I, O, D, 1><<<grid, block, 0, s>>>(b, (int)tile, share)) \
                                    : (void)(qk_backward_kernel<I, O, D, 0><<<grid, block, 0, s>>>(b, (int)tile, share)))
#define LASAD_QK_D(I, O) (a.d == 32 ? LASAD_QK(I, O, 32) : a.d == 64 ? LASAD_QK(I, O, 64) : LASAD_QK(I, O, 128))
        if (a.io_dtype == LASAD_BF16) { if (a.out_dtype == LASAD_BF16) LASAD_QK_D(1, 1); else LASAD_QK_D(1, 0); }
        else LASAD_QK_D(0, 0);
#undef LASAD_QK_D
#undef LASAD_QK
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (want) {
        const int columns = (a.shared ? 2 : heads) * a.d;
        const int64_t rows = a.shared ? groups * ((heads + share - 1) / share) : groups;
        qk_weight_kernel<<<dim3(columns / 32), dim3(kThreads), 0, s>>>(a.partial, rows, columns, (a.shared ? 1 : a.heads[0]) * a.d,
                                                                 a.dw[0], a.dw[1]);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace lasad
