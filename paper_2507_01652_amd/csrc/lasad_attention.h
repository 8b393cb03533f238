// Declarations shared by the kernels of the softmax layers (head norms with rotation, window attention) and their C ABI.
#pragma once

#include "lasad_internal.h"

namespace lasad {

// Status `code` with a message for lasad_last_error() (lasad_api.hip).
int fail(int code, const char *fmt, ...);
int hip_fail(const char *what, hipError_t e);

// Workgroups of 256 threads that a launch may have: HIP takes fewer than 2^32 threads along an axis.  What a call would launch is
// counted (the *_groups functions) before anything is.
constexpr int64_t kMostGroups = ((int64_t)1 << 24) - 1;

// Head norms and rotation; [0] queries, [1] keys.
struct QkArgs {
    const void *x[2];
    const void *dy[2];                 // backward: gradients of the outputs
    void *y[2];                        // outputs (backward: gradients of the inputs)
    const float *w[2];                 // [heads, d], shared: [d], or NULL (ones)
    lasad_layout_t in[2], dl[2], out[2];
    int heads[2];
    int io_dtype, out_dtype, B, n, d;  // B * n < 2^31
    int start_pos, grid_w, last_pos;   // positions 0 .. last_pos - 1 are on the grid
    const int32_t *pos_rows;           // position of token 0 of every batch row instead of start_pos, or NULL
    int rope, pairing;
    double log2_base;
    int norm, shared;
    float eps;
    float *dw[2];                      // backward: weight gradients laid out like the weights (per head without one), or NULL
    float *partial;                    // backward: qk_partial_bytes of workspace
};
hipError_t launch_qk_forward(const QkArgs &a, hipStream_t s);
hipError_t launch_qk_backward(const QkArgs &a, hipStream_t s);
int64_t qk_forward_groups(int64_t tokens, int d);
int64_t qk_backward_groups(int64_t tokens);
size_t qk_partial_bytes(int64_t tokens, int heads, int d, int shared);

// Attention with a window and sinks.  Key j is seen from position p if j <= p, j < length of the batch row, and
// p - j < window or j < sinks.
struct WindowArgs {
    const void *q, *k, *v, *d_o;
    void *o, *dq, *dk, *dv;
    float *lse;                        // [B, Hq, n]: written by the forward (or NULL), read by the backward
    lasad_layout_t lq, lk, lv, lo, ldo, ldq, ldk, ldv;
    int io_dtype, out_dtype, B, Hq, Hk, d, n, m;       // n queries from position start_pos on, m keys from 0 on
    int start_pos, window, sinks;
    const int32_t *lens;               // valid keys of the batch rows, or NULL: m
    float scale;
    float *delta;                      // backward workspace: [B, Hq, n] rows' sums of d_o o
    float *parts;                      // backward workspace: partial dk and dv of the sinks' key tiles
    int key_tile, sink_tiles, sink_parts;              // plan of the backward's key pass: keys of a tile, tiles with sinks, parts of each
};
hipError_t launch_window_forward(const WindowArgs &a, hipStream_t s);
hipError_t launch_window_forward_16(const WindowArgs &a, hipStream_t s);
hipError_t launch_window_backward(WindowArgs &a, void *workspace, hipStream_t s);
int64_t window_forward_groups(const WindowArgs &a);
int64_t window_backward_groups(const WindowArgs &a);           // of the pass that has more
hipError_t launch_window_dq_few(const WindowArgs &a, hipStream_t s);
hipError_t launch_window_dkv_few(const WindowArgs &a, hipStream_t s);
constexpr int kWindowKeyTile = 64;     // keys of a workgroup of launch_window_dkv_bf16
hipError_t launch_window_dkv_bf16(const WindowArgs &a, hipStream_t s);
hipError_t launch_window_dq_bf16(const WindowArgs &a, hipStream_t s);
size_t window_backward_bytes(int B, int Hq, int Hk, int d, int n, int m, int window, int sinks);

// One token against a cache [B, Hk, cap, d]: key j lies in row j < sinks ? j : sinks + (j - sinks) mod (cap - sinks).
struct WindowStepArgs {
    const void *q, *k, *v;
    void *o, *k_cache, *v_cache;
    int io_dtype, out_dtype, B, Hq, Hk, d, cap;
    int pos;
    const int32_t *pos_rows;
    int window, sinks;
    float scale;
    float *parts;                      // workspace of splits
    int splits;
};
int window_step_splits(int B, int Hk, int64_t seen);
size_t window_step_bytes(int B, int Hq, int d, int splits);
hipError_t launch_window_step(const WindowStepArgs &a, hipStream_t s);

}  // namespace lasad
