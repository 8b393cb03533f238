// Declarations shared by the kernels of the softmax layers (head norms with rotation, window attention) and their C ABI.
#pragma once

#include "lasad_internal.h"

namespace lasad {

// Status `code` with a message for lasad_last_error() (lasad_api.hip).
int fail(int code, const char *fmt, ...);
int hip_fail(const char *what, hipError_t e);

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
size_t qk_partial_bytes(int64_t tokens, int heads, int d, int shared);

}  // namespace lasad
