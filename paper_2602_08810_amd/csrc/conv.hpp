// Host-visible parameter block and launcher declarations of the short causal convolution.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lrnnx {

struct ConvParams {
    int B, seqs, D, W;                   // B: batch entries in memory (1 of a packed batch), seqs: sequences
    int64_t L;
    int io, act, time_last;              // io 1: bfloat16; act 0: silu, 1: none; time_last: [B,D,L], else [B,L,D]
    const int64_t *cu;                   // boundaries of a packed batch, or null
    const void *x, *dy, *x0, *dx_last;   // x0, dx_last [seqs,W-1,D]
    int64_t x_b, x_l, x_d, dy_b, dy_l, dy_d;
    const float *w, *bias;               // [D,W], [D]
    void *y, *x_last;                    // outputs of the forward pass; y has y_*
    void *dx, *dx0;                      // and of the backward pass; dx has y_*
    int64_t y_b, y_l, y_d;
    float *dw, *db, *sums;               // sums [blocks,W+1,D]: parts of the weights' gradients
    int blocks;                          // workgroups along the time axis (backward: parts)
    int tile, tile_log2;                 // steps a thread walks, or (a power of two) the lanes of a row take, at a time
    int64_t tiles_each, tiles;           // tiles of a batch entry; in all (a packed time axis: slots)
    int shift;                           // log2 of a workgroup's threads side by side along the contiguous axis
};

hipError_t launch_conv_rows(const ConvParams &p, bool backward, hipStream_t s);
hipError_t launch_conv_time(const ConvParams &p, bool backward, hipStream_t s);
hipError_t launch_conv_sums(const ConvParams &p, hipStream_t s);
// Tiles, workgroups and shift of a call (host only; sizes decide).
void plan_conv(ConvParams &p, bool backward);

struct ConvStepParams {
    int B, D, W, io, act;
    const void *x; int64_t x_b, x_d;
    const float *w, *bias;
    void *state;                         // [B,W-1,D]
    void *y; int64_t y_b, y_d;
};
hipError_t launch_conv_step(const ConvStepParams &p, hipStream_t s);

}  // namespace lrnnx
