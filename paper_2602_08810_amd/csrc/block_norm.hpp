// Host-visible parameter block and launcher declarations of the norms around a block.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lrnnx {

struct NormParams {
    int64_t M;                           // rows
    int D, groups, width;                // width: D / groups
    int post_shared;                     // post_weight has one group's width
    int io, res_io;                      // 1: bfloat16
    int gate_act;                        // 0: silu, 1: sigmoid
    float eps;
    const void *x, *gate, *res;
    int64_t x_s, gate_s, res_s;          // row strides
    const float *post, *scale, *pre;
    void *h, *y;                         // [M,D] contiguous
    // backward
    const void *dh, *dy;
    int64_t dh_s, dy_s;
    void *dx, *dgate, *dres;             // [M,D] contiguous
    float *dpost, *dscale, *dpre;
    float *sums;                         // [blocks, 3, D] partial sums of the three
    int blocks;
};

hipError_t launch_norm_fwd(const NormParams &p, hipStream_t s);
hipError_t launch_norm_bwd(NormParams p, hipStream_t s);
int norm_bwd_blocks(int64_t M, int D);

}  // namespace lrnnx
