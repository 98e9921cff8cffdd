// Host-visible parameter blocks and launcher declarations of the norm and the clipping of many tensors.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lrnnx {

// Tensors of one launch, passed by value: a captured graph keeps them, nothing is copied to the device.
constexpr int kGradTensors = 128;
struct GradList {
    const void *g[kGradTensors];
    void *out[kGradTensors];
    int64_t n[kGradTensors];             // elements
    uint32_t first[kGradTensors + 1];    // first piece (workgroup) of a tensor in this launch; behind the last one their number
    uint8_t io[kGradTensors];            // 1: bfloat16; 2: the output is
    int count, piece;                    // tensors; elements of a piece
    uint32_t base;                       // pieces of the launches before
};
static_assert(sizeof(GradList) <= 4000, "arguments of a launch");

hipError_t launch_grad_squares(const GradList &l, double *sums, hipStream_t s);
hipError_t launch_grad_total(const double *sums, uint32_t count, float *norm, hipStream_t s);
hipError_t launch_grad_scale(const GradList &l, const float *norm, float max_norm, float eps, bool in_place, hipStream_t s);

}  // namespace lrnnx
