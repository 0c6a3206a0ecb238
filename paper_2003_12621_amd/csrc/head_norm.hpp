// What the kernels of the head norms get.
#pragma once

#include "launch_util.hpp"
#include "rotary.hpp"

namespace fftsplit {

struct HeadNormArgs {
    // x (forward) or dy (backward) -> y or dx; inverse, copy_rest and wide are not used
    RotaryArgs r;
    const void* x[2];                // backward: the forward pass's input
    long long xs[2][3];
    const float* weight[2];          // or null: 1
    float* dweight[2];               // or null: not computed
    float* part;                     // [blocks][2][d]: the sums of each workgroup
    float eps;
    int access;                      // elements an access: 16 bytes' worth, or fewer where alignment asks for it
    int row_lanes;                   // lanes that share a head (a power of two), or 0: 64 with several pieces each
    int blocks;                      // workgroups of the backward kernel
    FastDiv by_heads[2], by_s, by_pairs;
};

// Workgroups of the backward kernel at most: each keeps the weights' sums of its share
// (of 4 x 3136 tokens of 8 + 8 heads of 64: 784 workgroups 24 us, 1568 29).
constexpr int kHeadNormBlocks = 1024;

hipError_t launch_head_norm(const HeadNormArgs& a, hipStream_t s, const LaunchEvents& ev);
hipError_t launch_head_norm_backward(const HeadNormArgs& a, hipStream_t s, const LaunchEvents& ev);

}  // namespace fftsplit
