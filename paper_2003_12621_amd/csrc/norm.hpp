// What the layer-norm kernels get.
#pragma once

#include "fftsplit_internal.hpp"

namespace fftsplit {

struct NormArgs {
    const void* x;
    void* y;
    const float *weight, *bias;      // null: 1 and 0
    float *mean, *rstd;              // written by the forward pass (or null), read by the backward pass
    const void* dy;
    void* dx;
    float *dweight, *dbias;
    float* part;                     // [workgroup][2][c]
    int n, s, c;
    int x_type, y_type;              // fftsplit_dtype_t of x and dx, of y and dy
    int x_first, y_first;            // channels first
    float eps;
    int wide;                        // 16-byte (channels last) or 4-element (channels first) accesses allowed
    int blocks;                      // workgroups of the backward pass
};

constexpr int kNormMaxLast = 8192;   // channels, last
constexpr int kNormMaxFirst = 2048;  // channels, first

// Workgroups of the backward pass, each with a partial sum per channel.
int norm_backward_blocks(int n, int s, bool first);
hipError_t launch_norm_forward(const NormArgs& a, hipStream_t s, const LaunchEvents& ev);
hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s, const LaunchEvents& ev);

}  // namespace fftsplit
