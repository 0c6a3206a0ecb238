// What the rotary kernel gets.
#pragma once

#include "fftsplit_internal.hpp"

namespace fftsplit {

struct RotaryArgs {
    const void* x[2];
    void* y[2];
    long long xs[2][3], ys[2][3];    // batch, token, head strides in elements
    int heads[2];
    const int* positions;
    long long pos_batch;             // elements between sequences' positions, 0: shared
    const float* freqs;
    int n, s, d, pairs, axes;
    int section_end[FFTSPLIT_ROTARY_MAX_AXES];
    int inverse, interleaved, dtype;
    int copy_rest;                   // elements that are not turned have to be copied
    int wide;                        // 16-byte accesses allowed
    int block_tokens;
};

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s, const LaunchEvents& ev);

}  // namespace fftsplit
