// Device helpers shared by the attention forward and backward kernels.
#pragma once

#include "attn_internal.hpp"
#include "attn_tiles.hpp"
#include "launch_util.hpp"

namespace fftsplit {

// Keys of sequence b that exist.
__device__ __forceinline__ int attn_length(const AttnArgs& a, int b) {
    if (!a.lengths) return a.sk;
    const int l = a.lengths[b];
    return l < 0 ? 0 : (l > a.sk ? a.sk : l);
}
// The last key that query row i sees (-1: none): causal rows are aligned to
// the end of the keys.
__device__ __forceinline__ int attn_last_key(const AttnArgs& a, int i, int length) {
    const int last = length - 1;
    if (!a.causal) return last;
    const int c = i + length - a.sq;
    return c < last ? (c < -1 ? -1 : c) : last;
}
__device__ __forceinline__ float attn_lambda(const AttnArgs& a, int h) {
    const int i = h * a.lam_step;
    return a.lam_f32 ? static_cast<const float*>(a.lam)[i] : float(static_cast<const __bf16*>(a.lam)[i]);
}

// Which tile, head and share of it a workgroup takes, of `parts` shares of
// `tiles` tiles of `heads` heads.  Neighbours share an XCD and its L2.  Under a
// causal mask tiles differ in length, and `place` counts from the longest: the
// heads of an XCD (as many as make 256 workgroups, which is at least as many as
// it runs at once) go through their tiles together, the longest first, and every
// other round of its 32 compute units backwards, so that a long and a short tile
// meet on a unit.  Head by head, longest first, 8192 tokens of 16 heads took 466
// us, not 433, and 2 x 1999 of 8 wide heads 104, not 87; every other head
// backwards, 536 and 90.
struct AttnPlace {
    int place, head, part;
};
__device__ __forceinline__ AttnPlace attn_place(const AttnArgs& a, int tiles, int heads, int parts) {
    const int id = xcd_logical_block(blockIdx.x, gridDim.x);
    int band = 1;
    if (a.causal) band = max(1, min(heads / kNumXcd, (256 + tiles * parts - 1) / (tiles * parts)));
    const int first = id / (band * tiles * parts) * band, n = min(band, heads - first);
    int i = id - first * tiles * parts;
    if (a.causal && (i & 32)) i = (i & ~31) + min(i | 31, n * tiles * parts - 1) - i;
    return {i / (n * parts), first + i / parts % n, i % parts};
}

// A value at an address that is the same in all lanes, written before this
// kernel started: by a scalar load, which the vector loads' count leaves out.
__device__ __forceinline__ float uniform_load(const float* p) {
    return *(const __attribute__((address_space(4))) float*)(p);
}

// 2^x by the hardware instruction (results below 2^-126 become zero: they are
// terms of a sum whose largest is about 1).
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace fftsplit
