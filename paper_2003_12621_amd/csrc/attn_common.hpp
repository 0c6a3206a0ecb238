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

// A value at an address that is the same in all lanes, written before this
// kernel started: by a scalar load, which the vector loads' count leaves out.
__device__ __forceinline__ float uniform_load(const float* p) {
    return *(const __attribute__((address_space(4))) float*)(p);
}

// 2^x by the hardware instruction (results below 2^-126 become zero: they are
// terms of a sum whose largest is about 1).
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace fftsplit
