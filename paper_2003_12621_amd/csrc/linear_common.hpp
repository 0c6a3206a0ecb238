// Device helpers of the linear attention kernels.
#pragma once

#include "attn_tiles.hpp"
#include "launch_util.hpp"
#include "linear_internal.hpp"

namespace fftsplit {

// A value that is the same in all lanes, in a scalar register: quotients come from
// vector instructions, and what is derived from them would stay in vector ones,
// branches included.
__device__ __forceinline__ int linear_scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float linear_scalar(float x) {
    return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x)));
}

// A value at an address that is the same in all lanes, which no kernel writes while
// this one runs: by a scalar load.
template <typename V>
__device__ __forceinline__ V linear_uniform(const V* p) {
    return *(const __attribute__((address_space(4))) V*)(p);
}

// Tokens of sequence b that exist.
__device__ __forceinline__ int linear_length(const int* lengths, int s, int b) {
    if (!lengths) return s;
    const int l = linear_scalar(linear_uniform(lengths + b));
    return l < 0 ? 0 : (l > s ? s : l);
}

// Steps of 16 along a row that the kernels pad its width to.
__device__ __forceinline__ int linear_steps(int width) {
    return width <= 32 ? 2 : width <= 64 ? 4 : width <= 128 ? 8 : 16;
}

// log2 of a head's decay.  Values above 0 are taken as 0; below -10^4 nothing is
// left after one token, and 0 times it has to be 0.  NaN stays.
__device__ __forceinline__ float decay_log2(float log_decay) {
    float x = log_decay * 1.44269504088896341f;
    x = x > 0.f ? 0.f : x;
    return x < -1e4f ? -1e4f : x;
}

// decay^e (results below 2^-126 become zero).
__device__ __forceinline__ float decay_power(float log2_decay, int e) {
    return __builtin_amdgcn_exp2f(log2_decay * float(e));
}

// decay^e - 1, for x decay^e as x + x (decay^e - 1): a factor near 1, rounded to
// fp32, would be off by the same 2^-25 at every step, 3e-4 after 8192 tokens.
__device__ __forceinline__ float decay_less_one(float log2_decay, int e) {
    return expm1f(log2_decay * 0.693147180559945309f * float(e));
}

}  // namespace fftsplit
