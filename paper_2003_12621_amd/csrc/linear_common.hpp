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

// Half s of an accumulator as the operand of a product: fp32 as it is; in bf16 as the
// sum of two operands, good to 2^-15 of each value where one is good to 2^-8.  What
// later products take is held like this:
//   the states before the segments.  A state's largest terms are what keys and values
//   have in common, and a product may cancel just these: rounded once, a dq of values
//   with a mean of 4 and gradients that add up to zero was off by 4.5e-2, like this by
//   1.7e-3, which is its own rounding.  4 x 3136 training tokens of 8 heads of 64 / 128
//   142 us, so 152; 4 x 16384 tokens of 16 heads 374, so 405;
//   the scores with their decay: an error of 1.66e-3 of each term next to the output's
//   own 1.66e-3.  The former 152 us, so 157; the latter 405, so 412; 8 x 784 tokens of 8
//   heads, one segment, 27 us, so 32.
// (The upper part is cut off, not rounded, which takes fewer registers, and no finite
// value becomes infinite by it.)
template <typename T>
struct Precise {
    static constexpr int kParts = sizeof(T) == 2 ? 2 : 1;
    Operand<T> part[kParts];
    __device__ __forceinline__ void set(const floatx16& c, int s) {
        if constexpr (kParts == 1) {
            part[0] = acc_operand<T>(c, s);
        } else {
            u32x4 high, low;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = c[8 * s + 2 * e], b = c[8 * s + 2 * e + 1];
                high[e] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
                low[e] = pack_bf16(a - __uint_as_float(__float_as_uint(a) & 0xffff0000u),
                                   b - __uint_as_float(__float_as_uint(b) & 0xffff0000u));
            }
            part[0].v = __builtin_bit_cast(bf16x8, high);
            part[1].v = __builtin_bit_cast(bf16x8, low);
        }
    }
};

}  // namespace fftsplit
