// Device parts of the kernels that rotate heads.
#pragma once

#include <hip/hip_runtime.h>

namespace fftsplit {

// cos and sin of p * f.  In fp32 the product alone would be off by p f / 2^24
// (1e-3 rad at p f = 2^14); quarter turns are taken off in 64 bits, whose few
// operations serve all heads of a token.
__device__ __forceinline__ float2 turn(int p, float f) {
    const double quarters = double(p) * double(f) * 0.63661977236758134308;   // 2 / pi
    const double whole = rint(quarters);
    float s, c;
    sincospif(float(quarters - whole) * 0.5f, &s, &c);
    const int q = int(whole - 4.0 * floor(whole * 0.25));
    const float c1 = (q & 1) ? -s : c, s1 = (q & 1) ? c : s;
    return (q & 2) ? make_float2(-c1, -s1) : make_float2(c1, s1);
}

template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
    T v[N];
};

}  // namespace fftsplit
