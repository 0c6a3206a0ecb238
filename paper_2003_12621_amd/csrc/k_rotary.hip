// Rotary positions over several axes: pair i of a head, which follows one of a
// token's coordinates p, is turned by the angle p * freqs[i].
//
// Bound by memory: every element is read and written once.  A workgroup takes
// a few tokens, computes their sines and cosines once into LDS (they serve
// all heads) and then streams the heads through in 16-byte accesses.  Measured:
// 4 x 16384 tokens of 40 heads of 64 (bf16) 135 us, 5.0 TB/s (a copy of 4 GiB
// reaches 4.8); 196 tokens of 32 heads of 32 (fp32) 3.4 to 3.9 us, a launch's latency.
#include "fftsplit_internal.hpp"
#include "launch_util.hpp"
#include "rotary.hpp"
#include "rotary_turn.hpp"

namespace fftsplit {

// N elements an access: 16 bytes' worth, or 1 where alignment does not allow that.
template <typename T, int N, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
    extern __shared__ float2 turns[];
    const long long token0 = (long long)blockIdx.x * a.block_tokens;
    const int tokens = int(min((long long)a.block_tokens, (long long)a.n * a.s - token0));
    for (int i = threadIdx.x; i < tokens * a.pairs; i += 256) {
        const int pair = i % a.pairs;
        const long long t = token0 + i / a.pairs;
        int axis = 0;
        while (axis + 1 < a.axes && pair >= a.section_end[axis]) ++axis;
        const long long b = t / a.s;
        const float2 cs = turn(a.positions[b * a.pos_batch + (t - b * a.s) * a.axes + axis], a.freqs[pair]);
        turns[i] = make_float2(cs.x, a.inverse ? -cs.y : cs.y);
    }
    __syncthreads();
    // items: pairs of N-element pieces (element i, i + pairs), or pieces of
    // N / 2 whole pairs (pairs of single elements where N = 1); then what is
    // not turned
    constexpr int kPiecePairs = INTERLEAVED && N > 1 ? N / 2 : N;
    const int turned = a.pairs / kPiecePairs, rest = a.copy_rest ? (a.d - 2 * a.pairs) / N : 0;
    const int per_head = turned + rest, heads = a.heads[0] + a.heads[1];
    for (int i = threadIdx.x; i < tokens * heads * per_head; i += 256) {
        const int piece = i % per_head, r = i / per_head;
        const int h = r % heads, tok = r / heads;
        const int which = h >= a.heads[0];
        const int head = which ? h - a.heads[0] : h;
        const long long t = token0 + tok, b = t / a.s, pos = t - b * a.s;
        const T* x = static_cast<const T*>(a.x[which]) + b * a.xs[which][0] + pos * a.xs[which][1] + head * a.xs[which][2];
        T* y = static_cast<T*>(a.y[which]) + b * a.ys[which][0] + pos * a.ys[which][1] + head * a.ys[which][2];
        using P = Pack<T, N>;
        if (piece >= turned) {
            const int e = 2 * a.pairs + (piece - turned) * N;
            *reinterpret_cast<P*>(y + e) = *reinterpret_cast<const P*>(x + e);
            continue;
        }
        const float2* cs = turns + tok * a.pairs + piece * kPiecePairs;
        if constexpr (INTERLEAVED && N > 1) {
            P u = *reinterpret_cast<const P*>(x + piece * N);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) {
                const float2 w = cs[j];
                const float p = float(u.v[2 * j]), q = float(u.v[2 * j + 1]);
                u.v[2 * j] = T(p * w.x - q * w.y);
                u.v[2 * j + 1] = T(q * w.x + p * w.y);
            }
            *reinterpret_cast<P*>(y + piece * N) = u;
        } else {
            const int e0 = INTERLEAVED ? 2 * piece : piece * N, e1 = INTERLEAVED ? e0 + 1 : e0 + a.pairs;
            P u = *reinterpret_cast<const P*>(x + e0), v = *reinterpret_cast<const P*>(x + e1);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float2 w = cs[j];
                const float p = float(u.v[j]), q = float(v.v[j]);
                u.v[j] = T(p * w.x - q * w.y);
                v.v[j] = T(q * w.x + p * w.y);
            }
            *reinterpret_cast<P*>(y + e0) = u;
            *reinterpret_cast<P*>(y + e1) = v;
        }
    }
}

namespace {
template <typename T, int N>
hipError_t launch_pieces(const RotaryArgs& a, hipStream_t s, const LaunchEvents& ev) {
    const long long blocks = ((long long)a.n * a.s + a.block_tokens - 1) / a.block_tokens;
    const unsigned lds = unsigned(a.block_tokens) * a.pairs * sizeof(float2);
    auto kernel = a.interleaved ? rotary_kernel<T, N, true> : rotary_kernel<T, N, false>;
    return launch_kernel(kernel, dim3(unsigned(blocks)), dim3(256), lds, s, ev.start, ev.stop, a);
}
}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s, const LaunchEvents& ev) {
    if (a.dtype == FFTSPLIT_BF16)
        return a.wide ? launch_pieces<__bf16, 8>(a, s, ev) : launch_pieces<__bf16, 1>(a, s, ev);
    return a.wide ? launch_pieces<float, 4>(a, s, ev) : launch_pieces<float, 1>(a, s, ev);
}

}  // namespace fftsplit
