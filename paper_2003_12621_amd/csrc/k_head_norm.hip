// Norm of every head by its root mean square, and rotation, in one pass; and the
// gradient of both.
//
// With r = 1 / sqrt(mean(x^2) + eps) and z = x r the forward pass is
// y = R (w z).  Backwards, u = R^T dy is the gradient behind the rotation, and
//     dx = r (w u - z mean(w u z)),    dw = sum over tokens and heads of u z,
// from x and dy alone: r is computed again from x, which has to be read anyway.
//
// Bound by memory: every element is read and written once.  A few lanes share a
// head: each takes two accesses' worth of elements that are turned into one
// another (or two neighbouring ones), so that the sums over the head are the
// only exchange, and a lane's elements are the same ones of every head, so that
// the weights' gradient stays in registers.  As in the rotation alone a
// workgroup computes its tokens' sines and cosines once for all heads.
#include "head_norm.hpp"
#include "launch_util.hpp"
#include "rotary_turn.hpp"

namespace fftsplit {

namespace {

constexpr int kThreads = 256;

// What a lane takes of a head: N elements from e0 and N from e1.
struct Piece {
    int e0, e1;
    bool turned, first, second;      // rotated; which of the two there are
};
template <int N, bool INTERLEAVED>
__device__ __forceinline__ Piece piece_of(const RotaryArgs& a, int i) {
    Piece p;
    const int turned = INTERLEAVED && N > 1 ? (2 * a.pairs / N + 1) / 2 : a.pairs / N;
    p.turned = i < turned;
    if (p.turned && !(INTERLEAVED && N > 1)) {
        p.e0 = INTERLEAVED ? 2 * i : i * N;
        p.e1 = INTERLEAVED ? p.e0 + 1 : p.e0 + a.pairs;
        p.first = p.second = true;
        return p;
    }
    const int start = p.turned ? 0 : 2 * a.pairs, end = p.turned ? 2 * a.pairs : a.d;
    p.e0 = start + 2 * N * (p.turned ? i : i - turned);
    p.e1 = p.e0 + N;
    p.first = p.e0 < end;
    p.second = p.e1 < end;
    return p;
}

template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p, bool there) {
    Pack<T, N> x;
#pragma unroll
    for (int j = 0; j < N; ++j) x.v[j] = T(0.f);
    if (there) x = *reinterpret_cast<const Pack<T, N>*>(p);
    return x;
}
template <typename T, int N>
__device__ __forceinline__ void widen(float (&u)[N], const Pack<T, N>& x) {
#pragma unroll
    for (int j = 0; j < N; ++j) u[j] = float(x.v[j]);
}
// A piece of x and (backwards) of dy, as they are in memory.
template <typename T, int N>
struct Loaded {
    Pack<T, N> u, v, gu, gv;
};
template <typename T, int N>
__device__ __forceinline__ void store_piece(T* p, const float (&u)[N], bool there) {
    Pack<T, N> x;
#pragma unroll
    for (int j = 0; j < N; ++j) x.v[j] = T(u[j]);
    if (there) *reinterpret_cast<Pack<T, N>*>(p) = x;
}

// Turns a lane's elements by the token's angles (BACK: by minus them).
template <int N, bool INTERLEAVED, bool BACK>
__device__ __forceinline__ void turn_piece(float (&u)[N], float (&v)[N], const Piece& p, const float2* cs) {
    if (!p.turned) return;
    auto by = [](float& x, float& y, float2 w) {
        const float s = BACK ? -w.y : w.y, t = x * w.x - y * s;
        y = y * w.x + x * s;
        x = t;
    };
    if constexpr (INTERLEAVED && N > 1) {
#pragma unroll
        for (int j = 0; j < N / 2; ++j) by(u[2 * j], u[2 * j + 1], cs[p.e0 / 2 + j]);
        if (p.second)
#pragma unroll
            for (int j = 0; j < N / 2; ++j) by(v[2 * j], v[2 * j + 1], cs[p.e1 / 2 + j]);
    } else {
        const float2* w = cs + (INTERLEAVED ? p.e0 / 2 : p.e0);
#pragma unroll
        for (int j = 0; j < N; ++j) by(u[j], v[j], w[j]);
    }
}

// The sum over the lanes that share a head.
__device__ __forceinline__ float head_sum(float x, int lanes) {
    for (int m = 1; m < lanes; m *= 2) x += __shfl_xor(x, m);
    return x;
}

// The angles of the tokens from token0 on, into LDS.
__device__ __forceinline__ void fill_turns(const HeadNormArgs& args, float2* turns, int token0, int tokens) {
    const RotaryArgs& a = args.r;
    for (int i = threadIdx.x; i < tokens * a.pairs; i += kThreads) {
        const int row = args.by_pairs.quotient(i), pair = i - row * a.pairs, t = token0 + row;
        int axis = 0;
        while (axis + 1 < a.axes && pair >= a.section_end[axis]) ++axis;
        const int b = args.by_s.quotient(t);
        turns[i] = turn(a.positions[b * a.pos_batch + (long long)(t - b * a.s) * a.axes + axis], a.freqs[pair]);
    }
}

}  // namespace

// ONE: a lane has one piece of a head, which it keeps in registers; else heads
// are so wide that 64 lanes take several pieces each, and read them again after
// the sums.  BACK: the gradients.
template <typename T, int N, bool INTERLEAVED, bool ONE, bool BACK>
__global__ __launch_bounds__(kThreads, BACK ? 4 : 6) void head_norm_kernel(HeadNormArgs a) {
    extern __shared__ float2 turns[];
    const RotaryArgs& r = a.r;
    const int lanes = a.row_lanes, part = threadIdx.x & (lanes - 1), group = threadIdx.x / lanes, groups = kThreads / lanes;
    const int all = r.n * r.s, token_groups = (all + r.block_tokens - 1) / r.block_tokens;
    // BACK: [groups][d] in place of the angles, for either tensor in turn; where
    // heads do not fit the registers, [2][groups][d] behind them
    float* sums = reinterpret_cast<float*>(ONE ? turns : turns + r.block_tokens * r.pairs);
    if constexpr (BACK && !ONE) {
        for (int i = threadIdx.x; i < 2 * groups * r.d; i += kThreads) sums[i] = 0.f;
    }
    float d0[2][N], d1[2][N];
    const Piece own = piece_of<N, INTERLEAVED>(r, part);
    auto load_weight = [&](float (&u)[N], float (&v)[N], int which, const Piece& p) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            u[j] = p.first && a.weight[which] ? a.weight[which][p.e0 + j] : 1.f;
            v[j] = p.second && a.weight[which] ? a.weight[which][p.e1 + j] : 1.f;
        }
    };
    // The weights stay in LDS, [2][d] behind the angles: in registers they cost waves
    // (4 x 16384 tokens of 32 + 8 heads of 64 in bf16 133 us, so 123; backwards of 4 x
    // 3136 tokens of 8 + 8 heads three waves a SIMD and 31 us, so four and 24).
    float* weights = reinterpret_cast<float*>(turns + r.block_tokens * r.pairs);
    auto kept_weight = [&](float (&u)[N], float (&v)[N], int which) {
        const auto x = *reinterpret_cast<const Pack<float, N>*>(weights + which * r.d + (own.first ? own.e0 : 0));
        const auto y = *reinterpret_cast<const Pack<float, N>*>(weights + which * r.d + (own.second ? own.e1 : 0));
#pragma unroll
        for (int j = 0; j < N; ++j) {
            u[j] = x.v[j];
            v[j] = y.v[j];
        }
    };
    if constexpr (ONE) {
        for (int i = threadIdx.x; i < 2 * r.d; i += kThreads) {
            const int which = i >= r.d;
            weights[i] = r.heads[which] && a.weight[which] ? a.weight[which][i - which * r.d] : 1.f;
        }
    }
    if constexpr (ONE) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
#pragma unroll
            for (int j = 0; j < N; ++j) d0[which][j] = d1[which][j] = 0.f;
        }
    }
    for (int tg = blockIdx.x; tg < token_groups; tg += gridDim.x) {
        const int token0 = tg * r.block_tokens, tokens = min(r.block_tokens, all - token0);
        // the rows of unit i of a tensor: x, dy (forwards x again) and the output
        struct Unit {
            const T *x, *in;
            T* out;
            int token;
        };
        auto unit = [&](int which, int i) {
            const int heads = r.heads[which], tok = a.by_heads[which].quotient(i), head = i - tok * heads, t = token0 + tok;
            const int b = a.by_s.quotient(t), pos = t - b * r.s;
            Unit w;
            w.token = tok;
            w.in = static_cast<const T*>(r.x[which]) + b * r.xs[which][0] + pos * r.xs[which][1] + head * r.xs[which][2];
            w.out = static_cast<T*>(r.y[which]) + b * r.ys[which][0] + pos * r.ys[which][1] + head * r.ys[which][2];
            w.x = w.in;
            if constexpr (BACK)
                w.x = static_cast<const T*>(a.x[which]) + b * a.xs[which][0] + pos * a.xs[which][1] + head * a.xs[which][2];
            return w;
        };
        auto fetch = [&](Loaded<T, N>& x, const Unit& w, const Piece& p) {
            x.u = load_pack<T, N>(w.x + p.e0, p.first);
            x.v = load_pack<T, N>(w.x + p.e1, p.second);
            if constexpr (BACK) {
                x.gu = load_pack<T, N>(w.in + p.e0, p.first);
                x.gv = load_pack<T, N>(w.in + p.e1, p.second);
            }
        };
        // The first rows are on their way while the angles are computed, the next ones
        // while one is worked on: 150 -> 133 us of the former.  (Backwards, with twice the
        // rows, it costs a wave a SIMD: 28 -> 32 us of the latter with its sums, and 29 -> 32
        // us of 5 x 4275 tokens of 6 + 3 heads of 40 in fp32.)
        Loaded<T, N> loaded[2];
        if constexpr (ONE && !BACK) {
#pragma unroll
            for (int which = 0; which < 2; ++which)
                if (r.heads[which]) fetch(loaded[which], unit(which, min(group, tokens * r.heads[which] - 1)), own);
        }
        if (BACK) __syncthreads();                   // (the last round's angles are no longer read)
        fill_turns(a, turns, token0, tokens);
        __syncthreads();
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const int count = tokens * r.heads[which];
            for (int first = 0; first < count; first += groups) {
                const int i = first + group;
                const Unit w = unit(which, min(i, count - 1));
                T* out = w.out;
                const float2* cs = turns + w.token * r.pairs;
                Loaded<T, N> x;
                if constexpr (ONE && !BACK) {
                    x = loaded[which];
                    if (first + groups < count) fetch(loaded[which], unit(which, min(i + groups, count - 1)), own);
                }
                if (i >= count) continue;
                float u[N], v[N], gu[N], gv[N];
                float square = 0.f, cross = 0.f;
                // one piece: its part of the sums over the head.  Backwards gu, gv
                // are the gradients behind the rotation.
                auto take = [&](const Piece& p, const float (&wu)[N], const float (&wv)[N]) {
                    if constexpr (!ONE || BACK) fetch(x, w, p);
                    widen(u, x.u);
                    widen(v, x.v);
                    if constexpr (BACK) {
                        widen(gu, x.gu);
                        widen(gv, x.gv);
                        turn_piece<N, INTERLEAVED, true>(gu, gv, p, cs);
                    }
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        square = fmaf(u[j], u[j], fmaf(v[j], v[j], square));
                        if constexpr (BACK) cross = fmaf(gu[j] * wu[j], u[j], fmaf(gv[j] * wv[j], v[j], cross));
                    }
                };
                float rstd = 0.f, mean = 0.f;
                auto give = [&](const Piece& p, const float (&wu)[N], const float (&wv)[N], float (&su)[N], float (&sv)[N]) {
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        u[j] *= rstd;
                        v[j] *= rstd;
                        if constexpr (BACK) {
                            su[j] = fmaf(gu[j], u[j], su[j]);
                            sv[j] = fmaf(gv[j], v[j], sv[j]);
                            u[j] = rstd * fmaf(-mean, u[j], gu[j] * wu[j]);
                            v[j] = rstd * fmaf(-mean, v[j], gv[j] * wv[j]);
                        } else {
                            u[j] *= wu[j];
                            v[j] *= wv[j];
                        }
                    }
                    if constexpr (!BACK) turn_piece<N, INTERLEAVED, false>(u, v, p, cs);
                    store_piece<T, N>(out + p.e0, u, p.first);
                    store_piece<T, N>(out + p.e1, v, p.second);
                };
                auto statistics = [&] {
                    rstd = 1.f / sqrtf(head_sum(square, lanes) / float(r.d) + a.eps);
                    if constexpr (BACK) mean = head_sum(cross, lanes) * rstd / float(r.d);
                };
                if constexpr (ONE) {
                    float wu[N], wv[N];
                    if constexpr (BACK) kept_weight(wu, wv, which);
                    take(own, wu, wv);
                    statistics();
                    if constexpr (!BACK) kept_weight(wu, wv, which);
                    give(own, wu, wv, d0[which], d1[which]);
                } else {
                    float wu[N], wv[N];
                    for (int k = part;; k += lanes) {
                        const Piece p = piece_of<N, INTERLEAVED>(r, k);
                        if (!p.first) break;
                        load_weight(wu, wv, which, p);
                        take(p, wu, wv);
                    }
                    statistics();
                    for (int k = part;; k += lanes) {
                        const Piece p = piece_of<N, INTERLEAVED>(r, k);
                        if (!p.first) break;
                        load_weight(wu, wv, which, p);
                        take(p, wu, wv);
                        float su[N], sv[N];
#pragma unroll
                        for (int j = 0; j < N; ++j) su[j] = sv[j] = 0.f;
                        give(p, wu, wv, su, sv);
                        if constexpr (BACK) {
                            float* s = sums + (which * groups + group) * r.d;
#pragma unroll
                            for (int j = 0; j < N; ++j) {
                                s[p.e0 + j] += su[j];
                                if (p.second) s[p.e1 + j] += sv[j];
                            }
                        }
                    }
                }
            }
        }
    }
    if constexpr (BACK) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (!a.dweight[which]) continue;
            const float* from = sums + (ONE ? 0 : which * groups * r.d);
            __syncthreads();
            if constexpr (ONE) {
                float* s = sums + group * r.d;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (own.first) s[own.e0 + j] = d0[which][j];
                    if (own.second) s[own.e1 + j] = d1[which][j];
                }
                __syncthreads();
            }
            // (slices of the groups side by side, where there are threads for them)
            float* partial = sums + (ONE ? 1 : 2) * groups * r.d;
            const int slices = kThreads / r.d > 1 ? kThreads / r.d : 1;
            const int slice = slices > 1 ? int(threadIdx.x) / r.d : 0;
            for (int i = threadIdx.x - slice * r.d; i < r.d && slice < slices; i += kThreads) {
                float sum = 0.f;
#pragma unroll 8
                for (int g = slice; g < groups; g += slices) sum += from[g * r.d + i];
                if (slices == 1)
                    a.part[(size_t(blockIdx.x) * 2 + which) * r.d + i] = sum;
                else
                    partial[threadIdx.x] = sum;
            }
            if (slices > 1) {
                __syncthreads();
                if (int(threadIdx.x) < r.d) {
                    float sum = 0.f;
                    for (int g = 0; g < slices; ++g) sum += partial[g * r.d + threadIdx.x];
                    a.part[(size_t(blockIdx.x) * 2 + which) * r.d + threadIdx.x] = sum;
                }
            }
        }
    }
}

// The weights' gradients from the workgroups' sums, in a fixed order: 8 columns a
// workgroup, 8 loads a lane in flight.
__global__ __launch_bounds__(1024) void head_norm_sum_kernel(HeadNormArgs a) {
    constexpr int kColumns = 8, kLanes = 1024 / kColumns, kAhead = 8;
    __shared__ float sums[kLanes][kColumns + 1];
    const int column = blockIdx.x * kColumns + threadIdx.x % kColumns, row = threadIdx.x / kColumns, width = 2 * a.r.d;
    float sum = 0.f;
    if (column < width && a.dweight[column / a.r.d])
        for (int i = row; i < a.blocks; i += kAhead * kLanes) {
            float v[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int at = i + j * kLanes;
                v[j] = a.part[size_t(at < a.blocks ? at : i) * width + column];
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) sum += i + j * kLanes < a.blocks ? v[j] : 0.f;
        }
    sums[row][threadIdx.x % kColumns] = sum;
    for (int half = kLanes / 2; half; half /= 2) {
        __syncthreads();
        if (row < half) sums[row][threadIdx.x % kColumns] += sums[row + half][threadIdx.x % kColumns];
    }
    if (row || column >= width) return;
    const int which = column / a.r.d;
    if (a.dweight[which]) a.dweight[which][column % a.r.d] = sums[0][threadIdx.x];
}

namespace {

template <typename T, int N, bool BACK>
hipError_t launch_pieces(const HeadNormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    const RotaryArgs& r = a.r;
    const bool one = a.row_lanes > 0;
    HeadNormArgs b = a;
    if (!one) b.row_lanes = 64;
    for (int i = 0; i < 2; ++i) b.by_heads[i] = fast_div(r.heads[i]);
    b.by_s = fast_div(r.s);
    b.by_pairs = fast_div(r.pairs);
    auto kernel = r.interleaved
                      ? (one ? head_norm_kernel<T, N, true, true, BACK> : head_norm_kernel<T, N, true, false, BACK>)
                      : (one ? head_norm_kernel<T, N, false, true, BACK> : head_norm_kernel<T, N, false, false, BACK>);
    const long long token_groups = ((long long)r.n * r.s + r.block_tokens - 1) / r.block_tokens;
    const int turns = r.block_tokens * r.pairs * 8, sums = BACK ? kThreads / b.row_lanes * r.d * 4 : 0;
    const int partial = BACK ? kThreads * 4 : 0;
    const int angles = turns + 2 * r.d * 4;
    const int lds = one ? (angles > sums + partial ? angles : sums + partial) : turns + 2 * sums + partial;
    if (hipError_t e = allow_dynamic_lds(kernel, lds)) return e;
    return launch_kernel(kernel, dim3(unsigned(BACK ? a.blocks : token_groups)), dim3(kThreads), unsigned(lds), s, ev.start,
                         ev.stop, b);
}

template <bool BACK>
hipError_t launch_typed(const HeadNormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    if (a.r.dtype == FFTSPLIT_BF16) {
        switch (a.access) {
            case 8: return launch_pieces<__bf16, 8, BACK>(a, s, ev);
            case 4: return launch_pieces<__bf16, 4, BACK>(a, s, ev);
            case 2: return launch_pieces<__bf16, 2, BACK>(a, s, ev);
            default: return launch_pieces<__bf16, 1, BACK>(a, s, ev);
        }
    }
    switch (a.access) {
        case 4: return launch_pieces<float, 4, BACK>(a, s, ev);
        case 2: return launch_pieces<float, 2, BACK>(a, s, ev);
        default: return launch_pieces<float, 1, BACK>(a, s, ev);
    }
}

}  // namespace

hipError_t launch_head_norm(const HeadNormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    return launch_typed<false>(a, s, ev);
}

hipError_t launch_head_norm_backward(const HeadNormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    if (!a.dweight[0] && !a.dweight[1]) return launch_typed<true>(a, s, ev);
    if (hipError_t e = launch_typed<true>(a, s, LaunchEvents{ev.start, nullptr})) return e;
    return launch_kernel(head_norm_sum_kernel, dim3(unsigned((2 * a.r.d + 7) / 8)), dim3(1024), 0, s, nullptr, ev.stop, a);
}

}  // namespace fftsplit
