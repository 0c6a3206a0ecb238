// Layer norm over the channels of tokens (channels last) or of a feature map
// (channels first, as the convolutions give and take), forward and backward.
//
// All are bound by memory: x is read once and kept in registers between the
// mean, the squared deviations and the output (two passes over registers, so
// that a large mean costs no precision); the backward pass keeps x and dy
// likewise.  The gradients of weight and bias are summed in registers over all
// rows that a workgroup takes, written once per workgroup, and added up by a
// second kernel in a fixed order.
//
// Measured: 32 x 256 channels of 56 x 56 (fp32, first) 45 us, 4.6 TB/s; 32 x 784
// tokens of 1024 channels (bf16) forward 20 us, 5.1 TB/s, backward 30 us, 5.1 TB/s
// (a copy of 4 GiB reaches 4.8; part of these fits the caches), and 4 us for the
// sum of the parts.
#include "launch_util.hpp"
#include "norm.hpp"

namespace fftsplit {

namespace {

template <typename T, int N>
struct alignas((sizeof(T) * N) > 16 ? 16 : sizeof(T) * N) Vec {
    T v[N];
};

// N consecutive elements, 1 or a multiple of 16 bytes (8 for 4 bf16) aligned to it.
template <typename T, int N>
__device__ __forceinline__ void load_n(float (&y)[N], const T* p) {
    const Vec<T, N> u = *reinterpret_cast<const Vec<T, N>*>(p);
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = float(u.v[j]);
}
template <typename T, int N>
__device__ __forceinline__ void store_n(T* p, const float (&y)[N]) {
    Vec<T, N> u;
#pragma unroll
    for (int j = 0; j < N; ++j) u.v[j] = T(y[j]);
    *reinterpret_cast<Vec<T, N>*>(p) = u;
}

// N values of a parameter, `or_else` where there is none.
template <int N>
__device__ __forceinline__ void load_param(float (&y)[N], const float* p, int c, float or_else) {
    if (p) {
        load_n<float, N>(y, p + c);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = or_else;
    }
}

// Sum over the G lanes (or, G = 256, threads of the workgroup) of a row, the same in all.
template <int G>
__device__ __forceinline__ float row_sum(float x, float* lds) {
#pragma unroll
    for (int m = 1; m < (G < 64 ? G : 64); m *= 2) x += __shfl_xor(x, m, 64);
    if constexpr (G == 256) {
        if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
        __syncthreads();
        x = lds[0] + lds[1] + lds[2] + lds[3];
        __syncthreads();
    }
    return x;
}

}  // namespace

// ---- channels last: G threads a row, NV pieces of N elements a thread, piece
// i of thread l at element (i G + l) N.  A row stays in the registers of one
// group of lanes; the group is the smallest that holds it, so that a workgroup
// has many rows in flight. ----

template <typename TX, typename TY, int G, int NV, int N>
__global__ __launch_bounds__(256) void norm_last_forward_kernel(NormArgs a) {
    __shared__ float lds[4];
    const int l = threadIdx.x % G;
    const long long rows = (long long)a.n * a.s, row = (long long)blockIdx.x * (256 / G) + threadIdx.x / G;
    if (row >= rows) return;      // (G = 256: the same for the whole workgroup)
    const TX* x = static_cast<const TX*>(a.x) + row * a.c;
    float v[NV][N];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * G + l) * N;
        if (c < a.c) {
            load_n<TX, N>(v[i], x + c);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) v[i][j] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < N; ++j) sum += v[i][j];
    }
    const float mean = row_sum<G>(sum, lds) / float(a.c);
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if ((i * G + l) * N < a.c)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                v[i][j] -= mean;
                sum = fmaf(v[i][j], v[i][j], sum);
            }
    const float rstd = 1.f / sqrtf(row_sum<G>(sum, lds) / float(a.c) + a.eps);
    TY* y = static_cast<TY*>(a.y) + row * a.c;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * G + l) * N;
        if (c >= a.c) continue;
        float w[N], b[N], o[N];
        load_param<N>(w, a.weight, c, 1.f);
        load_param<N>(b, a.bias, c, 0.f);
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] = fmaf(v[i][j] * rstd, w[j], b[j]);
        store_n<TY, N>(y + c, o);
    }
    if (a.mean && l == 0) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
}

template <typename TX, typename TY, int G, int NV, int N>
__global__ __launch_bounds__(256) void norm_last_backward_kernel(NormArgs a) {
    constexpr int kRows = 256 / G;
    extern __shared__ float lds[];     // [kRows][2][c] at the end; 4 floats in between
    const int l = threadIdx.x % G, group = threadIdx.x / G;
    const long long rows = (long long)a.n * a.s;
    float dw[NV][N], db[NV][N];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) dw[i][j] = db[i][j] = 0.f;
    const float inv_c = 1.f / float(a.c);
    for (long long row = (long long)blockIdx.x * kRows + group; row < rows; row += (long long)gridDim.x * kRows) {
        const TX* x = static_cast<const TX*>(a.x) + row * a.c;
        const TY* g = static_cast<const TY*>(a.dy) + row * a.c;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float v[NV][N], u[NV][N];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * G + l) * N;
            if (c >= a.c) continue;
            load_n<TX, N>(v[i], x + c);
            load_n<TY, N>(u[i], g + c);
            float w[N];
            load_param<N>(w, a.weight, c, 1.f);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                v[i][j] = (v[i][j] - mean) * rstd;
                db[i][j] += u[i][j];
                dw[i][j] = fmaf(u[i][j], v[i][j], dw[i][j]);
                u[i][j] *= w[j];
                s1 += u[i][j];
                s2 = fmaf(u[i][j], v[i][j], s2);
            }
        }
        s1 = row_sum<G>(s1, lds) * inv_c;
        s2 = row_sum<G>(s2, lds) * inv_c;
        TX* dx = static_cast<TX*>(a.dx) + row * a.c;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * G + l) * N;
            if (c >= a.c) continue;
            float o[N];
#pragma unroll
            for (int j = 0; j < N; ++j) o[j] = rstd * (u[i][j] - s1 - v[i][j] * s2);
            store_n<TX, N>(dx + c, o);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int c = (i * G + l) * N + j;
            if (c < a.c) {
                lds[(group * 2 + 0) * a.c + c] = dw[i][j];
                lds[(group * 2 + 1) * a.c + c] = db[i][j];
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.c; i += 256) {
        float t = 0.f;
        for (int r = 0; r < kRows; ++r) t += lds[r * 2 * a.c + i];
        a.part[(size_t)blockIdx.x * 2 * a.c + i] = t;
    }
}

// ---- channels first: LP threads side by side take VP positions each, NT / LP
// threads above one another take every (NT / LP)-th channel, NH of them ----

namespace {

// Sum over the channel rows of a workgroup, per position, the same in all threads.
template <int NT, int LP, int VP, int K>
__device__ __forceinline__ void column_sum(float (&x)[K][VP], float* lds) {
    constexpr int kRows = NT / LP, kPos = LP * VP;
    const int lp = threadIdx.x % LP, cr = threadIdx.x / LP;
    // rows of one wave by lane exchange, then waves through LDS
    constexpr int kWaveRows = LP < 64 ? 64 / LP : 1, kGroups = kRows / kWaveRows;
#pragma unroll
    for (int m = LP; m < 64; m *= 2)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int p = 0; p < VP; ++p) x[k][p] += __shfl_xor(x[k][p], m, 64);
    if (cr % kWaveRows == 0)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int p = 0; p < VP; ++p) lds[(cr / kWaveRows * K + k) * kPos + lp * VP + p] = x[k][p];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int p = 0; p < VP; ++p) {
            float t = 0.f;
#pragma unroll
            for (int r = 0; r < kGroups; ++r) t += lds[(r * K + k) * kPos + lp * VP + p];
            x[k][p] = t;
        }
    __syncthreads();
}

// Channels that pass through LDS at a time between a map's and the tokens' layout.
constexpr int kSwapChannels = 64;

template <int NT, int LP, int VP>
struct FirstShape {
    static constexpr int kRows = NT / LP, kPos = LP * VP;
    static constexpr int kSteps = kRows >= kSwapChannels ? 1 : kSwapChannels / kRows;   // channel steps a swap holds
    static constexpr int kSwap = kSteps * kRows;
    static constexpr int kPitch = kSwap + 1;
    static constexpr int kSumFloats = (LP < 64 ? NT / 64 : kRows) * 2 * kPos;
    static constexpr int lds(bool swap) {
        const int a = kSumFloats * 4, b = swap ? kPos * kPitch * 4 : 0;
        return a > b ? a : b;
    }
};

// VP consecutive positions of the channels of a thread: channel i of NH at
// base + i * step, of which those below `channels` exist, and of the positions
// `count`; all others are zero.  `base` is the same for the workgroup, `off` (in
// elements) the lane's, so that an access needs no 64-bit lane address.  fp32
// rows need no alignment: 16-byte accesses to memory ask for 4.
template <typename T, int VP>
struct alignas(sizeof(T) == 4 ? 4 : sizeof(T) * VP) Positions {
    T v[VP];
};
template <typename T, int VP, int NH>
__device__ __forceinline__ void load_positions(float (&y)[NH][VP], const T* base, size_t step, unsigned off, int count,
                                               int channels) {
#pragma unroll
    for (int i = 0; i < NH; ++i)
#pragma unroll
        for (int j = 0; j < VP; ++j) y[i][j] = 0.f;
    if (count == VP) {
#pragma unroll
        for (int i = 0; i < NH; ++i)
            if (i < channels) {
                const char* p = reinterpret_cast<const char*>(base + i * step) + off * unsigned(sizeof(T));
                const Positions<T, VP> u = *reinterpret_cast<const Positions<T, VP>*>(p);
#pragma unroll
                for (int j = 0; j < VP; ++j) y[i][j] = float(u.v[j]);
            }
    } else if (count > 0) {      // the last positions of a row
#pragma unroll
        for (int i = 0; i < NH; ++i)
#pragma unroll
            for (int j = 0; j < VP; ++j)
                if (i < channels && j < count) y[i][j] = float((base + i * step)[off + j]);
    }
}
template <typename T, int VP, int NH>
__device__ __forceinline__ void store_positions(T* base, size_t step, unsigned off, const float (&y)[NH][VP], int count,
                                                int channels) {
    if (count == VP) {
#pragma unroll
        for (int i = 0; i < NH; ++i)
            if (i < channels) {
                Positions<T, VP> u;
#pragma unroll
                for (int j = 0; j < VP; ++j) u.v[j] = T(y[i][j]);
                char* p = reinterpret_cast<char*>(base + i * step) + off * unsigned(sizeof(T));
                *reinterpret_cast<Positions<T, VP>*>(p) = u;
            }
    } else if (count > 0) {
#pragma unroll
        for (int i = 0; i < NH; ++i)
#pragma unroll
            for (int j = 0; j < VP; ++j)
                if (i < channels && j < count) (base + i * step)[off + j] = T(y[i][j]);
    }
}

}  // namespace

template <typename TX, typename TY, int NT, int LP, int VP, int NH, bool SWAP>
__global__ __launch_bounds__(NT) void norm_first_forward_kernel(NormArgs a) {
    using Shape = FirstShape<NT, LP, VP>;
    extern __shared__ float lds[];
    const int lp = threadIdx.x % LP, cr = threadIdx.x / LP;
    const int tiles = (a.s + Shape::kPos - 1) / Shape::kPos;
    const int b = blockIdx.x / tiles, pos0 = blockIdx.x % tiles * Shape::kPos, pos = pos0 + lp * VP;
    const int count = max(0, min(VP, a.s - pos));       // positions of this thread that exist
    const size_t at = (size_t)b * a.c * a.s + pos0, step = (size_t)Shape::kRows * a.s;
    const unsigned off = unsigned(cr * a.s + lp * VP);
    const int channels = (a.c - cr + Shape::kRows - 1) / Shape::kRows;   // of this thread's that exist
    float v[NH][VP];
    float sum[1][VP];
    load_positions<TX, VP, NH>(v, static_cast<const TX*>(a.x) + at, step, off, count, channels);
#pragma unroll
    for (int p = 0; p < VP; ++p) sum[0][p] = 0.f;
#pragma unroll
    for (int i = 0; i < NH; ++i)
#pragma unroll
        for (int p = 0; p < VP; ++p) sum[0][p] += v[i][p];
    column_sum<NT, LP, VP, 1>(sum, lds);
    float mean[VP], rstd[VP];
#pragma unroll
    for (int p = 0; p < VP; ++p) {
        mean[p] = sum[0][p] / float(a.c);
        sum[0][p] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < NH; ++i)
        if (cr + i * Shape::kRows < a.c)
#pragma unroll
            for (int p = 0; p < VP; ++p) {
                v[i][p] -= mean[p];
                sum[0][p] = fmaf(v[i][p], v[i][p], sum[0][p]);
            }
    column_sum<NT, LP, VP, 1>(sum, lds);
#pragma unroll
    for (int p = 0; p < VP; ++p) rstd[p] = 1.f / sqrtf(sum[0][p] / float(a.c) + a.eps);
    if (a.mean && cr == 0)
#pragma unroll
        for (int p = 0; p < VP; ++p)
            if (p < count) {
                a.mean[(size_t)b * a.s + pos + p] = mean[p];
                a.rstd[(size_t)b * a.s + pos + p] = rstd[p];
            }
#pragma unroll
    for (int i = 0; i < NH; ++i) {
        const int c = cr + i * Shape::kRows;
        const float w = a.weight && c < a.c ? a.weight[c] : 1.f, bias = a.bias && c < a.c ? a.bias[c] : 0.f;
#pragma unroll
        for (int p = 0; p < VP; ++p) v[i][p] = fmaf(v[i][p] * rstd[p], w, bias);
    }
    if constexpr (!SWAP) {
        store_positions<TY, VP, NH>(static_cast<TY*>(a.y) + at, step, off, v, count, channels);
    } else {
        TY* y = static_cast<TY*>(a.y) + ((size_t)b * a.s + pos0) * a.c;
        const int positions = min(Shape::kPos, a.s - pos0);
#pragma unroll
        for (int i0 = 0; i0 < NH; i0 += Shape::kSteps) {
            const int c0 = i0 * Shape::kRows;
            if (c0 >= a.c) break;
#pragma unroll
            for (int i = 0; i < Shape::kSteps; ++i)
                if (i0 + i < NH)
#pragma unroll
                    for (int p = 0; p < VP; ++p)
                        lds[(lp * VP + p) * Shape::kPitch + i * Shape::kRows + cr] = v[i0 + i < NH ? i0 + i : 0][p];
            __syncthreads();
            const int width = min(Shape::kSwap, a.c - c0);
            for (int e = threadIdx.x; e < positions * Shape::kSwap; e += NT) {
                const int p = e / Shape::kSwap, c = e % Shape::kSwap;
                if (c < width) y[(size_t)p * a.c + c0 + c] = TY(lds[p * Shape::kPitch + c]);
            }
            __syncthreads();
        }
    }
}

template <typename TX, typename TY, int NT, int LP, int VP, int NH, bool SWAP>
__global__ __launch_bounds__(NT) void norm_first_backward_kernel(NormArgs a) {
    using Shape = FirstShape<NT, LP, VP>;
    extern __shared__ float lds[];
    const int lp = threadIdx.x % LP, cr = threadIdx.x / LP;
    const int tiles = (a.s + Shape::kPos - 1) / Shape::kPos;
    const size_t step = (size_t)Shape::kRows * a.s;
    const unsigned off = unsigned(cr * a.s + lp * VP);
    const float inv_c = 1.f / float(a.c);
    const int channels = (a.c - cr + Shape::kRows - 1) / Shape::kRows;
    float dw[NH], db[NH];
#pragma unroll
    for (int i = 0; i < NH; ++i) dw[i] = db[i] = 0.f;
    for (long long tile = blockIdx.x; tile < (long long)a.n * tiles; tile += gridDim.x) {
        const int b = int(tile / tiles), pos0 = int(tile % tiles) * Shape::kPos, pos = pos0 + lp * VP;
        const int count = max(0, min(VP, a.s - pos));
        const size_t at = (size_t)b * a.c * a.s + pos0;
        float v[NH][VP], u[NH][VP];
        float mean[VP], rstd[VP], sum[2][VP];
#pragma unroll
        for (int p = 0; p < VP; ++p) {
            mean[p] = p < count ? a.mean[(size_t)b * a.s + pos + p] : 0.f;
            rstd[p] = p < count ? a.rstd[(size_t)b * a.s + pos + p] : 0.f;
            sum[0][p] = sum[1][p] = 0.f;
        }
        load_positions<TX, VP, NH>(v, static_cast<const TX*>(a.x) + at, step, off, count, channels);
        if constexpr (!SWAP) {
            load_positions<TY, VP, NH>(u, static_cast<const TY*>(a.dy) + at, step, off, count, channels);
        } else {
#pragma unroll
            for (int i = 0; i < NH; ++i)
#pragma unroll
                for (int p = 0; p < VP; ++p) u[i][p] = 0.f;
        }
        if constexpr (SWAP) {
            const TY* g = static_cast<const TY*>(a.dy) + ((size_t)b * a.s + pos0) * a.c;
            const int positions = min(Shape::kPos, a.s - pos0);
#pragma unroll
            for (int i0 = 0; i0 < NH; i0 += Shape::kSteps) {
                const int c0 = i0 * Shape::kRows;
                if (c0 >= a.c) break;
                const int width = min(Shape::kSwap, a.c - c0);
                __syncthreads();
                for (int e = threadIdx.x; e < positions * Shape::kSwap; e += NT) {
                    const int p = e / Shape::kSwap, c = e % Shape::kSwap;
                    if (c < width) lds[p * Shape::kPitch + c] = float(g[(size_t)p * a.c + c0 + c]);
                }
                __syncthreads();
#pragma unroll
                for (int i = 0; i < Shape::kSteps; ++i)
                    if (i0 + i < NH && c0 + i * Shape::kRows + cr < a.c)
#pragma unroll
                        for (int p = 0; p < VP; ++p)
                            u[i0 + i < NH ? i0 + i : 0][p] =
                                p < count ? lds[(lp * VP + p) * Shape::kPitch + i * Shape::kRows + cr] : 0.f;
            }
            __syncthreads();
        }
        // (positions and channels that do not exist have rstd or dy zero: no terms)
#pragma unroll
        for (int i = 0; i < NH; ++i) {
            const int c = cr + i * Shape::kRows;
            const float w = a.weight && c < a.c ? a.weight[c] : 1.f;
#pragma unroll
            for (int p = 0; p < VP; ++p) {
                v[i][p] = (v[i][p] - mean[p]) * rstd[p];
                db[i] += u[i][p];
                dw[i] = fmaf(u[i][p], v[i][p], dw[i]);
                u[i][p] *= w;
                sum[0][p] += u[i][p];
                sum[1][p] = fmaf(u[i][p], v[i][p], sum[1][p]);
            }
        }
        column_sum<NT, LP, VP, 2>(sum, lds);
#pragma unroll
        for (int i = 0; i < NH; ++i)
#pragma unroll
            for (int p = 0; p < VP; ++p)
                u[i][p] = rstd[p] * (u[i][p] - sum[0][p] * inv_c - v[i][p] * (sum[1][p] * inv_c));
        store_positions<TX, VP, NH>(static_cast<TX*>(a.dx) + at, step, off, u, count, channels);
    }
#pragma unroll
    for (int i = 0; i < NH; ++i) {
#pragma unroll
        for (int m = 1; m < LP; m *= 2) {
            dw[i] += __shfl_xor(dw[i], m, 64);
            db[i] += __shfl_xor(db[i], m, 64);
        }
        const int c = cr + i * Shape::kRows;
        if (lp == 0 && c < a.c) {
            a.part[(size_t)blockIdx.x * 2 * a.c + c] = dw[i];
            a.part[(size_t)blockIdx.x * 2 * a.c + a.c + c] = db[i];
        }
    }
}

// dweight and dbias from the workgroups' parts: 64 sums a workgroup, 16
// threads each, in a fixed order.  Bound by its latency: 4 us at 512 parts of
// 2 x 1024 sums.
__global__ __launch_bounds__(1024) void norm_gradient_sum_kernel(NormArgs a) {
    __shared__ float lds[16][64];
    const int i = blockIdx.x * 64 + threadIdx.x % 64, part = threadIdx.x / 64;
    float t = 0.f;
    if (i < 2 * a.c) {
#pragma unroll 8
        for (int b = part; b < a.blocks; b += 16) t += a.part[(size_t)b * 2 * a.c + i];
    }
    lds[part][threadIdx.x % 64] = t;
    __syncthreads();
    if (part == 0 && i < 2 * a.c) {
        for (int r = 1; r < 16; ++r) t += lds[r][threadIdx.x];
        float* out = i < a.c ? a.dweight : a.dbias;
        if (out) out[i < a.c ? i : i - a.c] = t;
    }
}

namespace {

template <typename TX, typename TY, int G, int NV, int N>
hipError_t last(bool backward, const NormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    if (!backward) {
        // a grid holds below 2^32 threads: more rows than that go in several launches
        constexpr int kRows = 256 / G;
        const long long rows = (long long)a.n * a.s, most = 0xffffffLL * kRows;
        for (long long row = 0; row < rows; row += most) {
            NormArgs part = a;
            part.n = 1;
            part.s = int(rows - row < most ? rows - row : most);
            part.x = static_cast<const TX*>(a.x) + row * a.c;
            part.y = static_cast<TY*>(a.y) + row * a.c;
            if (a.mean) {
                part.mean = a.mean + row;
                part.rstd = a.rstd + row;
            }
            if (hipError_t e = launch_kernel(norm_last_forward_kernel<TX, TY, G, NV, N>, dim3(unsigned((part.s + kRows - 1) / kRows)),
                                             dim3(256), 0, s, row == 0 ? ev.start : nullptr,
                                             row + most >= rows ? ev.stop : nullptr, part))
                return e;
        }
        return hipSuccess;
    }
    const int lds = 256 / G * 2 * a.c * 4 > 16 ? 256 / G * 2 * a.c * 4 : 16;
    auto kernel = norm_last_backward_kernel<TX, TY, G, NV, N>;
    if (hipError_t e = allow_dynamic_lds(kernel, lds)) return e;
    return launch_kernel(kernel, dim3(a.blocks), dim3(256), lds, s, ev.start, nullptr, a);
}

template <typename TX, typename TY>
hipError_t last_sized(bool backward, const NormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    if (a.wide) {
        const int pieces = a.c / 8;
        if (pieces <= 16) return last<TX, TY, 16, 1, 8>(backward, a, s, ev);
        if (pieces <= 64) return last<TX, TY, 64, 1, 8>(backward, a, s, ev);
        if (pieces <= 128) return last<TX, TY, 64, 2, 8>(backward, a, s, ev);
        if (pieces <= 512) return last<TX, TY, 256, 2, 8>(backward, a, s, ev);
        return last<TX, TY, 256, 4, 8>(backward, a, s, ev);
    }
    if (a.c <= 256) return last<TX, TY, 64, 4, 1>(backward, a, s, ev);
    if (a.c <= 1024) return last<TX, TY, 256, 4, 1>(backward, a, s, ev);
    return last<TX, TY, 256, 32, 1>(backward, a, s, ev);
}

template <typename TX, typename TY, int NT, int LP, int VP, int NH, bool SWAP>
hipError_t first_forward(const NormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    using Shape = FirstShape<NT, LP, VP>;
    const long long blocks = (long long)a.n * ((a.s + Shape::kPos - 1) / Shape::kPos);
    auto kernel = norm_first_forward_kernel<TX, TY, NT, LP, VP, NH, SWAP>;
    if (hipError_t e = allow_dynamic_lds(kernel, Shape::lds(SWAP))) return e;
    return launch_kernel(kernel, dim3(unsigned(blocks)), dim3(NT), Shape::lds(SWAP), s, ev.start, ev.stop, a);
}
template <typename TX, typename TY, int NT, int LP, int VP, int NH, bool SWAP>
hipError_t first_backward(const NormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    using Shape = FirstShape<NT, LP, VP>;
    auto kernel = norm_first_backward_kernel<TX, TY, NT, LP, VP, NH, SWAP>;
    if (hipError_t e = allow_dynamic_lds(kernel, Shape::lds(SWAP))) return e;
    return launch_kernel(kernel, dim3(a.blocks), dim3(NT), Shape::lds(SWAP), s, ev.start, nullptr, a);
}

// Positions side by side are what memory sees as one piece: 64 (256 bytes of
// fp32) where there are enough of them for every compute unit, else 16 (512 x 14 x
// 14: 7.7 us with 16, 13.6 with 64; 32 x 256 x 56 x 56: 48 us with 16, 34 with 64,
// both repeated on data that the caches hold).  A thread holds up to 64 elements
// forward; 2 x 64 and 2 x 16 sums backward.
template <typename TX, typename TY, bool SWAP>
hipError_t first_sized(bool backward, const NormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    const bool small = (long long)a.n * ((a.s + 63) / 64) < 256;
    if (!backward) {
        if (a.wide && small) {
            if (a.c <= 256) return first_forward<TX, TY, 256, 4, 4, 4, SWAP>(a, s, ev);
            if (a.c <= 512) return first_forward<TX, TY, 512, 4, 4, 4, SWAP>(a, s, ev);
            if (a.c <= 1024) return first_forward<TX, TY, 1024, 4, 4, 4, SWAP>(a, s, ev);
            return first_forward<TX, TY, 1024, 4, 4, 8, SWAP>(a, s, ev);
        }
        if (a.wide) {
            if (a.c <= 64) return first_forward<TX, TY, 256, 16, 4, 4, SWAP>(a, s, ev);
            if (a.c <= 128) return first_forward<TX, TY, 256, 16, 4, 8, SWAP>(a, s, ev);
            if (a.c <= 256) return first_forward<TX, TY, 256, 16, 4, 16, SWAP>(a, s, ev);
            if (a.c <= 512) return first_forward<TX, TY, 512, 16, 4, 16, SWAP>(a, s, ev);
            if (a.c <= 1024) return first_forward<TX, TY, 1024, 8, 4, 8, SWAP>(a, s, ev);
            return first_forward<TX, TY, 1024, 4, 4, 8, SWAP>(a, s, ev);
        }
    } else if (a.wide) {
        if (a.c <= 64) return first_backward<TX, TY, 256, 16, 4, 4, SWAP>(a, s, ev);
        if (a.c <= 128) return first_backward<TX, TY, 256, 16, 4, 8, SWAP>(a, s, ev);
        if (a.c <= 256) return first_backward<TX, TY, 256, 16, 4, 16, SWAP>(a, s, ev);
        if (a.c <= 512) return first_backward<TX, TY, 512, 8, 4, 8, SWAP>(a, s, ev);
        if (a.c <= 1024) return first_backward<TX, TY, 512, 4, 4, 8, SWAP>(a, s, ev);
        return first_backward<TX, TY, 512, 4, 4, 16, SWAP>(a, s, ev);
    }
    // rows with bf16 elements and a length that 4 does not divide
    if constexpr (sizeof(TX) == 2 || (sizeof(TY) == 2 && !SWAP)) {
        if (!backward) {
            if (a.c <= 128) return first_forward<TX, TY, 512, 64, 1, 16, SWAP>(a, s, ev);
            if (a.c <= 512) return first_forward<TX, TY, 1024, 32, 1, 16, SWAP>(a, s, ev);
            return first_forward<TX, TY, 1024, 8, 1, 16, SWAP>(a, s, ev);
        }
        if (a.c <= 128) return first_backward<TX, TY, 512, 64, 1, 16, SWAP>(a, s, ev);
        if (a.c <= 512) return first_backward<TX, TY, 512, 16, 1, 16, SWAP>(a, s, ev);
        return first_backward<TX, TY, 512, 8, 1, 32, SWAP>(a, s, ev);
    }
    return hipErrorInvalidValue;      // (not reached: rows of fp32 alone are always wide)
}

template <typename TX, typename TY>
hipError_t laid_out(bool backward, const NormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    if (!a.x_first) return last_sized<TX, TY>(backward, a, s, ev);
    return a.y_first ? first_sized<TX, TY, false>(backward, a, s, ev) : first_sized<TX, TY, true>(backward, a, s, ev);
}

hipError_t typed(bool backward, const NormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    if (a.x_type == FFTSPLIT_BF16) return laid_out<__bf16, __bf16>(backward, a, s, ev);
    return a.y_type == FFTSPLIT_BF16 ? laid_out<float, __bf16>(backward, a, s, ev)
                                     : laid_out<float, float>(backward, a, s, ev);
}

}  // namespace

// Two workgroups a compute unit keep the memory busy; more only add parts to be
// summed.  The two kernels at 32 x 784 tokens of 1024 channels with 256, 512 and
// 1024 workgroups: 47.4, 33.9, 34.5 us; at 5 x 77 x 57 x 75: 15.1, 13.4, 16.8 us.
int norm_backward_blocks(int n, int s, bool first) {
    const long long work = first ? (long long)n * ((s + 15) / 16) : ((long long)n * s + 3) / 4;
    return work < 512 ? int(work) : 512;
}

hipError_t launch_norm_forward(const NormArgs& a, hipStream_t s, const LaunchEvents& ev) { return typed(false, a, s, ev); }

hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s, const LaunchEvents& ev) {
    if (hipError_t e = typed(true, a, s, ev)) return e;
    return launch_kernel(norm_gradient_sum_kernel, dim3((2 * a.c + 63) / 64), dim3(1024), 0, s, nullptr, ev.stop, a);
}

}  // namespace fftsplit
