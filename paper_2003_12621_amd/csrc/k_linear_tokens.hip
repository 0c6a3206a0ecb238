// Linear attention of a few tokens: the recurrence itself,
//     S = decay S + k_t v_t^T,   o_t = scale q_t^T S,
// in fp32, with the state read once and written once.
//
// Bound by the state's bytes.  A workgroup takes 64 columns of one key head's
// state: 16 lanes a row, 4 columns a lane, rows dealt out to 16 groups, so that
// every row is one run of 256 bytes and the state stays in registers over the
// tokens.  The sums over the rows are joined through LDS.  The tokens' rows are
// read into LDS side by side with the state, as many as fit: one after the other
// they cost a wait for memory each (5 tokens of 16 sequences of 16 heads (4) of 64 /
// 128 18 us, so 11; single tokens of 64 sequences of 16 heads 15 us either way, 67 MB
// of states at a copy's rate).
#include "linear_common.hpp"

namespace fftsplit {

namespace {
constexpr int kTokenColumns = 64, kTokenGroups = 16;
// Query heads whose outputs are joined at once.
constexpr int kTokenHeads = 4;
// Bytes of LDS for the tokens' rows.
constexpr int kTokenBytes = 49152;

// Rows in LDS, at a time: of k, v and `heads` query heads of `tokens` tokens.
struct TokenStage {
    int tokens, heads;
};
}  // namespace

// ROWS: of the state in a thread.
template <typename T, int ROWS, bool WIDE>
__global__ __launch_bounds__(256) void linear_tokens_kernel(LinearTokens a, TokenStage stage) {
    // [token][k, query heads][d], then [token][column] of v
    constexpr int kWidth = kTokenGroups * ROWS;
    extern __shared__ __align__(16) char lds[];
    __shared__ float4 join[2][kTokenHeads][4][16];
    T* rows = reinterpret_cast<T*>(lds);
    const int per = stage.heads + 1;
    T* values = rows + stage.tokens * per * kWidth;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, group = tid >> 4;
    const int slices = (a.dv + kTokenColumns - 1) / kTokenColumns;
    const int slice = blockIdx.x % slices, head = blockIdx.x / slices, h = head % a.hk, b = head / a.hk;
    const int column = slice * kTokenColumns + 4 * (tid & 15), heads = a.hq / a.hk;
    const int length = linear_length(a.lengths, a.s, b);
    const float less_one = decay_less_one(decay_log2(a.log_decay[h]), 1);
    const size_t at = size_t(head) * a.d * a.dv + column;

    float4 state[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int row = group + kTokenGroups * i;
        float e[4] = {0.f, 0.f, 0.f, 0.f};
        if (a.state && row < a.d) {
            const float* p = a.state + at + size_t(row) * a.dv;
            if constexpr (WIDE) {
                if (column < a.dv) *reinterpret_cast<float4*>(e) = *reinterpret_cast<const float4*>(p);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (column + j < a.dv) e[j] = p[j];
            }
        }
        state[i] = make_float4(e[0], e[1], e[2], e[3]);
    }
    T* o = static_cast<T*>(a.o) + (size_t(b) * a.s * a.hq + size_t(h) * heads) * a.dv + column;
    const int there = min(length, a.s);
    for (int t = there; t < a.s; ++t)
        for (int g = group; g < heads; g += kTokenGroups)
            store4(o + (size_t(t) * a.hq + g) * a.dv, 0, a.dv - column, WIDE, 0.f, 0.f, 0.f, 0.f);
    int buffer = 0;
    for (int t0 = 0; t0 < there; t0 += stage.tokens) {
        const int tokens = min(stage.tokens, there - t0);
        // (several turns over the heads only where one token at a time does not fit)
        for (int first = 0; first < heads; first += stage.heads) {
            const int members = min(stage.heads, heads - first), total = tokens * per * kWidth;
            if (t0 || first) __syncthreads();
            for (int i0 = tid; i0 < total; i0 += 8 * 256) {
                T e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int i = min(i0 + j * 256, total - 1), which = i / kWidth % per, t = t0 + i / kWidth / per;
                    const int col = min(i % kWidth, a.d - 1), g = min(which - 1, members - 1);
                    const T* p = which ? static_cast<const T*>(a.q.p) + b * a.q.b + t * a.q.t +
                                             (long long)(h * heads + first + g) * a.q.h
                                       : static_cast<const T*>(a.k.p) + b * a.k.b + t * a.k.t + h * a.k.h;
                    e[j] = p[col];
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int i = i0 + j * 256;
                    if (i < total) rows[i] = i % kWidth < a.d ? e[j] : T(0.f);
                }
            }
            if (!first)
                for (int i = tid; i < tokens * kTokenColumns; i += 256) {
                    const int col = slice * kTokenColumns + i % kTokenColumns;
                    values[i] = col < a.dv ? (static_cast<const T*>(a.v.p) + b * a.v.b + (t0 + i / kTokenColumns) * a.v.t +
                                              h * a.v.h)[col] : T(0.f);
                }
            __syncthreads();
            for (int t = 0; t < tokens; ++t) {
                const T* k = rows + t * per * kWidth + group;
                if (!first) {
                    float x[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = float(values[t * kTokenColumns + 4 * (tid & 15) + j]);
#pragma unroll
                    for (int i = 0; i < ROWS; ++i) {
                        const float y = float(k[kTokenGroups * i]);
                        float4& s = state[i];
                        s.x = fmaf(y, x[0], fmaf(s.x, less_one, s.x));
                        s.y = fmaf(y, x[1], fmaf(s.y, less_one, s.y));
                        s.z = fmaf(y, x[2], fmaf(s.z, less_one, s.z));
                        s.w = fmaf(y, x[3], fmaf(s.w, less_one, s.w));
                    }
                }
                for (int g0 = 0; g0 < members; g0 += kTokenHeads, buffer ^= 1) {
                    const int n = min(members - g0, kTokenHeads);
#pragma unroll
                    for (int g = 0; g < kTokenHeads; ++g) {
                        if (g >= n) break;
                        const T* q = k + (1 + g0 + g) * kWidth;
                        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (int i = 0; i < ROWS; ++i) {
                            const float y = float(q[kTokenGroups * i]);
                            sum.x = fmaf(y, state[i].x, sum.x);
                            sum.y = fmaf(y, state[i].y, sum.y);
                            sum.z = fmaf(y, state[i].z, sum.z);
                            sum.w = fmaf(y, state[i].w, sum.w);
                        }
#pragma unroll
                        for (int m = 16; m < 64; m *= 2) {
                            sum.x += __shfl_xor(sum.x, m);
                            sum.y += __shfl_xor(sum.y, m);
                            sum.z += __shfl_xor(sum.z, m);
                            sum.w += __shfl_xor(sum.w, m);
                        }
                        if (lane < 16) join[buffer][g][wave][lane] = sum;
                    }
                    // (the other buffer's readers are past the barrier after it)
                    __syncthreads();
                    if (group < n) {
                        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const float4 z = join[buffer][group][w][tid & 15];
                            y = make_float4(y.x + z.x, y.y + z.y, y.z + z.z, y.w + z.w);
                        }
                        store4(o + (size_t(t0 + t) * a.hq + first + g0 + group) * a.dv, 0, a.dv - column, WIDE, y.x * a.scale,
                               y.y * a.scale, y.z * a.scale, y.w * a.scale);
                    }
                }
            }
        }
    }
    if (!a.state_out) return;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int row = group + kTokenGroups * i;
        if (row >= a.d) continue;
        store4(a.state_out + at + size_t(row) * a.dv, 0, a.dv - column, WIDE, state[i].x, state[i].y, state[i].z,
               state[i].w);
    }
}

namespace {
template <typename T, int ROWS>
hipError_t launch_rows(const LinearTokens& a, hipStream_t s, const LaunchEvents& ev) {
    const long long blocks = (long long)a.n * a.hk * ((a.dv + kTokenColumns - 1) / kTokenColumns);
    auto kernel = a.state_wide ? linear_tokens_kernel<T, ROWS, true> : linear_tokens_kernel<T, ROWS, false>;
    constexpr int kRow = kTokenGroups * ROWS * int(sizeof(T)), kValues = kTokenColumns * int(sizeof(T));
    const int heads = a.hq / a.hk, most = (kTokenBytes - kValues) / kRow - 1;
    TokenStage stage{1, heads < most ? heads : most};
    const int token = (stage.heads + 1) * kRow + kValues;
    if (stage.heads == heads) stage.tokens = kTokenBytes / token < a.s ? kTokenBytes / token : a.s;
    const int lds = stage.tokens * token;
    if (hipError_t e = allow_dynamic_lds(kernel, lds)) return e;
    return launch_kernel(kernel, dim3(unsigned(blocks)), dim3(256), unsigned(lds), s, ev.start, ev.stop, a, stage);
}

template <typename T>
hipError_t launch_typed(const LinearTokens& a, hipStream_t s, const LaunchEvents& ev) {
    if (a.d <= 32) return launch_rows<T, 2>(a, s, ev);
    if (a.d <= 64) return launch_rows<T, 4>(a, s, ev);
    if (a.d <= 128) return launch_rows<T, 8>(a, s, ev);
    return launch_rows<T, 16>(a, s, ev);
}
}  // namespace

hipError_t launch_linear_tokens(const LinearTokens& a, int dtype, hipStream_t s, const LaunchEvents& ev) {
    return dtype == FFTSPLIT_BF16 ? launch_typed<__bf16>(a, s, ev) : launch_typed<float>(a, s, ev);
}

}  // namespace fftsplit
