// Linear attention with a decay for each head.
//
// A sequence is cut into segments.  Within one, the terms of all pairs of tokens
// are taken one by one, as in attention without a softmax: a wave owns 32 query
// rows, goes over the keys of its segment in tiles of 32 and adds
//     decay^(i - j) (q_i . k_j) v_j
// to its outputs.  What lies before the segment comes from the state S (d x dv)
// before it, as decay^i q_i^T S.  So no wave waits for another one's state:
//   parts  adds up what each segment adds to the state,
//   join   makes of these the state before each segment,
//   pass   computes the outputs of all rows at once.
//
// The gradients are the same sums with other roles: dq that of (dO, v, k), and
// dk and dv those of (v, dO, q) and (k, q, dO) from the last token to the first.
#include "linear_pass.hpp"

namespace fftsplit {

namespace {

// What a wave's accumulators of the state hold in register r: rows in the order
// in which a product over them takes an operand read along a tile's row.
__device__ __forceinline__ int state_row(int r, int hi) { return 16 * (r >> 3) + 8 * hi + (r & 7); }

// A lane's part of the address of read_column where its rows are to be in that
// order: bits 2 and 3 of the column change places.
template <typename T, int W>
__device__ __forceinline__ unsigned state_column_lane(int lane) {
    using Shape = TileShape<T, W>;
    if constexpr (sizeof(T) == 4) {
        const int c = (lane & 31) / 4;
        return Shape::at(4 * (lane >> 5), (c & 4) | (c & 1) << 1 | (c >> 1 & 1)) + (lane & 3) * 4;
    }
    return Shape::at(4 * (lane >> 5) + ((lane >> 2) & 3), 2 * ((lane >> 4) & 1) + (lane & 1)) + ((lane >> 1) & 1) * 8;
}

// An operand's elements times factors, as the sum of PARTS operands.  bf16 elements
// times fp32 factors have 24 significant bits, three bf16 numbers of 8, cut off one
// after the other: that is what a state that the caller gets is summed from.  Where
// it only serves as an operand of two parts, good to 2^-15, two of them do (off by
// 2^-14 at most, by 2^-16 in the mean).  fp32 elements are one.
template <typename T, int PARTS>
struct Weighted {
    Operand<T> part[PARTS];
    __device__ __forceinline__ Weighted(const Operand<T>& x, const float* w) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 8; ++e) part[0].v[e] = x.v[e] * w[e];
        } else {
            u32x4 p[PARTS];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float a = float(x.v[2 * e]) * w[2 * e], b = float(x.v[2 * e + 1]) * w[2 * e + 1];
#pragma unroll
                for (int i = 0; i < PARTS; ++i) {
                    // (the upper halves)
                    p[i][e] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
                    a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
                    b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
                }
            }
#pragma unroll
            for (int i = 0; i < PARTS; ++i) part[i].v = __builtin_bit_cast(bf16x8, p[i]);
        }
    }
};

struct PassPair {
    LinearPass pass[2];
    int first_blocks;                // of pass[0]; the rest belong to pass[1]
};

}  // namespace

template <typename T, int D, int COLUMNS, bool WIDE>
__global__ __launch_bounds__(64 * kPassWaves, (PassShape<T, D, COLUMNS>::kPassOccupancy))
void linear_pass_kernel(PassPair pair) {
    const bool second = int(blockIdx.x) >= pair.first_blocks;
    linear_pass<T, D, COLUMNS, WIDE>(pair.pass[second], int(blockIdx.x) - (second ? pair.first_blocks : 0),
                                     second ? int(gridDim.x) - pair.first_blocks : pair.first_blocks);
}

// What one segment of one head adds to the state, from zero: 32 WAVES columns, 32 a
// wave, whose accumulators keep the state while the keys pass.  PARTS: of the
// weighted values (Weighted).  4 x 16384 tokens of 16 heads of 64 / 128 in bf16: 537 MB in
// 110 us, a copy's rate, with vector instructions (the weights and their parts) issued 73
// % of the time.
template <typename T, int D, int WAVES, bool WIDE, int PARTS>
__global__ __launch_bounds__(64 * WAVES, (D <= 128 ? 2 : 1)) void linear_parts_kernel(PassPair pair) {
    constexpr int kTile = kLinearTile, DT = D / 32, kColumns = 32 * WAVES;
    using Shape = StageShape<T, D, kColumns, WAVES, 0>;
    extern __shared__ __align__(16) char lds[];
    const bool second = int(blockIdx.x) >= pair.first_blocks;
    const LinearPass& a = pair.pass[second];
    const int lane = threadIdx.x & 63, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int slices = (a.dv + kColumns - 1) / kColumns;
    const int blocks = second ? int(gridDim.x) - pair.first_blocks : pair.first_blocks;
    int id = xcd_logical_block(int(blockIdx.x) - (second ? pair.first_blocks : 0), blocks);
    const int column0 = linear_scalar(id % slices * kColumns);
    id /= slices;
    const int segment = linear_scalar(id % a.part_count) + a.first_part, head = linear_scalar(id / a.part_count);
    const int h = linear_scalar(head % a.hk), b = linear_scalar(head / a.hk);
    const int begin = segment * a.segment_tokens;
    const float log2_decay = decay_log2(linear_uniform(a.log_decay + h));
    const int end = int(min((long long)begin + a.segment_tokens, (long long)linear_length(a.lengths, a.s, b)));

    KeyStream<T, D, kColumns, WAVES, 0, WIDE> stream(a, unsigned(reinterpret_cast<uintptr_t>(lds)), b, h, column0, begin, end,
                                                     0, 0, wave, lane);
    for (int i = 0; i + 1 < Shape::kStages; ++i) stream.fetch(wave, lane);
    // a token's weight is decay to its distance from the segment's end (backwards,
    // from one before its beginning): of its place in the tile, times the tile's
    const int reverse = linear_scalar(a.reverse), k_heads = linear_scalar(a.k_heads);
    const float update_scale = linear_scalar(a.update_scale);
    float weight[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int key = acc_row(r, hi);
        weight[r] = update_scale * decay_power(log2_decay, reverse ? key + 1 : kTile - 1 - key);
    }
    floatx16 state[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) state[d] = zero16();
    const unsigned k_column = stream.base + state_column_lane<T, D>(lane);
    const unsigned v_column = stream.base + column_lane<T, kColumns>(lane) + Shape::kRowBytes;
    int stage = 0;
    for (int n = 0; n < stream.stages; ++n) {
        for (int g = 0; g < k_heads; ++g) {
            stream.advance(wave, lane);
#pragma unroll
            for (int j = 0; j < Shape::kRows / kTile; ++j) {
                const int first = n * Shape::kRows + j * kTile, keys = end - begin - first;
                float w[16];
                const float far = decay_power(log2_decay, reverse ? first : max(keys - kTile, 0));
#pragma unroll
                for (int r = 0; r < 16; ++r) w[r] = weight[r] * far;
                if (keys < kTile && !reverse) {
                    // (behind the last, values are zero)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        w[r] = update_scale * decay_power(log2_decay, max(keys - 1 - acc_row(r, hi), 0));
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const Weighted<T, PARTS> x(read_column<T, kColumns>(v_column + stage, kTile * j, 32 * wave, i), w + 8 * i);
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const Operand<T> y = read_column<T, D>(k_column + stage, kTile * j, 32 * d, i);
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) mma(state[d], y, x.part[p]);
                    }
                }
            }
            stage = stage + Shape::kStageBytes == Shape::kLds ? 0 : stage + Shape::kStageBytes;
        }
    }
    own_copies_done<0>();
    const int column = column0 + 32 * wave + (lane & 31);
    float* to = a.parts + (size_t(head) * a.segments + segment) * a.d * a.dv + column;
    if (column < a.dv)
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = 32 * d + state_row(r, hi);
                if (row < a.d) to[unsigned(row * a.dv)] = state[d][r];
            }
}

struct JoinJobs {
    LinearJoin job[3];
    int end[3];                      // workgroups up to and including each
};

// A lane: 8 rows of one column of the operands.  The segments are taken WAVES * RUN at a
// time, a run of RUN of them to a wave, whose loads are in flight together; each wave
// adds up its own run, reads the other waves' sums for the state before it, and goes
// through its run once more.  The order is that of the segments, whatever the timing.
// VEC: the 8 rows lie side by side in a state.  64 segments of 64 heads of 64 / 128 in
// bf16: 268 MB in 52 us, a copy's rate; of 4 heads 12 us, of waits.
template <typename T, int WAVES, int RUN, bool VEC>
__device__ __forceinline__ void linear_join(const LinearJoin& a, int block, float (&sums)[WAVES][8][64]) {
    const int items = a.rows / 8 * a.columns, per = items / 64;
    const int head = block / per, lane = threadIdx.x & 63, item = block % per * 64 + lane;
    const int wave = linear_scalar(int(threadIdx.x >> 6));
    const int step = item / 64 % (a.rows / 16), strip = item / 64 / (a.rows / 16);
    const int row0 = 16 * step + 8 * (lane >> 5), column = 32 * strip + (lane & 31);
    const int length = linear_scalar(linear_length(a.lengths, a.s, head / a.hk));
    const float log2_decay = decay_log2(linear_uniform(a.log_decay + head % a.hk));
    const int elements = a.d * a.dv, row_step = a.turned ? 1 : a.dv, column_step = a.turned ? a.dv : 1;
    const int rows = min((a.turned ? a.dv : a.d) - row0, 8);
    const bool there = column < (a.turned ? a.d : a.dv);
    const int at = row0 * row_step + column * column_step;
    // (loads that do not branch, for many at a time: what is not there reads element 0)
    auto load = [&](float (&e)[8], const float* p) {
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
                const float4 v = *reinterpret_cast<const float4*>(p + (there && j < rows ? at + j : 0));
                e[j] = v.x;
                e[j + 1] = v.y;
                e[j + 2] = v.z;
                e[j + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = p[there && j < rows ? at + j * row_step : 0];
        }
    };
    auto keep = [&](float (&e)[8], bool given) {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = given && there && j < rows ? e[j] : 0.f;
    };
    const float whole = decay_less_one(log2_decay, a.segment_tokens);
    const float whole_run = decay_less_one(log2_decay, RUN * a.segment_tokens);
    // decay over the segments from `first` on, in the order of the join, less one
    auto carry_over = [&](int first, int count) {
        const int low = a.reverse ? a.segments - first - count : first;
        const int tokens = max(0, min(length - low * a.segment_tokens, count * a.segment_tokens));
        if (tokens == a.segment_tokens) return whole;
        if (tokens == RUN * a.segment_tokens) return whole_run;
        return tokens ? decay_less_one(log2_decay, tokens) : 0.f;
    };
    auto advance = [&](float (&state)[8], float carry, const float (&added)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) state[j] = fmaf(state[j], carry, state[j]) + added[j];
    };
    float state[8];
    load(state, a.init ? a.init + size_t(head) * elements : a.parts);
    keep(state, a.init != nullptr);
    const float* parts = a.parts + size_t(head) * a.segments * elements;
    constexpr int kParts = Precise<T>::kParts;
    Operand<T>* starts =
        static_cast<Operand<T>*>(a.starts) + (size_t(head) * a.segments * items + item / 64 * 64) * kParts + lane;
    for (int m0 = 0; m0 < a.segments; m0 += RUN * WAVES) {
        // the run of any wave in this turn
        auto first_of = [&](int w) { return min(m0 + w * RUN, a.segments); };
        const int first = first_of(wave), count = first_of(wave + 1) - first;
        auto segment = [&](int i) {
            const int m = min(first + i, a.segments - 1);
            return a.reverse ? a.segments - 1 - m : m;
        };
        float added[RUN][8], sum[8] = {};
#pragma unroll
        for (int i = 0; i < RUN; ++i) load(added[i], parts + (long long)segment(i) * elements);
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            const int m = segment(i);
            keep(added[i], i < count && m >= a.first_part && m < a.first_part + a.part_count);
            if (i < count) advance(sum, carry_over(first + i, 1), added[i]);
        }
        if (m0) __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[wave][j][lane] = sum[j];
        __syncthreads();
        // the state before this wave's run, and before the next turn
        float next[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) next[j] = state[j];
        for (int w = 0; w < WAVES; ++w) {
            const int f = first_of(w), c = first_of(w + 1) - f;
            if (!c) break;
            float other[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) other[j] = sums[w][j][lane];
            advance(next, carry_over(f, c), other);
            if (w < wave)
#pragma unroll
                for (int j = 0; j < 8; ++j) state[j] = next[j];
        }
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            if (i >= count) break;
            if (a.starts) {
                floatx16 c;
#pragma unroll
                for (int j = 0; j < 8; ++j) c[j] = state[j];
                Precise<T> x;
                x.set(c, 0);
#pragma unroll
                for (int p = 0; p < kParts; ++p) starts[size_t(segment(i)) * items * kParts + 64 * p] = x.part[p];
            }
            advance(state, carry_over(first + i, 1), added[i]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) state[j] = next[j];
    }
    if (a.last && there && !wave)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < rows) a.last[size_t(head) * elements + at + j * row_step] = state[j];
}

template <typename T, int WAVES, int RUN>
__global__ __launch_bounds__(64 * WAVES, 4) void linear_join_kernel(JoinJobs jobs) {
    __shared__ float sums[WAVES][8][64];
    const int which = int(blockIdx.x) < jobs.end[0] ? 0 : int(blockIdx.x) < jobs.end[1] ? 1 : 2;
    const LinearJoin& a = jobs.job[which];
    const int block = blockIdx.x - (which ? jobs.end[which - 1] : 0);
    if (a.turned && a.dv % 4 == 0)
        linear_join<T, WAVES, RUN, true>(a, block, sums);
    else
        linear_join<T, WAVES, RUN, false>(a, block, sums);
}

namespace {

long long part_blocks(const LinearPass& a, int columns) {
    return (long long)a.n * a.hk * a.part_count * ((a.dv + columns - 1) / columns);
}

// MAIN: the pass; else the parts.
template <typename T, int D, int COLUMNS, bool MAIN>
hipError_t launch_shaped(const LinearPass& a, const LinearPass* b, hipStream_t s, const LaunchEvents& ev) {
    constexpr int kWaves = MAIN ? kPassWaves : COLUMNS / 32, kBehind = MAIN ? kDiagonalBytes : 0;
    using Shape = StageShape<T, D, COLUMNS, kWaves, kBehind>;
    auto blocks = [](const LinearPass& p) { return MAIN ? pass_blocks(p, COLUMNS) : part_blocks(p, COLUMNS); };
    const PassPair pair{{a, b ? *b : a}, int(blocks(a))};
    void (*kernel)(PassPair);
    if constexpr (MAIN) {
        kernel = a.wide ? linear_pass_kernel<T, D, COLUMNS, true> : linear_pass_kernel<T, D, COLUMNS, false>;
    } else {
        constexpr int kAll = sizeof(T) == 2 ? 3 : 1, kSome = sizeof(T) == 2 ? 2 : 1;
        if (a.exact || (b && b->exact))
            kernel = a.wide ? linear_parts_kernel<T, D, kWaves, true, kAll> : linear_parts_kernel<T, D, kWaves, false, kAll>;
        else
            kernel = a.wide ? linear_parts_kernel<T, D, kWaves, true, kSome> : linear_parts_kernel<T, D, kWaves, false, kSome>;
    }
    constexpr int kLds = Shape::kLds + kBehind;
    if (hipError_t e = allow_dynamic_lds(kernel, kLds)) return e;
    return launch_kernel(kernel, dim3(unsigned(blocks(a) + (b ? blocks(*b) : 0))), dim3(64 * kWaves), kLds, s, ev.start, ev.stop,
                         pair);
}

template <typename T, bool MAIN>
hipError_t launch_typed(const LinearPass& a, const LinearPass* b, hipStream_t s, const LaunchEvents& ev) {
    const bool few = linear_columns(a.dv) == 64;
    switch (linear_padded(a.d)) {
        case 32: return few ? launch_shaped<T, 32, 64, MAIN>(a, b, s, ev) : launch_shaped<T, 32, 128, MAIN>(a, b, s, ev);
        case 64: return few ? launch_shaped<T, 64, 64, MAIN>(a, b, s, ev) : launch_shaped<T, 64, 128, MAIN>(a, b, s, ev);
        case 128: return few ? launch_shaped<T, 128, 64, MAIN>(a, b, s, ev) : launch_shaped<T, 128, 128, MAIN>(a, b, s, ev);
        default: return few ? launch_shaped<T, 256, 64, MAIN>(a, b, s, ev) : launch_shaped<T, 256, 128, MAIN>(a, b, s, ev);
    }
}

// Few waves, each with a longer run, cost less where one turn goes over all segments; for
// more, more waves save turns.  Measured, 4 / 8 waves (us): 13 and 16 segments of the
// three joins of a training step of 4 x 3136 tokens of 8 heads of 64 / 128 19 / 26, of 2 x
// 1999 tokens of 8 heads (4) of 128 / 256 24 / 31; 64 segments of 4 heads 17 / 12 (of 64
// heads 55 / 52, which is their bytes).
template <typename T>
hipError_t launch_join(const JoinJobs& j, int blocks, hipStream_t s, const LaunchEvents& ev) {
    const int segments = j.job[0].segments;
    auto launch = [&](auto kernel, int waves) {
        return launch_kernel(kernel, dim3(unsigned(blocks)), dim3(64 * waves), 0, s, ev.start, ev.stop, j);
    };
    if (segments <= 4) return launch(linear_join_kernel<T, 4, 1>, 4);
    if (segments <= 8) return launch(linear_join_kernel<T, 4, 2>, 4);
    if (segments <= 16) return launch(linear_join_kernel<T, 4, 4>, 4);
    return launch(linear_join_kernel<T, 8, 4>, 8);
}

}  // namespace

hipError_t launch_linear_pass(const LinearPass& a, const LinearPass* b, int dtype, hipStream_t s, const LaunchEvents& ev) {
    return dtype == FFTSPLIT_BF16 ? launch_typed<__bf16, true>(a, b, s, ev) : launch_typed<float, true>(a, b, s, ev);
}

hipError_t launch_linear_parts(const LinearPass& a, const LinearPass* b, int dtype, hipStream_t s, const LaunchEvents& ev) {
    return dtype == FFTSPLIT_BF16 ? launch_typed<__bf16, false>(a, b, s, ev) : launch_typed<float, false>(a, b, s, ev);
}

hipError_t launch_linear_join(const LinearJoin* jobs, int count, int dtype, hipStream_t s, const LaunchEvents& ev) {
    JoinJobs j{};
    int blocks = 0;
    for (int i = 0; i < 3; ++i) {
        j.job[i] = jobs[i < count ? i : 0];
        if (i < count) blocks += j.job[i].heads * (j.job[i].rows / 8 * j.job[i].columns / 64);
        j.end[i] = blocks;
    }
    return dtype == FFTSPLIT_BF16 ? launch_join<__bf16>(j, blocks, s, ev) : launch_join<float>(j, blocks, s, ev);
}

}  // namespace fftsplit
