// The sum over the tokens of a segment that the forward pass and the gradients of
// linear attention share.
#pragma once

#include <type_traits>

#include "linear_common.hpp"

namespace fftsplit {

// LDS of a compute unit.
constexpr int kLinearLds = 163840;

// A stage: some rows of k and of v, of D and COLUMNS columns, on their way from
// memory straight into LDS, in pieces of 1024 bytes that are dealt out to the waves
// alike, so that every wave has the same number of copies in flight.  BEHIND: bytes
// of LDS that the kernel needs behind the ring of stages.
template <typename T, int D, int COLUMNS, int WAVES, int BEHIND>
struct StageShape {
    // Whether the pass's accumulators leave room for three waves a SIMD: then stages of
    // one tile and fewer operands read ahead, which take 6 % off all kernels of 4 x 16384
    // tokens of 16 heads of 64 / 128 and 11 % off those of training of 4 x 3136 tokens of 8
    // heads (466 -> 439 and 185 -> 165 us); of 128 / 256 nothing.
    static constexpr bool kLean = sizeof(T) == 2 && D * COLUMNS <= 8192;
    static constexpr int kPassOccupancy = kLean ? 3 : D <= 128 || sizeof(T) == 2 ? 2 : 1;
    // (as many as the registers hold)
    static constexpr int kPassAhead = kLean ? (COLUMNS > 64 ? 1 : 2) : sizeof(T) == 4 && D * COLUMNS >= 16384 ? 2 : 3;
    // Two tiles a stage, where two workgroups with rings of two stages fit a compute unit
    // (one alone took twice the time: gradients of 4 x 3136 tokens of 8 heads of 64 / 256 in
    // bf16 388 us, with one tile a stage 185; forward pass of 8 x 784 tokens of 256 / 64 187
    // and 36)
    static constexpr int kRows =
        !kLean && 2 * 64 * (D + COLUMNS) * int(sizeof(T)) + BEHIND <= kLinearLds / 2 ? 64 : 32;
    static constexpr int kRowBytes = TileShape<T, D>::bytes(kRows);
    static constexpr int kUsedBytes = kRowBytes + TileShape<T, COLUMNS>::bytes(kRows);
    static constexpr int kPer = (kUsedBytes / 1024 + WAVES - 1) / WAVES;             // copies of a wave
    static constexpr int kStageBytes = kPer * WAVES * 1024;
    // Stages in LDS: the one worked on, and those on their way.
    static constexpr int kStages = 3 * kStageBytes + BEHIND <= kLinearLds / 2 ? 3 : 2;
    static constexpr int kLds = kStages * kStageBytes;
};

template <typename T, int D, int COLUMNS, int WAVES, int BEHIND, bool WIDE>
struct StageCopy {
    using Shape = StageShape<T, D, COLUMNS, WAVES, BEHIND>;
    using Rows = TileShape<T, D>;
    using Values = TileShape<T, COLUMNS>;
    static constexpr int kRowPieces = Shape::kRowBytes / 1024, kPieces = Shape::kUsedBytes / 1024;
    unsigned off[Shape::kPer];
    int row[Shape::kPer];

    // Which tensor a wave's piece i belongs to: 0 k, 1 v, in this order in LDS (or
    // 2: none, filled up with zeros).
    static __device__ __forceinline__ int tensor(int wave, int i) {
        // (where all waves have the same, that is known here)
        const int piece = i * WAVES + (kRowPieces % WAVES || kPieces % WAVES ? wave : 0);
        return piece < kRowPieces ? 0 : piece < kPieces ? 1 : 2;
    }
    // Column of a lane's chunk of that piece, and its row.
    static __device__ __forceinline__ int place(int wave, int lane, int i, int& row) {
        const int which = tensor(wave, i), at = (wave + i * WAVES - (which ? kRowPieces : 0)) * 64 + lane;
        row = which ? at / Values::kRowChunks : at / Rows::kRowChunks;
        return which ? ((at % Values::kRowChunks) ^ Values::swizzle(row)) * Values::kChunk
                     : ((at % Rows::kRowChunks) ^ Rows::swizzle(row)) * Rows::kChunk;
    }
    __device__ __forceinline__ StageCopy(long long k_stride, int k_cols, long long v_stride, int v_cols, int wave,
                                         int lane) {
#pragma unroll
        for (int i = 0; i < Shape::kPer; ++i) {
            const int which = tensor(wave, i), col = place(wave, lane, i, row[i]);
            off[i] = which < 2 && col < (which ? v_cols : k_cols)
                         ? unsigned((row[i] * (which ? v_stride : k_stride) + col) * int(sizeof(T))) : kOutOfRange;
        }
    }
    // Starts the copies of the first `rows` rows of a stage (at most all, possibly none or
    // less) from k and v on, which reach `size` bytes.  The rest of the stage becomes zero,
    // whatever the strides: nothing else keeps what lies behind a sequence's end out of
    // the sums.
    __device__ __forceinline__ void start(unsigned stage, const char* k, const char* v, unsigned size_k, unsigned size_v,
                                          int rows, int k_cols, int v_cols, int wave, int lane) const {
#pragma unroll
        for (int i = 0; i < Shape::kPer; ++i) {
            const int which = tensor(wave, i);
            const unsigned to = stage + (wave + i * WAVES) * 1024, at = row[i] < rows ? off[i] : kOutOfRange;
            const char* from = which ? v : k;
            const unsigned size = which ? size_v : size_k;
            if constexpr (WIDE) {
                copy16(copy_source(from, size), at, __builtin_amdgcn_readfirstlane(to));
            } else {
                const BufRsrc rsrc = make_rsrc(from, size);
                int unused;
                const int col = place(wave, lane, i, unused);
                constexpr int kChunk = 16 / sizeof(T);
                T e[kChunk];
#pragma unroll
                for (int j = 0; j < kChunk; ++j) {
                    const unsigned o = col + j < (which ? v_cols : k_cols) ? at + j * unsigned(sizeof(T)) : kOutOfRange;
                    if constexpr (sizeof(T) == 4)
                        e[j] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rsrc, o, 0, 0));
                    else
                        e[j] = __builtin_bit_cast(__bf16, __builtin_amdgcn_raw_buffer_load_b16(rsrc, o, 0, 0));
                }
                u32x4 u;
                __builtin_memcpy(&u, e, 16);
                *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(
                    (__attribute__((address_space(3))) char*)(to + lane * 16)) = u;
            }
        }
    }
};

// The keys that a workgroup goes over in stages, of each the heads of k and v that
// share a state one after another: copies them into a ring.  First the tokens from
// `first` on to `end`, then those from `other` on to `other_end` (either possibly
// none); rows of the last stage that are not there become zero.
template <typename T, int D, int COLUMNS, int WAVES, int BEHIND, bool WIDE>
struct KeyStream {
    using Shape = StageShape<T, D, COLUMNS, WAVES, BEHIND>;
    static constexpr int kBytes = sizeof(T);
    const StageCopy<T, D, COLUMNS, WAVES, BEHIND, WIDE> copy;
    const char *k, *v;
    // to the next head; further from the last one to the next stage's first; and further
    // to the first of the other tokens
    long long to_head_k, to_head_v, to_next_k, to_next_v, to_other_k, to_other_v;
    unsigned size_k, size_v;
    int own, stages, heads, k_cols, v_cols, next_stage = 0, next_head = 0, rows, to_other_rows;
    unsigned base, next;             // LDS: of the ring, and of the stage to fill next

    __device__ __forceinline__ KeyStream(const LinearPass& a, unsigned ring, int b, int h, int column0, int first, int end,
                                         int other, int other_end, int wave, int lane)
        : copy(a.k.t, a.d, a.v.t, min(a.dv - column0, COLUMNS), wave, lane) {
        base = next = ring;
        heads = linear_scalar(a.k_heads);
        k_cols = a.d;
        v_cols = min(a.dv - column0, COLUMNS);
        rows = end - first;
        const int other_rows = other_end - other;
        own = rows > 0 ? (rows + Shape::kRows - 1) / Shape::kRows : 0;
        stages = own + (other_rows > 0 ? (other_rows + Shape::kRows - 1) / Shape::kRows : 0);
        to_other_rows = other_rows + own * Shape::kRows - rows;
        k = static_cast<const char*>(a.k.p) + (b * a.k.b + (long long)h * heads * a.k.h + first * a.k.t) * kBytes;
        v = static_cast<const char*>(a.v.p) + (b * a.v.b + (long long)h * heads * a.v.h + first * a.v.t + column0) * kBytes;
        to_head_k = a.k.h * kBytes;
        to_head_v = a.v.h * kBytes;
        to_next_k = Shape::kRows * kBytes * a.k.t - heads * to_head_k;
        to_next_v = Shape::kRows * kBytes * a.v.t - heads * to_head_v;
        const long long jump = (long long)(other - first) - own * Shape::kRows;
        to_other_k = jump * kBytes * a.k.t;
        to_other_v = jump * kBytes * a.v.t;
        size_k = unsigned(((Shape::kRows - 1) * a.k.t + k_cols) * kBytes);
        size_v = unsigned(((Shape::kRows - 1) * a.v.t + v_cols) * kBytes);
    }
    // Starts the copy of the next step; behind the last, of nothing.
    __device__ __forceinline__ void fetch(int wave, int lane) {
        copy.start(next, k, v, size_k, size_v, next_stage < stages ? rows : 0, k_cols, v_cols, wave, lane);
        next = next + Shape::kStageBytes == base + Shape::kLds ? base : next + Shape::kStageBytes;
        // (sums, not a choice among members, for which the compiler keeps them in memory)
        const bool last_head = next_head + 1 == heads, jump = last_head && next_stage == own - 1;
        k += to_head_k + (last_head ? to_next_k : 0) + (jump ? to_other_k : 0);
        v += to_head_v + (last_head ? to_next_v : 0) + (jump ? to_other_v : 0);
        rows += (last_head ? -Shape::kRows : 0) + (jump ? to_other_rows : 0);
        next_stage += last_head ? 1 : 0;
        next_head = last_head ? 0 : next_head + 1;
    }
    // The next stage is there, and all waves are done with the one before, whose
    // place the copy that starts here fills.
    __device__ __forceinline__ void advance(int wave, int lane) {
        own_copies_done<(Shape::kStages - 2) * Shape::kPer>();
        __syncthreads();
        fetch(wave, lane);
    }
};

// Waves of a workgroup, and bytes of the factors of a tile on the diagonal.
constexpr int kPassWaves = kLinearRows / kLinearTile;
constexpr int kDiagonalBytes = kLinearTile * kLinearTile * 4;
template <typename T, int D, int COLUMNS>
using PassShape = StageShape<T, D, COLUMNS, kPassWaves, kDiagonalBytes>;

inline long long pass_blocks(const LinearPass& a, int columns) {
    return (long long)a.n * a.hk * a.q_heads * ((a.dv + columns - 1) / columns) * ((a.s + kLinearRows - 1) / kLinearRows);
}

// One workgroup: 128 query rows of one head, COLUMNS columns; a wave takes 32 of
// the rows.  Scores are computed transposed (keys down, queries across the
// lanes), so that they are in place as the operand of the product with the values.
//
// The decay of a pair in tiles m >= 1 apart, with a the query's and b the key's
// place in its tile, is decay^(32 (m - 1) + a) of the lane times decay^(32 - b) of
// the register, neither of which can overflow.
//
// Bound by memory and the waits for it: 4 x 16384 tokens of 16 heads of 64 / 128 in bf16
// move 939 MB in 263-286 us, with the matrix instructions running 24 % and vector ones
// issued 29 % of the time; single segments of 784 tokens (32-33 us, 30 % and 31 %) by the
// chain of a wave's tiles.
template <typename T, int D, int COLUMNS, bool WIDE>
__device__ __forceinline__ void linear_pass(const LinearPass& a, int block, int blocks) {
    using Shape = PassShape<T, D, COLUMNS>;
    static_assert(Shape::kPassOccupancy * (Shape::kLds + kDiagonalBytes) <= kLinearLds, "the workgroups aimed at fit");
    constexpr int kTile = kLinearTile, kSteps = D / 16, kBlocks = COLUMNS / 32;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (the tiles, columns and query heads of one head next to one another, the
    // tiles with most keys first)
    const int slices = (a.dv + COLUMNS - 1) / COLUMNS, row_tiles = (a.s + kLinearRows - 1) / kLinearRows;
    int id = xcd_logical_block(block, blocks);
    const int column0 = linear_scalar(id % slices * COLUMNS);
    id /= slices;
    const int member = linear_scalar(id % a.q_heads);
    id /= a.q_heads;
    const int place = linear_scalar(id % row_tiles), head = linear_scalar(id / row_tiles);
    const int h = linear_scalar(head % a.hk), b = linear_scalar(head / a.hk);
    const int row0 = (a.reverse ? place : row_tiles - 1 - place) * kLinearRows;
    const float log2_decay = decay_log2(linear_uniform(a.log_decay + h));
    const int length = linear_length(a.lengths, a.s, b);
    const size_t o_row = size_t(a.hk) * a.q_heads * a.dv;
    const int own0 = row0 + kTile * wave, row = own0 + (lane & 31);
    T* o = static_cast<T*>(a.o) + (size_t(b) * a.s + row) * o_row + (size_t(h) * a.q_heads + member) * a.dv;
    floatx16 out[kBlocks];
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) out[c] = zero16();

    if (row0 < length) {
        const int segment = linear_scalar(row0 / a.segment_tokens), begin = segment * a.segment_tokens;
        const int end = int(min((long long)begin + a.segment_tokens, (long long)length));
        // first the keys of the workgroup's own rows, then those further on (all of them
        // before its rows, backwards behind them)
        const int own_end = min(row0 + kLinearRows, end);
        KeyStream<T, D, COLUMNS, kPassWaves, kDiagonalBytes, WIDE> stream(
            a, unsigned(reinterpret_cast<uintptr_t>(lds)), b, h, column0, row0, own_end, a.reverse ? own_end : begin,
            a.reverse ? end : row0, wave, lane);
        for (int i = 0; i + 1 < Shape::kStages; ++i) stream.fetch(wave, lane);
        Operand<T> q[kSteps];
        load_row_operands<T, D, WIDE>(q, static_cast<const T*>(a.q.p) + b * a.q.b + row * a.q.t +
                                             ((long long)h * a.q_heads + member) * a.q.h, a.d, row < length, lane);
        const int query = lane & 31;
        // (in registers: what is read again behind a copy's start would be loaded again)
        const int reverse = linear_scalar(a.reverse), k_heads = linear_scalar(a.k_heads);
        const float pair_scale = linear_scalar(a.pair_scale);
        // decay^(32 - b) (backwards decay^b) of b = acc_row(r, hi), as a product
        float eights[4], ones[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            eights[r] = pair_scale * decay_power(log2_decay, reverse ? 8 * r : 24 - 8 * r);
            ones[r] = decay_power(log2_decay, reverse ? 4 * hi + r : 8 - 4 * hi - r);
        }
        const float place0 = float(reverse ? kTile - query : query) - float(kTile);
        // the factors of a wave's own tile, which no such product can give: in LDS, as
        // the registers of a lane
        float4* diagonal = reinterpret_cast<float4*>(lds + Shape::kLds);
        {
            const int i = threadIdx.x >> 6;
            float e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = acc_row(4 * i + j, hi), apart = reverse ? key - query : query - key;
                e[j] = apart >= 0 ? pair_scale * decay_power(log2_decay, apart) : 0.f;
            }
            diagonal[i * 64 + lane] = make_float4(e[0], e[1], e[2], e[3]);
        }
        if (a.starts) {
            // what came before the segment
            constexpr int kParts = Precise<T>::kParts;
            const int rows = linear_steps(a.d), all = (a.dv + 31) / 32;
            const Operand<T>* p = static_cast<const Operand<T>*>(a.starts) +
                                  (size_t(head) * a.segments + segment) * all * rows * kParts * 64 + lane;
            // (as many loads side by side as the registers hold, of strips that exist: the
            // columns behind the last are not stored)
            constexpr int kAll = kBlocks * kSteps * kParts, kGroup = kAll < 16 / int(sizeof(T)) ? kAll : 16 / int(sizeof(T));
            Operand<T> x[2][kGroup];
            auto load = [&](int j) {
#pragma unroll
                for (int i = j; i < j + kGroup; ++i)
                    x[j / kGroup % 2][i - j] =
                        p[size_t((min(column0 / 32 + i / kParts / kSteps, all - 1) * rows + i / kParts % kSteps) * kParts +
                                 i % kParts) * 64];
            };
            load(0);
#pragma unroll
            for (int j = 0; j < kAll; j += kGroup) {
                if (j + kGroup < kAll) load(j + kGroup);
                in_order();
#pragma unroll
                for (int i = j; i < j + kGroup; ++i)
                    mma(out[i / kParts / kSteps], x[j / kGroup % 2][i - j], q[i / kParts % kSteps]);
            }
            const float f = a.inter_scale * decay_power(log2_decay, max(a.reverse ? end - 1 - row : row - begin + 1, 0));
#pragma unroll
            for (int c = 0; c < kBlocks; ++c)
#pragma unroll
                for (int r = 0; r < 16; ++r) out[c][r] *= f;
        }
        settle(q);
        const unsigned k_row = stream.base + row_lane<T, D>(lane);
        const unsigned v_column = stream.base + column_lane<T, COLUMNS>(lane) + Shape::kRowBytes;
        constexpr int kTiles = Shape::kRows / kTile;
        // TILES tiles of a stage, from its tile j on, side by side; operands are read
        // kAhead products before they are used.  weigh(s, t): scores become terms.
        auto take = [&](auto tiles, int stage, int j, auto weigh) {
            constexpr int TILES = decltype(tiles)::value;
            constexpr int kScores = TILES * kSteps, kEnd = kScores + 2 * TILES * kBlocks, kAhead = Shape::kPassAhead;
            const unsigned k_at = k_row + stage + j * kTile * int(sizeof(T)) * D;
            const unsigned v_at = v_column + stage + j * kTile * int(sizeof(T)) * COLUMNS;
            floatx16 s[TILES];
            Operand<T> ring[kAhead + 1];
            Precise<T> p[2 * TILES];
#pragma unroll
            for (int t = 0; t < TILES; ++t) s[t] = zero16();
            auto read = [&](int i) {
                if (i >= kEnd) return;
                const int v = i - kScores;
                ring[i % (kAhead + 1)] =
                    i < kScores ? read_row<T, D>(k_at, kTile * (i % TILES), i / TILES)
                                : read_column<T, COLUMNS>(v_at, kTile * (v / kBlocks / 2), 32 * (v % kBlocks), v / kBlocks % 2);
            };
#pragma unroll
            for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
            for (int i = 0; i < kEnd; ++i) {
                in_order();
                read(i + kAhead);
                in_order();
                if (i == kScores) {
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        weigh(s[t], t);
                        p[2 * t].set(s[t], 0);
                        p[2 * t + 1].set(s[t], 1);
                    }
                }
                const Operand<T>& x = ring[i % (kAhead + 1)];
                const int v = i - kScores;
                if (i < kScores) {
                    mma(s[i % TILES], x, q[i / TILES]);
                } else {
#pragma unroll
                    for (int j = 0; j < Precise<T>::kParts; ++j) mma(out[v % kBlocks], x, p[v / kBlocks].part[j]);
                }
            }
        };
        // Terms of a tile `between` tokens from the wave's own.
        auto apart = [&](floatx16& s, int between) {
            const float far = __builtin_amdgcn_exp2f(log2_decay * (place0 + float(between)));
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] *= eights[r / 4] * far * ones[r % 4];
        };
        int stage = 0;
        const int own_tile = wave, step = reverse ? 1 : -1;
        for (int n = 0; n < stream.own; ++n)
            for (int g = 0; g < k_heads; ++g) {
                stream.advance(wave, lane);
#pragma unroll 1
                for (int j = 0; j < kTiles; ++j) {
                    const int between = (n * kTiles + j - own_tile) * step;
                    if (between < 0) continue;
                    take(std::integral_constant<int, 1>{}, stage, j, [&](floatx16& s, int) {
                        if (between) {
                            apart(s, between * kTile);
                        } else {
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const float4 e = diagonal[r * 64 + lane];
                                s[4 * r] *= e.x;
                                s[4 * r + 1] *= e.y;
                                s[4 * r + 2] *= e.z;
                                s[4 * r + 3] *= e.w;
                            }
                        }
                    });
                }
                stage = stage + Shape::kStageBytes == Shape::kLds ? 0 : stage + Shape::kStageBytes;
            }
        int between = reverse ? kLinearRows - own_tile * kTile : own0 - begin;
        for (int n = stream.own; n < stream.stages; ++n, between += step * Shape::kRows)
            for (int g = 0; g < k_heads; ++g) {
                stream.advance(wave, lane);
                take(std::integral_constant<int, kTiles>{}, stage, 0,
                     [&](floatx16& s, int t) { apart(s, between + step * kTile * t); });
                stage = stage + Shape::kStageBytes == Shape::kLds ? 0 : stage + Shape::kStageBytes;
            }
        // (no copy may be on its way to the LDS of a workgroup that has ended)
        own_copies_done<0>();
    }
    if (row >= a.s) return;
    const bool there = row < length;                 // (tokens behind the last: zero)
#pragma unroll
    for (int c = 0; c < kBlocks; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            store4(o, column0 + 32 * c + acc_row(4 * r, hi), a.dv, WIDE || a.o_wide, there ? out[c][4 * r] : 0.f,
                   there ? out[c][4 * r + 1] : 0.f, there ? out[c][4 * r + 2] : 0.f, there ? out[c][4 * r + 3] : 0.f);
}

}  // namespace fftsplit
