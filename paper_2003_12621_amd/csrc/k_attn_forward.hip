// Differential attention, forward: o = (softmax(q1 k1^T) - lam softmax(q2 k2^T)) v.
//
// Each map is taken in one pass over the keys with a running maximum and sum
// and an output accumulator of its own: the two softmax denominators are known
// only at the end, where the outputs are joined.  With values as wide as both
// maps together that costs what a second pass over the keys for the
// denominators would (4 d + 4 dv operations per query and key, or 8 d + 2 dv).
#include "attn_common.hpp"

namespace fftsplit {

namespace {

// Growth of the running maximum (in powers of two) up to which sums and
// outputs are kept relative to the old one.  Terms are then at most 2^8, far
// from overflow, and rounding is relative, so the result is as precise; the
// accumulators are rescaled a few times per row instead of at every tile.
constexpr float kMaxSlack = 8.f;

// Running softmax of one map for the query in this lane's column.
struct RowState {
    float m, l;     // reference maximum (log2 units), sum of this half's terms
};
// Before a row has seen a key: below every score, but finite, so that the terms
// of hidden keys are zero.
constexpr float kNoMax = -3e38f;

// Scores of 32 keys become terms exp2(score - m); `acc` is rescaled where the
// reference maximum moves.  (The maximum of three NaNs is one, and stays out of
// m: a NaN score makes its row NaN through its term.)
template <int DT>
__device__ __forceinline__ void softmax_step(floatx16& s, RowState& st, floatx16 (&acc)[DT], float scale_log2) {
    float top = vmax(s[0], s[1]);
#pragma unroll
    for (int r = 2; r < 16; r += 2) top = vmax3(top, s[r], s[r + 1]);
    const float2 t2 = both_halves(top);
    top = vmax(t2.x, t2.y) * scale_log2;
    if (__ballot(top > st.m + kMaxSlack) != 0) {
        const float m = top > st.m ? top : st.m;
        const float alpha = exp2_fast(st.m - m);
        st.m = m;
        st.l *= alpha;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[d][r] *= alpha;
    }
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        s[r] = exp2_fast(fmaf(s[r], scale_log2, -st.m));
        sum += s[r];
    }
    st.l += sum;
}

// Hides keys beyond `last` (of the lane's query) in a score tile of keys key0 ...
__device__ __forceinline__ void mask_scores(floatx16& s, int key0, int last, int hi) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = acc_row(r, hi) > last - key0 ? -kInf : s[r];
}

// A wave takes one map of 32 query rows: two waves work on the first map and
// two on the second of the same rows, and their outputs are joined through LDS
// at the end.  That leaves a lane 128 registers' worth of state at 128-wide
// values, so that four workgroups a compute unit hide one another's waits: with
// 64 rows a wave, which reads half as many operands from LDS, and two
// workgroups, 4 x 8 heads of 3136 x 3136 (bf16, 64 / 128 wide) took 366 us, not
// 305.
template <typename T, int D, int DV>
struct ForwardShape {
    static constexpr int kWaves = 4;
    static constexpr int kThreads = 64 * kWaves;
    // Keys per stage: 64 where four such double buffers fit a compute unit's LDS
    // (4 x 1024 tokens of 8 heads of 32 / 64: 30.9 us; with 32 keys 34.1).
    static constexpr int kKeys = sizeof(T) * DV <= 128 ? 64 : 32;
    // Operands from LDS are read this many products before they are used: one,
    // and two where two waves a SIMD have the registers for it (2 x 1999 causal
    // tokens of 8 heads of 128 / 256, bf16: 83.5 us; none 88.5, one 85.3, four
    // 83.9).  With four waves a SIMD one is no faster than none in bf16 (4 x 3136,
    // 64 / 128: 303 and 306 us), but in fp32 (6 x 301, 32 / 64: 26.7 and 28.1 us),
    // and two do not fit.
    static constexpr int kAhead = sizeof(T) == 2 && D == 128 ? 2 : 1;
    // workgroups per compute unit aimed at
    static constexpr int kBlocks = sizeof(T) * DV <= 256 ? 4 : (sizeof(T) * DV <= 512 ? 2 : 1);
    static constexpr int kKeyBytes = TileShape<T, D>::bytes(kKeys);
    static constexpr int kBufferBytes = 2 * kKeyBytes + TileShape<T, DV>::bytes(kKeys);
    static constexpr int kJoinBytes = kAttnTiledRows * DV * 4;
    static constexpr int kLds = 2 * kBufferBytes > kJoinBytes ? 2 * kBufferBytes : kJoinBytes;
};

}  // namespace

// One workgroup: 64 query rows of one head; the keys pass through LDS in
// double-buffered stages that all waves read.  Scores are computed transposed
// (keys down, queries across the lanes): a lane then holds 16 scores of one
// query, whose maximum and sum need one exchange with the other half wave, and
// the terms stay in the lane as the next product's operand.  The terms enter it
// rounded to bf16 (the sum is of the unrounded ones): 1.66e-3 of each map's output
// with random inputs, as much as the output's own rounding to bf16 adds.  Where
// the maps cancel it is that of the maps, not of their difference: with a
// difference of a tenth of either, 1e-2 of the output (fp32 tensors keep all).  A
// second product with what the rounding left out, which the kernel for few rows
// has time for, is two thirds more matrix instructions here: 441, 285, 50 and 81
// us of the four calls below became 705, 409, 68 and 102.
//
// Bound by issue: at 8192 causal tokens of 16 heads (bf16, 64 / 128) vector
// instructions are issued 77 % and matrix instructions run 62 % of a compute
// unit's busy time, both 32 %, with no LDS read conflicts; the units are busy 86 %
// of the launch (what is left is its ends).  Of the cycles that issue vector
// instructions the matrix instructions take 10 %, and the softmax's fma,
// exponential (two cycles), sum and conversion of each term 61 %.  Measured (bf16,
// 4 d + 4 dv operations for each visible pair; from many calls in a stream to a
// few under the profiler, on several machines):
//     8192 x 8192 causal, 16 heads (4 of keys), 64 / 128    407-489 us  840-1010 TFLOP/s
//     4 x 3136 x 3136, 8 heads, 64 / 128                    285-305 us  790-850 TFLOP/s
//     8 x 784 x 784, 8 heads, 64 / 128                        46-51 us  590-660 TFLOP/s
//     2 x 1999 x 1999 causal, 8 heads (4), 128 / 256          80-86 us  570-610 TFLOP/s
template <typename T, int D, int DV, bool WIDE>
__global__ __launch_bounds__((ForwardShape<T, D, DV>::kThreads), (ForwardShape<T, D, DV>::kBlocks)) void
attn_forward_kernel(AttnArgs a) {
    using Shape = ForwardShape<T, D, DV>;
    constexpr int kKeys = Shape::kKeys, DT = DV / 32;
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, hi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), map = wave & 1, group = wave >> 1;
    const int tiles = (a.sq + kAttnTiledRows - 1) / kAttnTiledRows;
    const AttnPlace place = attn_place(a, tiles, a.n * a.hq, 1);
    const int tile = tiles - 1 - place.place, h = place.head % a.hq, b = place.head / a.hq;
    const int hkv = h / (a.hq / a.hk);
    const int length = attn_length(a, b);

    const int first = tile * kAttnTiledRows + group * 32, row = first + (lane & 31);
    const int first_last = attn_last_key(a, first, length);          // last key of the wave's first row
    const int wave_end = attn_last_key(a, min(first + 32, a.sq) - 1, length) + 1;
    const int end = attn_last_key(a, min(tile * kAttnTiledRows + kAttnTiledRows, a.sq) - 1, length) + 1;

    const T* k1 = static_cast<const T*>(a.k) + b * a.kb + hkv * a.kh;
    const T* v = static_cast<const T*>(a.v) + b * a.vb + hkv * a.vh;

    Operand<T> q[D / 16];
    load_row_operands<T, D, WIDE>(
        q, static_cast<const T*>(a.q) + b * a.qb + (long long)row * a.qt + h * a.qh + map * a.qm, a.d, row < a.sq, lane);
    settle(q);
    floatx16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = zero16();
    RowState st{kNoMax, 0.f};
    const int last = attn_last_key(a, row, length);

    using KeyCopy = RowCopy<T, D, kKeys, Shape::kThreads, WIDE>;
    using ValueCopy = RowCopy<T, DV, kKeys, Shape::kThreads, WIDE>;
    const KeyCopy key_copy(a.kt, a.d, tid);
    const ValueCopy value_copy(a.vt, a.dv, tid);
    const unsigned base = unsigned(reinterpret_cast<uintptr_t>(lds));
    const unsigned key_lane = row_lane<T, D>(lane) + map * Shape::kKeyBytes;
    const unsigned value_lane = column_lane<T, DV>(lane) + 2 * Shape::kKeyBytes;
    auto fetch = [&](int key, unsigned buffer) {
        key_copy.start(buffer, k1 + (long long)key * a.kt, a.kt, end - key, tid);
        key_copy.start(buffer + Shape::kKeyBytes, k1 + a.km + (long long)key * a.kt, a.kt, end - key,
                       tid);
        value_copy.start(buffer + 2 * Shape::kKeyBytes, v + (long long)key * a.vt, a.vt, end - key,
                         tid);
    };
    if (end > 0) fetch(0, base);
    for (int i = 0, key = 0; key < end; ++i, key += kKeys) {
        const unsigned buffer = base + (i & 1) * Shape::kBufferBytes;
        const unsigned tk = buffer + key_lane, tv = buffer + value_lane;
        // this stage is there, and all waves are done with the other buffer
        copies_done();
        if (key + kKeys < end) fetch(key + kKeys, base + ((i + 1) & 1) * Shape::kBufferBytes);
#pragma unroll
        for (int sub = 0; sub < kKeys; sub += 32) {
            const int key0 = key + sub;
            if (key0 >= wave_end) break;
            floatx16 c = zero16();
            constexpr int kT = D / 16, kEnd = kT + DV / 16, kAhead = Shape::kAhead;
            Operand<T> ring[kAhead + 1];
            auto read = [&](int i) {
                if (i >= kEnd) return;
                if (i < kT)
                    ring[i % (kAhead + 1)] = read_row<T, D>(tk, sub, i);
                else
                    ring[i % (kAhead + 1)] = read_column<T, DV>(tv, sub, 32 * ((i - kT) % DT), (i - kT) / DT);
            };
            Operand<T> p[2];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
            for (int i = 0; i < kEnd; ++i) {
                in_order();
                read(i + kAhead);
                in_order();
                const Operand<T>& x = ring[i % (kAhead + 1)];
                if (i == kT) {
                    if (key0 + 31 > first_last) mask_scores(c, key0, last, hi);
                    softmax_step(c, st, o, a.scale_log2);
                    p[0] = acc_operand<T>(c, 0);
                    p[1] = acc_operand<T>(c, 1);
                }
                if (i < kT)
                    mma(c, x, q[i]);
                else
                    mma(o[(i - kT) % DT], x, p[(i - kT) / DT % 2]);
            }
        }
    }

    // each map's own output, then the second map's scaled by lam to the waves of the first
    const bool none = last < 0;                        // no key is visible: the row is zero, whatever lam is
    const float lam = none ? 0.f : attn_lambda(a, h);
    float4* join = reinterpret_cast<float4*>(lds) + group * (DT * 4 * 64) + lane;
    const float2 halves = both_halves(st.l);
    const float l = halves.x + halves.y;
    const float inv = 1.f / l;
    const bool valid = row < a.sq;
    const size_t at = ((size_t(b) * a.sq + row) * a.hq + h) * a.dv;
    float* own = a.o1 && valid ? (map ? a.o2 : a.o1) + at : nullptr;
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
#pragma unroll
            for (int j = 0; j < 4; ++j) o[d][4 * g + j] = none ? 0.f : o[d][4 * g + j] * inv;
            const float4 y = make_float4(o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]);
            if (own) store4(own, 32 * d + acc_row(4 * g, hi), a.dv, a.o_wide, y.x, y.y, y.z, y.w);
            if (map) join[(d * 4 + g) * 64] = make_float4(y.x * lam, y.y * lam, y.z * lam, y.w * lam);
        }
    if (a.lse && hi == 0 && valid)
        a.lse[((size_t(b) * a.hq + h) * 2 + map) * a.sq + row] = none ? 0.f : st.m + log2f(l);
    __syncthreads();
    if (map || !valid) return;
    T* out = static_cast<T*>(a.o) + at;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 z = join[(d * 4 + g) * 64];
            store4(out, 32 * d + acc_row(4 * g, hi), a.dv, a.o_wide, o[d][4 * g] - z.x, o[d][4 * g + 1] - z.y,
                   o[d][4 * g + 2] - z.z, o[d][4 * g + 3] - z.w);
        }
}

// ---- few rows: single tokens over a long cache ----
//
// Bound by reading k and v once: 41 to 44 us for the 201 MB of 16 sequences' caches
// of up to 8192 keys (4.6 to 4.9 TB/s; a copy reaches 4.8).  The rows of all heads that share a key head
// are packed into tiles of 32, and the keys of a tile are shared by several
// workgroups, whose partial results a second kernel joins.  Within a
// workgroup every wave goes over key blocks of its own, copied into LDS of its
// own, so nothing waits at a barrier; the waves are joined at the end.  The
// matrix instructions have time to spare, so the terms of the softmax enter as
// two bf16 numbers (the rounded term and what that left out).

namespace {

template <typename T, int D, int DV>
struct FewShape {
    static constexpr int kKeys = 32;
    // Maps a wave takes: both, or one where the outputs of both would take 256
    // registers (the two waves of a block then each copy its values).
    static constexpr int kMaps = DV <= 128 ? 2 : 1;
    static constexpr int kKeyBytes = TileShape<T, D>::bytes(kKeys);
    static constexpr int kStageBytes = kMaps * kKeyBytes + TileShape<T, DV>::bytes(kKeys);
    // the next stage on its way while one is worked on, in at most 128 KB
    static constexpr int kBuffers = kStageBytes <= 16384 || kMaps == 2 ? 2 : 1;
    static constexpr int kWaves = kStageBytes <= (kMaps == 2 ? 16384 : 24576) ? 4 : 2;
    static constexpr int kKeyWaves = kWaves * kMaps / 2;                // key blocks worked on at a time
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kJoinBytes = kMaps * (DV / 32) * 16 * 64 * 4;  // a wave's outputs
    static constexpr int kStatBytes = kKeyWaves * 2 * 2 * 32 * 4;
    static constexpr int kTileBytes = kBuffers * kStageBytes > kJoinBytes ? kBuffers * kStageBytes : kJoinBytes;
    static constexpr int kLds = kWaves * kTileBytes + kStatBytes;
};

// The rounding error of an operand's elements, as an operand.
__device__ __forceinline__ Operand<__bf16> rest_operand(const floatx16& c, const Operand<__bf16>& rounded, int s) {
    floatx16 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = c[8 * s + e] - float(rounded.v[e]);
    return acc_operand<__bf16>(r, 0);
}

}  // namespace

template <typename T, int D, int DV, bool WIDE>
__global__ __launch_bounds__((FewShape<T, D, DV>::kThreads)) void attn_few_rows_kernel(AttnArgs a) {
    using Shape = FewShape<T, D, DV>;
    constexpr int kWaves = Shape::kWaves, kKeyWaves = Shape::kKeyWaves, MAPS = Shape::kMaps, DT = DV / 32;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int key_wave = MAPS == 2 ? wave : wave >> 1, map0 = MAPS == 2 ? 0 : wave & 1;
    const int group = a.hq / a.hk, rows = group * a.sq, tiles = (rows + kAttnFewRows - 1) / kAttnFewRows;
    const int id = xcd_logical_block(blockIdx.x, gridDim.x);
    // (the tiles of one key head and share of the keys next to one another)
    const int tile = id % tiles, split = id / tiles % a.splits, hkv = id / tiles / a.splits % a.hk;
    const int b = id / tiles / a.splits / a.hk;
    const int length = attn_length(a, b);
    const int packed = tile * kAttnFewRows + (lane & 31);
    const bool valid = packed < rows;
    const int head = hkv * group + (valid ? packed / a.sq : 0), i = valid ? packed % a.sq : 0;
    const int last = valid ? attn_last_key(a, i, length) : -1;
    // this workgroup's keys: a whole number of blocks for each wave
    constexpr int kStep = Shape::kKeys * kKeyWaves;
    const int share = ((length + a.splits - 1) / a.splits + kStep - 1) / kStep * kStep;
    const int begin = int(min(split * (long long)share, (long long)length)), end = min(begin + share, length);

    const T* k = static_cast<const T*>(a.k) + b * a.kb + hkv * a.kh + map0 * a.km;
    const T* v = static_cast<const T*>(a.v) + b * a.vb + hkv * a.vh;
    Operand<T> q[MAPS][D / 16];
    floatx16 o[MAPS][DT];
    RowState st[MAPS];
#pragma unroll
    for (int m = 0; m < MAPS; ++m) {
        load_row_operands<T, D, WIDE>(
            q[m], static_cast<const T*>(a.q) + b * a.qb + (long long)i * a.qt + head * a.qh + (map0 + m) * a.qm, a.d, valid,
            lane);
        settle(q[m]);
#pragma unroll
        for (int d = 0; d < DT; ++d) o[m][d] = zero16();
        st[m] = RowState{kNoMax, 0.f};
    }

    using KeyCopy = RowCopy<T, D, Shape::kKeys, 64, WIDE>;
    using ValueCopy = RowCopy<T, DV, Shape::kKeys, 64, WIDE>;
    const KeyCopy key_copy(a.kt, a.d, lane);
    const ValueCopy value_copy(a.vt, a.dv, lane);
    constexpr int kCopies = MAPS * KeyCopy::kCopies + ValueCopy::kCopies;
    const unsigned base = unsigned(reinterpret_cast<uintptr_t>(lds)) + wave * Shape::kTileBytes;
    const unsigned key_lane = row_lane<T, D>(lane), value_lane = column_lane<T, DV>(lane) + MAPS * Shape::kKeyBytes;
    auto fetch = [&](int key, unsigned buffer) {
#pragma unroll
        for (int m = 0; m < MAPS; ++m)
            key_copy.start(buffer + m * Shape::kKeyBytes, k + m * a.km + (long long)key * a.kt, a.kt, end - key, lane);
        value_copy.start(buffer + MAPS * Shape::kKeyBytes, v + (long long)key * a.vt, a.vt, end - key, lane);
    };
    int key = begin + key_wave * Shape::kKeys;
    if (Shape::kBuffers == 2 && key < end) fetch(key, base);
    for (int n = 0; key < end; ++n, key += kStep) {
        unsigned buffer = base;
        own_reads_done();
        if constexpr (Shape::kBuffers == 2) {
            buffer += (n & 1) * Shape::kStageBytes;
            if (key + kStep < end) {
                fetch(key + kStep, base + ((n + 1) & 1) * Shape::kStageBytes);
                own_copies_done<kCopies>();
            } else {
                own_copies_done<0>();
            }
        } else {
            fetch(key, buffer);
            own_copies_done<0>();
        }
        const unsigned tk = buffer + key_lane, tv = buffer + value_lane;
        floatx16 c[MAPS];
#pragma unroll
        for (int m = 0; m < MAPS; ++m) c[m] = zero16();
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int m = 0; m < MAPS; ++m) mma(c[m], read_row<T, D>(tk + m * Shape::kKeyBytes, 0, s), q[m][s]);
#pragma unroll
        for (int m = 0; m < MAPS; ++m) {
            mask_scores(c[m], key, last, hi);
            softmax_step(c[m], st[m], o[m], a.scale_log2);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            Operand<T> p[MAPS], e[MAPS];
#pragma unroll
            for (int m = 0; m < MAPS; ++m) {
                p[m] = acc_operand<T>(c[m], s);
                if constexpr (sizeof(T) == 2) e[m] = rest_operand(c[m], p[m], s);
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const Operand<T> x = read_column<T, DV>(tv, 0, 32 * d, s);
#pragma unroll
                for (int m = 0; m < MAPS; ++m) {
                    mma(o[m][d], x, p[m]);
                    if constexpr (sizeof(T) == 2) mma(o[m][d], x, e[m]);
                }
            }
        }
    }

    // join the waves: outputs relative to the largest maximum, added up through LDS
    float* stats = reinterpret_cast<float*>(lds + kWaves * Shape::kTileBytes);   // [key wave][map][maximum, sum][32]
#pragma unroll
    for (int m = 0; m < MAPS; ++m) {
        const float2 halves = both_halves(st[m].l);
        if (hi == 0) {
            float* x = stats + (key_wave * 2 + map0 + m) * 64 + lane;
            x[0] = st[m].m;
            x[32] = halves.x + halves.y;
        }
    }
    __syncthreads();
    float top[2] = {kNoMax, kNoMax}, sum[2] = {0.f, 0.f};
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const float* x = stats + m * 64 + (lane & 31);
#pragma unroll
        for (int w = 0; w < kKeyWaves; ++w) top[m] = fmaxf(top[m], x[w * 128]);
#pragma unroll
        for (int w = 0; w < kKeyWaves; ++w)
            sum[m] = fmaf(exp2_fast(x[w * 128] - top[m]), x[w * 128 + 32], sum[m]);
    }
    {
        float4* own = reinterpret_cast<float4*>(lds + wave * Shape::kTileBytes) + lane;
#pragma unroll
        for (int m = 0; m < MAPS; ++m) {
            const float f = exp2_fast(st[m].m - (map0 + m ? top[1] : top[0]));
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    own[((m * DT + d) * 4 + g) * 64] = make_float4(o[m][d][4 * g] * f, o[m][d][4 * g + 1] * f,
                                                                   o[m][d][4 * g + 2] * f, o[m][d][4 * g + 3] * f);
        }
    }
    __syncthreads();
    if (!valid) return;
    const size_t at = ((size_t(b) * a.hk + hkv) * rows + packed) * a.splits + split;
    if (wave == 0 && hi == 0)
        *reinterpret_cast<float4*>(a.part_stats + at * 4) = make_float4(top[0], sum[0], top[1], sum[1]);
    for (int e = wave; e < 2 * DT * 4; e += kWaves) {
        const int m = e / (DT * 4), d = e / 4 % DT, g = e % 4;
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kKeyWaves; ++w) {
            const char* from = lds + (MAPS == 2 ? w : 2 * w + m) * Shape::kTileBytes;
            const float4 x = reinterpret_cast<const float4*>(from)[(MAPS == 2 ? e : e % (DT * 4)) * 64 + lane];
            t = make_float4(t.x + x.x, t.y + x.y, t.z + x.z, t.w + x.w);
        }
        *reinterpret_cast<float4*>(a.part + (at * 2 + m) * DV + 32 * d + acc_row(4 * g, hi)) = t;
    }
}

// Joins the workgroups that shared a row's keys: 128 threads a row, 64 a map, 4
// columns each.  Bound by its own latency: 4.2 to 4.8 us for 256 rows of 4 parts.
template <typename T, int DV>
__global__ __launch_bounds__(128) void attn_few_rows_join_kernel(AttnArgs a) {
    __shared__ float4 second[64];
    const int map = threadIdx.x >> 6, col = 4 * (threadIdx.x & 63);
    const int group = a.hq / a.hk, rows = group * a.sq;
    const int packed = blockIdx.x % rows, kv = blockIdx.x / rows, b = kv / a.hk, h = kv % a.hk * group + packed / a.sq;
    const int i = packed % a.sq;
    const float4* stats = reinterpret_cast<const float4*>(a.part_stats) + size_t(blockIdx.x) * a.splits;
    float top = kNoMax;
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, map ? stats[s].z : stats[s].x);
    float sum = 0.f;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < a.splits; ++s) {
        const float4 st = stats[s];
        const float m = map ? st.z : st.x, l = map ? st.w : st.y;
        // (no key was visible.  A share whose only scores are NaN has no maximum
        // either, but a sum, which makes the row NaN.)
        if (l == 0.f) continue;
        const float f = exp2_fast(m - top);
        sum = fmaf(l, f, sum);
        if (col < DV) {
            const float4 x = *reinterpret_cast<const float4*>(a.part + ((size_t(blockIdx.x) * a.splits + s) * 2 + map) * DV + col);
            y = make_float4(fmaf(x.x, f, y.x), fmaf(x.y, f, y.y), fmaf(x.z, f, y.z), fmaf(x.w, f, y.w));
        }
    }
    const bool none = attn_last_key(a, i, attn_length(a, b)) < 0;
    const float inv = 1.f / sum;
    y = none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
    const size_t at = ((size_t(b) * a.sq + i) * a.hq + h) * a.dv;
    if (a.o1) store4((map ? a.o2 : a.o1) + at, col, a.dv, a.o_wide, y.x, y.y, y.z, y.w);
    if (a.lse && col == 0)
        a.lse[((size_t(b) * a.hq + h) * 2 + map) * a.sq + i] = none ? 0.f : top + log2f(sum);
    if (map) second[threadIdx.x & 63] = y;
    __syncthreads();
    if (map) return;
    const float4 z = second[threadIdx.x];
    const float lam = none ? 0.f : attn_lambda(a, h);
    store4(static_cast<T*>(a.o) + at, col, a.dv, a.o_wide, y.x - lam * z.x, y.y - lam * z.y, y.z - lam * z.z,
           y.w - lam * z.w);
}

namespace {
template <typename T, int D, int DV>
hipError_t launch_tiled(const AttnArgs& a, hipStream_t s, const LaunchEvents& ev) {
    using Shape = ForwardShape<T, D, DV>;
    const long long blocks = (long long)a.n * a.hq * ((a.sq + kAttnTiledRows - 1) / kAttnTiledRows);
    auto kernel = a.wide ? attn_forward_kernel<T, D, DV, true> : attn_forward_kernel<T, D, DV, false>;
    if (hipError_t e = allow_dynamic_lds(kernel, Shape::kLds)) return e;
    return launch_kernel(kernel, dim3(unsigned(blocks)), dim3(Shape::kThreads), Shape::kLds, s, ev.start,
                         ev.stop, a);
}

template <typename T, int D, int DV>
hipError_t launch_few_rows(const AttnArgs& a, hipStream_t s, const LaunchEvents& ev) {
    using Shape = FewShape<T, D, DV>;
    const long long rows = (long long)(a.hq / a.hk) * a.sq, heads = (long long)a.n * a.hk;
    const long long blocks = heads * ((rows + kAttnFewRows - 1) / kAttnFewRows) * a.splits;
    auto kernel = a.wide ? attn_few_rows_kernel<T, D, DV, true> : attn_few_rows_kernel<T, D, DV, false>;
    if (hipError_t e = allow_dynamic_lds(kernel, Shape::kLds)) return e;
    if (hipError_t e = launch_kernel(kernel, dim3(unsigned(blocks)), dim3(Shape::kThreads), Shape::kLds, s, ev.start,
                                     nullptr, a))
        return e;
    return launch_kernel(attn_few_rows_join_kernel<T, DV>, dim3(unsigned(heads * rows)), dim3(128), 0, s, nullptr, ev.stop,
                         a);
}

template <typename T, int D, int DV>
hipError_t launch_shaped(const AttnArgs& a, hipStream_t s, const LaunchEvents& ev) {
    return a.splits ? launch_few_rows<T, D, DV>(a, s, ev) : launch_tiled<T, D, DV>(a, s, ev);
}

template <typename T>
hipError_t launch_typed(const fftsplit_attention_plan_s& p, const AttnArgs& a, hipStream_t s, const LaunchEvents& ev) {
    switch (p.shape) {
        case 0: return launch_shaped<T, 32, 64>(a, s, ev);
        case 1: return launch_shaped<T, 64, 128>(a, s, ev);
        default: return launch_shaped<T, 128, 256>(a, s, ev);
    }
}
}  // namespace

hipError_t launch_attn_forward(const fftsplit_attention_plan_s& p, const AttnArgs& a, hipStream_t s,
                               const LaunchEvents& ev) {
    return p.prob.dtype == FFTSPLIT_BF16 ? launch_typed<__bf16>(p, a, s, ev) : launch_typed<float>(p, a, s, ev);
}

}  // namespace fftsplit
