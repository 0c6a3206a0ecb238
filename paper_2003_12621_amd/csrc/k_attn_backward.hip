// Differential attention, backward.
//
// With P1, P2 the two maps (recomputed from the saved log sums), t = dO v^T and
// D1 = <dO, o1>, D2 = <dO, o2> per row:
//     dv = (P1 - lam P2)^T dO,   dlam = - sum P2 t,
//     dS1 = P1 (t - D1),   dS2 = lam P2 (D2 - t),
//     dqm = scale dSm km,   dkm = scale dSm^T qm.
// t and the value product are shared by both maps.  The key side (dk, dv) and
// the query side (dq) are two kernels that each own their outputs and
// recompute the scores, rather than one that would add to dq with atomics:
// results do not depend on the order of workgroups.  D1 and D2 come from the
// saved outputs, which are fp32: dS sums to zero over a row's keys, and an error
// of D is one of that sum, which a common part of the keys carries into dq (saved
// in bf16, 2e-2 of dq at 2 x 333 tokens with keys of mean 0.5 and values of mean
// 2; in fp32 3e-3).  dlam, a sum in which much cancels, comes in bf16 from the
// terms themselves (those of o1 and o2 are rounded), and in fp32 from the saved
// outputs, as - sum D2 (the log sums, of about 10, are rounded to 5e-7, which is
// each term's relative error).
#include <algorithm>

#include "attn_common.hpp"

namespace fftsplit {

namespace {

constexpr int kDeltaLanes = 16;   // lanes that share a row

// Sum over the 16 lanes of a row group, the same in all of them.
__device__ __forceinline__ float row_group_sum(float x) {
#pragma unroll
    for (int m = 1; m < kDeltaLanes; m *= 2) x += __shfl_xor(x, m, 64);
    return x;
}

template <typename T>
__device__ __forceinline__ void load8(float (&y)[8], const T* p, int left, bool wide) {
    if (wide && left >= 8) {
        T e[8];
#pragma unroll
        for (int j = 0; j < 8; j += 16 / int(sizeof(T)))
            *reinterpret_cast<uint4*>(e + j) = *reinterpret_cast<const uint4*>(p + j);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = float(e[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = j < left ? float(p[j]) : 0.f;
    }
}

}  // namespace

// -D1 and lam D2 of kAttnDeltaRows rows of one head, 16 lanes a row.  Bound by
// memory: 20 us for the 128 MB of 4 x 3136 rows of 8 heads of 128 (dO in bf16;
// 6.4 TB/s, part of it from the caches).
template <typename T>
__global__ __launch_bounds__(256) void attn_delta_kernel(AttnArgs a) {
    const int chunks = (a.sq + kAttnDeltaRows - 1) / kAttnDeltaRows;
    const int h = blockIdx.x % a.hq, c = blockIdx.x / a.hq % chunks, b = blockIdx.x / a.hq / chunks;
    const int l = threadIdx.x % kDeltaLanes, group = threadIdx.x / kDeltaLanes;
    const bool wide = a.wide && a.dv % 8 == 0;
    const float lam = attn_lambda(a, h);
    if (b == 0 && c == 0 && threadIdx.x == 0) a.lam32[h] = lam;
    for (int i = group; i < kAttnDeltaRows; i += 256 / kDeltaLanes) {
        const int row = c * kAttnDeltaRows + i;
        if (row >= a.sq) break;      // (the same in all lanes of the group)
        const size_t at = ((size_t(b) * a.sq + row) * a.hq + h) * a.dv;
        const float *o1 = a.o1 + at, *o2 = a.o2 + at;
        const T* g = static_cast<const T*>(a.dout) + b * a.gb + row * a.gt + h * a.gh;
        float s1 = 0.f, s2 = 0.f;
        for (int col = l * 8; col < a.dv; col += kDeltaLanes * 8) {
            float x[8], y[8], z[8];
            load8(x, g + col, a.dv - col, wide);
            load8(y, o1 + col, a.dv - col, wide);
            load8(z, o2 + col, a.dv - col, wide);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s1 = fmaf(x[j], y[j], s1);
                s2 = fmaf(x[j], z[j], s2);
            }
        }
        s1 = row_group_sum(s1);
        s2 = row_group_sum(s2);
        if (l == 0) {
            float* delta = a.delta + (size_t(b) * a.hq + h) * 2 * a.sq + row;
            delta[0] = -s1;
            delta[a.sq] = lam * s2;
            if constexpr (sizeof(T) == 4) a.second[(size_t(b) * a.hq + h) * a.sq + row] = s2;
        }
    }
}

namespace {

// What a workgroup of the key side computes: all gradients of its keys, those
// of one map's keys, or those of the values.
constexpr int kAll = 0, kOneMap = 1, kValues = 2;

constexpr int kKeySideKeys = 128;   // 4 waves of 32 keys

// At the largest widths the operands and accumulators of all gradients do not
// fit a lane's registers: separate workgroups compute them, and what they share
// (t, the scores) more than once.  In bf16 that is 3/2 and 4/3 of the products, but two
// workgroups run on a compute unit, not one: the two sides of 2 x 1999 causal
// tokens of 8 heads (4 key heads) take 136 and 90 us, not 259 and 147.  (fp32 at
// 64 / 128 would fit two as well; it is bound by the products: 466 and 303 us,
// not 342 and 256, at 4 x 1024 tokens of 8 heads.)
template <int D> constexpr bool kApart = D == 128;

// Operands from LDS are read this many products before they are used, as many as
// the registers have room for: one where all gradients are computed together (4 x
// 3136 tokens of 8 heads of 64 / 128, bf16, key side: 495 us; none 513, two 498,
// three 557, from scratch), two where they are not (2 x 1999 causal tokens of 8
// heads of 128 / 256, key and query side: 133 and 83 us; none 137 and 89, one 134
// and 86).
template <int D> constexpr int kOperandsAhead = kApart<D> ? 2 : 1;

template <typename T, int D, int DV, int DO>
struct KeySideShape {
    static constexpr int kRows = 32;                                   // queries per stage
    static constexpr int kMaps = DO == kOneMap ? 1 : 2;
    static constexpr int kQueryBytes = TileShape<T, D>::bytes(kRows);
    static constexpr int kGradBytes = TileShape<T, DV>::bytes(kRows);
    static constexpr int kStatBytes = 1024;                            // 4 values a row; tiles start at multiples of 1024
    static constexpr int kQueries = kMaps * kQueryBytes;
    static constexpr int kBufferBytes = kQueries + kGradBytes + kStatBytes;
    // workgroups a compute unit aimed at
    static constexpr int kBlocks = sizeof(T) * DV <= 256 || (sizeof(T) == 2 && kApart<D>) ? 2 : 1;
    // Where all gradients are computed by two workgroups a compute unit, the keys
    // stay in LDS: as operands in registers they would not leave room for that
    // (D / 2 of a lane's 256 registers, of which 250 are in use as it is).
    static constexpr bool kKeysInLds = sizeof(T) * DV <= 256;
    static constexpr int kKeyBytes = kKeysInLds ? TileShape<T, D>::bytes(kKeySideKeys) : 0;
    static constexpr int kLds = 2 * kBufferBytes + 2 * kKeyBytes;
};

// Four values of an array in LDS that belong to rows 4 g .. 4 g + 3 of a lane's
// accumulator registers.
__device__ __forceinline__ float4 rows_of(const float* x, int g, int hi) {
    return *reinterpret_cast<const float4*>(x + acc_row(4 * g, hi));
}

// A transposed accumulator [columns of the row][rows = lanes] to a dense row in memory.
template <typename T, int N>
__device__ __forceinline__ void store_row(T* p, const floatx16 (&acc)[N], int cols, bool wide, float scale, int hi) {
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            store4(p, 32 * d + acc_row(4 * g, hi), cols, wide, acc[d][4 * g] * scale, acc[d][4 * g + 1] * scale,
                   acc[d][4 * g + 2] * scale, acc[d][4 * g + 3] * scale);
}

}  // namespace

// Key side: one workgroup takes 128 keys of one key head, 32 a wave, and goes
// over the queries of all heads that share it (or over its share of them), 32 a
// step, double buffered in LDS with the statistics of their rows.  Each wave
// keeps its rows of k1, k2 and v as operands and dk1, dk2, dv as accumulators in
// registers.  (Heads that share a key head are summed in the accumulators: their
// gradients need no other sum.)  Deeper buffers were no faster.
//
// P1 - lam P2 and dS enter the products rounded to bf16, 1.66e-3 of a gradient of
// random inputs, as much as its own rounding adds; a common part of the other
// factor magnifies it.  Second products with what that leaves out find no
// registers at 64 / 128: the key side took 1010 us with them for dS and 1240 for
// both, not 505, and the query side 445, not 350 (4 x 3136 tokens of 8 heads).
//
// Bound by the chain scores - terms - t - dS - dk of a step and its reads from
// LDS, which two workgroups a compute unit (registers allow no third) hide in
// part: matrix instructions take 40 %, vector instructions 43 % of a unit's busy
// time, and with 3.1 workgroups a unit its last ones run alone (units are busy
// 80 % of the launch).  Measured (bf16, 8 d + 4 dv operations a pair): 4 x 3136
// tokens, 8 heads of 64 / 128 477 to 521 us, 620 to 680 TFLOP/s.
template <typename T, int D, int DV, bool WIDE, int DO>
__device__ __forceinline__ void key_side(const AttnArgs& a, const AttnPlace& place, int map) {
    using Shape = KeySideShape<T, D, DV, DO>;
    constexpr int kRows = Shape::kRows;
    constexpr bool ONE = DO == kOneMap, DK = DO != kValues, DVAL = DO != kOneMap;
    constexpr bool M2 = !ONE, DK2 = DK && M2;     // (with one map, that takes the first one's place)
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = place.place, hkv = place.head % a.hk, b = place.head / a.hk, split = place.part % a.key_splits;
    const int group = a.hq / a.hk;
    const int length = attn_length(a, b), offset = length - a.sq;
    const int first = tile * kKeySideKeys, wave_first = first + wave * 32, key = wave_first + (lane & 31);
    const bool exists = key < length;
    // this lane's key is visible to rows from `from` on, `seen` of them
    const int from = !exists ? a.sq : (a.causal ? max(0, key - offset) : 0), seen = max(0, a.sq - from);
    // every row from here on sees all of the wave's keys
    const int all_from = wave_first + 31 >= length ? 0x7fffffff : (a.causal ? wave_first + 31 - offset : 0);

    constexpr bool kKeysInLds = Shape::kKeysInLds;
    const unsigned base = unsigned(reinterpret_cast<uintptr_t>(lds));
    Operand<T> k1[kKeysInLds ? 1 : D / 16], k2[kKeysInLds || !M2 ? 1 : D / 16], v[DK ? DV / 16 : 1];
    unsigned key1 = 0;      // LDS address of this lane's key
    {
        if constexpr (kKeysInLds) {
            const unsigned tile1 = base + 2 * Shape::kBufferBytes;
            const RowCopy<T, D, kKeySideKeys, 256, WIDE> key_copy(a.kt, a.d, tid);
            const T* p = static_cast<const T*>(a.k) + b * a.kb + (long long)first * a.kt + hkv * a.kh + map * a.km;
            key_copy.start(tile1, p, a.kt, length - first, tid);
            if constexpr (M2) key_copy.start(tile1 + Shape::kKeyBytes, p + a.km, a.kt, length - first, tid);
            key1 = tile1 + row_lane<T, D>(lane) + wave * TileShape<T, D>::bytes(32);
        } else {
            const T* p = static_cast<const T*>(a.k) + b * a.kb + (long long)key * a.kt + hkv * a.kh + map * a.km;
            load_row_operands<T, D, WIDE>(k1, p, a.d, exists, lane);
            if constexpr (M2) load_row_operands<T, D, WIDE>(k2, p + a.km, a.d, exists, lane);
        }
        if constexpr (DK)
            load_row_operands<T, DV, WIDE>(v, static_cast<const T*>(a.v) + b * a.vb + (long long)key * a.vt + hkv * a.vh,
                                     a.dv, exists, lane);
    }
    if constexpr (!kKeysInLds) settle(k1);
    if constexpr (!kKeysInLds && M2) settle(k2);
    if constexpr (DK) settle(v);
    floatx16 dk1[DK ? D / 32 : 1], dk2[DK2 ? D / 32 : 1], dval[DVAL ? DV / 32 : 1];
#pragma unroll
    for (auto& x : dk1) x = zero16();
#pragma unroll
    for (auto& x : dk2) x = zero16();
#pragma unroll
    for (auto& x : dval) x = zero16();

    // The steps start at the first row that sees any of the workgroup's keys: rows
    // that see no key are not read, whatever they hold.
    const int first_row = !a.causal ? 0 : max(0, first - offset);
    const int per_head = first >= length ? 0 : max(0, a.sq - first_row + kRows - 1) / kRows;
    // this workgroup's share of the steps
    const long long steps = (long long)per_head * group;
    const int begin = int(steps * split / a.key_splits), end = int(steps * (split + 1) / a.key_splits);

    using QueryCopy = RowCopy<T, D, kRows, 256, WIDE>;
    using GradCopy = RowCopy<T, DV, kRows, 256, WIDE>;
    const QueryCopy query_copy(a.qt, a.d, tid);
    const GradCopy grad_copy(a.gt, a.dv, tid);
    const unsigned query_row = row_lane<T, D>(lane), query_column = column_lane<T, D>(lane);
    const unsigned grad_row = row_lane<T, DV>(lane) + Shape::kQueries;
    const unsigned grad_column = column_lane<T, DV>(lane) + Shape::kQueries;
    // A wave copies lse of both maps or delta of both: 2 x 32 values (and two
    // waves copy the same).
    const float* const stat = wave & 1 ? a.delta : a.lse;
    const unsigned stat_off = unsigned((lane & 31) + hi * a.sq) * 4;
    auto fetch = [&](int h, int row0, unsigned buffer) {
        const int left = a.sq - row0;
        const T* q = static_cast<const T*>(a.q) + b * a.qb + (long long)row0 * a.qt + h * a.qh + map * a.qm;
        query_copy.start(buffer, q, a.qt, left, tid);
        if constexpr (M2) query_copy.start(buffer + Shape::kQueryBytes, q + a.qm, a.qt, left, tid);
        grad_copy.start(buffer + Shape::kQueries,
                        static_cast<const T*>(a.dout) + b * a.gb + (long long)row0 * a.gt + h * a.gh, a.gt, left, tid);
        // (Rows beyond the last have zero log sums and delta.)
        copy4(copy_source(stat + (size_t(b) * a.hq + h) * 2 * a.sq + row0, unsigned(2 * a.sq - row0) * 4),
              (lane & 31) < left ? stat_off : kOutOfRange,
              __builtin_amdgcn_readfirstlane(buffer + Shape::kQueries + Shape::kGradBytes + (wave & 1) * 2 * kRows * 4));
    };
    // the rows of this step
    int h = hkv * group + (begin < end ? begin / per_head : 0);
    int row0 = first_row + (begin < end ? begin % per_head : 0) * kRows;
    if (begin < end) fetch(h, row0, base);
    for (int step = begin; step < end; ++step) {
        const unsigned buffer = base + ((step - begin) & 1) * Shape::kBufferBytes;
        const unsigned r1 = buffer + query_row, c1 = buffer + query_column;
        const unsigned r2 = r1 + Shape::kQueryBytes, c2 = c1 + Shape::kQueryBytes;
        const unsigned rg = buffer + grad_row, cg = buffer + grad_column;
        const float* ts = reinterpret_cast<const float*>(lds + (buffer - base) + Shape::kQueries + Shape::kGradBytes);
        const float lam = uniform_load(a.lam32 + h), turn = map ? -lam : 1.f;
        const int block_row0 = row0;
        row0 += kRows;
        if (row0 >= a.sq) {
            row0 = first_row;
            ++h;
        }
        // this stage is there, and all waves are done with the other buffer
        copies_done();
        if (step + 1 < end) fetch(h, row0, base + ((step + 1 - begin) & 1) * Shape::kBufferBytes);
        floatx16 p1 = zero16(), p2 = zero16();
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            mma(p1, read_row<T, D>(r1, 0, s), kKeysInLds ? read_row<T, D>(key1, 0, s) : k1[kKeysInLds ? 0 : s]);
            if constexpr (M2)
                mma(p2, read_row<T, D>(r2, 0, s),
                    kKeysInLds ? read_row<T, D>(key1 + Shape::kKeyBytes, 0, s) : k2[kKeysInLds ? 0 : s]);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 l1 = rows_of(ts + map * kRows, g, hi), l2 = rows_of(ts + kRows, g, hi);
            const float m1[4] = {l1.x, l1.y, l1.z, l1.w}, m2[4] = {l2.x, l2.y, l2.z, l2.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p1[4 * g + j] = exp2_fast(fmaf(p1[4 * g + j], a.scale_log2, -m1[j]));
                if constexpr (M2) p2[4 * g + j] = exp2_fast(fmaf(p2[4 * g + j], a.scale_log2, -m2[j]));
            }
        }
        // rows that do not see the key, and rows beyond the last
        if (block_row0 < all_from || block_row0 + kRows > a.sq) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const bool hidden = unsigned(block_row0 + acc_row(r, hi) - from) >= unsigned(seen);
                p1[r] = hidden ? 0.f : p1[r];
                p2[r] = hidden ? 0.f : p2[r];
            }
        }
        // The products after the scores: dv (columns of dO), t (rows of dO) and dk
        // (columns of q); their operands from LDS are read kAhead before they are used.
        constexpr int N = DV / 16, kAhead = kOperandsAhead<D>;
        constexpr int kT = DVAL ? N : 0, kK = kT + (DK ? N : 0), kEnd = kK + (DK ? (M2 ? N : N / 2) : 0);
        Operand<T> ring[kAhead + 1];
        auto read = [&](int i) {
            if (i >= kEnd) return;
            Operand<T>& o = ring[i % (kAhead + 1)];
            if (i < kT) {
                o = read_column<T, DV>(cg, 0, 32 * (i % (DV / 32)), i / (DV / 32));
            } else if (i < kK) {
                o = read_row<T, DV>(rg, 0, i - kT);
            } else {
                const int e = M2 ? (i - kK) % 2 : 0, x = M2 ? (i - kK) / 2 : i - kK;
                o = read_column<T, D>(e ? c2 : c1, 0, 32 * (x % (D / 32)), x / (D / 32));
            }
        };
        floatx16 t = zero16();
        Operand<T> w[2], s1[2], s2[2];
        if constexpr (DVAL) {
            floatx16 difference;
#pragma unroll
            for (int r = 0; r < 16; ++r) difference[r] = fmaf(-lam, p2[r], p1[r]);
            w[0] = acc_operand<T>(difference, 0);
            w[1] = acc_operand<T>(difference, 1);
        }
        in_order();
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
        for (int i = 0; i < kEnd; ++i) {
            in_order();
            read(i + kAhead);
            in_order();
            const Operand<T>& o = ring[i % (kAhead + 1)];
            if (DK && i == kK) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 u1 = rows_of(ts + (2 + map) * kRows, g, hi), u2 = rows_of(ts + 3 * kRows, g, hi);
                    const float d1[4] = {u1.x, u1.y, u1.z, u1.w}, d2[4] = {u2.x, u2.y, u2.z, u2.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        p1[4 * g + j] *= ONE ? fmaf(turn, t[4 * g + j], d1[j]) : t[4 * g + j] + d1[j];
                        if constexpr (M2) p2[4 * g + j] *= fmaf(-lam, t[4 * g + j], d2[j]);
                    }
                }
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    s1[s] = acc_operand<T>(p1, s);
                    s2[s] = acc_operand<T>(p2, s);
                }
            }
            if (i < kT) {
                mma(dval[DVAL ? i % (DV / 32) : 0], o, w[i / (DV / 32) % 2]);
            } else if (i < kK) {
                mma(t, o, v[DK ? i - kT : 0]);
            } else {
                const int e = M2 ? (i - kK) % 2 : 0, x = M2 ? (i - kK) / 2 : i - kK, d = x % (D / 32), s = x / (D / 32) % 2;
                if (e)
                    mma(dk2[DK2 ? d : 0], o, s2[s]);
                else
                    mma(dk1[DK ? d : 0], o, s1[s]);
            }
        }
    }
    if (key >= a.sk) return;
    if (!exists) {      // (a row that is not finite would leave zero times it)
#pragma unroll
        for (auto& x : dk1) x = zero16();
#pragma unroll
        for (auto& x : dk2) x = zero16();
#pragma unroll
        for (auto& x : dval) x = zero16();
    }
    const size_t at = (size_t(b) * a.sk + key) * a.hk + hkv;
    const bool whole = a.d % 4 == 0;
    if (a.key_splits > 1) {
        // [split][key][dk1, dk2, dv], unscaled
        float* part = a.key_part + (size_t(split) * a.n * a.sk * a.hk + at) * (2 * a.d + a.dv);
        if constexpr (DK) store_row(part + map * a.d, dk1, a.d, whole && a.o_wide, 1.f, hi);
        if constexpr (DK2) store_row(part + a.d, dk2, a.d, whole && a.o_wide, 1.f, hi);
        if constexpr (DVAL) store_row(part + 2 * a.d, dval, a.dv, whole && a.o_wide, 1.f, hi);
        return;
    }
    T* dk = static_cast<T*>(a.dk) + at * 2 * a.d;
    if constexpr (DK) store_row(dk + map * a.d, dk1, a.d, whole, a.scale, hi);
    if constexpr (DK2) store_row(dk + a.d, dk2, a.d, whole, a.scale, hi);
    if constexpr (DVAL) store_row(static_cast<T*>(a.dv_out) + at * a.dv, dval, a.dv, a.o_wide, 1.f, hi);
}

template <typename T, int D, int DV, bool WIDE>
__global__ __launch_bounds__(256, (KeySideShape<T, D, DV, kAll>::kBlocks)) void attn_key_side_kernel(AttnArgs a) {
    const AttnPlace place = attn_place(a, (a.sk + kKeySideKeys - 1) / kKeySideKeys, a.n * a.hk, a.key_splits * (kApart<D> ? 3 : 1));
    if constexpr (kApart<D>) {
        const int which = place.part / a.key_splits;
        if (which < 2)
            key_side<T, D, DV, WIDE, kOneMap>(a, place, which);
        else
            key_side<T, D, DV, WIDE, kValues>(a, place, 0);
    } else {
        key_side<T, D, DV, WIDE, kAll>(a, place, 0);
    }
}

namespace {
template <typename T, int D, int DV>
struct QuerySideShape {
    static constexpr int kKeys = 32;
    static constexpr int kMaps = kApart<D> ? 1 : 2;
    static constexpr int kKeyBytes = TileShape<T, D>::bytes(kKeys);
    static constexpr int kMapBytes = kMaps * kKeyBytes;
    static constexpr int kBufferBytes = kMapBytes + TileShape<T, DV>::bytes(kKeys);
    static constexpr int kBlocks = sizeof(T) * DV <= 256 || (sizeof(T) == 2 && kApart<D>) ? 2 : 1;
    static constexpr int kLds = 2 * kBufferBytes;
};
}  // namespace

// Query side: one workgroup takes 128 query rows of one head, 32 a wave, and
// goes over the keys, as the forward kernel does; q1, q2 and dO are operands, dq1
// and dq2 accumulators in registers.  Bound as the key side is (matrix
// instructions 45 %, vector instructions 57 % of busy time).  Measured (bf16,
// 8 d + 2 dv operations a pair): 4 x 3136 tokens, 8 heads of 64 / 128 328 to 361
// us, 670 to 740 TFLOP/s (with 64 rows a workgroup 371 us, not 352).
template <typename T, int D, int DV, bool WIDE>
__global__ __launch_bounds__(256, (QuerySideShape<T, D, DV>::kBlocks)) void attn_query_side_kernel(AttnArgs a) {
    using Shape = QuerySideShape<T, D, DV>;
    constexpr int kKeys = Shape::kKeys;
    constexpr bool ONE = kApart<D>, M2 = !ONE;      // (with one map, that takes the first one's place)
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tiles = (a.sq + kAttnRows - 1) / kAttnRows;
    const AttnPlace place = attn_place(a, tiles, a.n * a.hq, a.query_splits * (ONE ? 2 : 1));
    const int tile = tiles - 1 - place.place, h = place.head % a.hq, b = place.head / a.hq;
    const int split = place.part % a.query_splits, map = place.part / a.query_splits;
    const int hkv = h / (a.hq / a.hk);
    const int length = attn_length(a, b);
    const int first = tile * kAttnRows + wave * 32, row = first + (lane & 31);
    const int last = attn_last_key(a, row, length);
    const int first_last = attn_last_key(a, first, length);
    const int wave_end = attn_last_key(a, min(first + 31, a.sq - 1), length) + 1;
    const int seen = attn_last_key(a, min(tile * kAttnRows + kAttnRows, a.sq) - 1, length) + 1;
    // this workgroup's share of the stages
    const long long stages = (seen + kKeys - 1) / kKeys;
    const int begin = int(stages * split / a.query_splits) * kKeys;
    const int end = min(seen, int(stages * (split + 1) / a.query_splits) * kKeys);
    const float lam = attn_lambda(a, h);

    const T* kp = static_cast<const T*>(a.k) + b * a.kb + hkv * a.kh + map * a.km;
    const T* vp = static_cast<const T*>(a.v) + b * a.vb + hkv * a.vh;
    const bool valid = row < a.sq;
    Operand<T> q1[D / 16], q2[M2 ? D / 16 : 1], g[DV / 16];
    {
        const T* q = static_cast<const T*>(a.q) + b * a.qb + (long long)row * a.qt + h * a.qh + map * a.qm;
        load_row_operands<T, D, WIDE>(q1, q, a.d, valid, lane);
        if constexpr (M2) load_row_operands<T, D, WIDE>(q2, q + a.qm, a.d, valid, lane);
        load_row_operands<T, DV, WIDE>(g, static_cast<const T*>(a.dout) + b * a.gb + (long long)row * a.gt + h * a.gh, a.dv,
                                 valid, lane);
    }
    const size_t at = ((size_t(b) * a.hq + h) * 2 + map) * a.sq + row;
    float lse1 = valid ? a.lse[at] : kInf, lse2 = valid && M2 ? a.lse[at + a.sq] : kInf;
    float d1 = valid ? a.delta[at] : 0.f, d2 = valid && M2 ? a.delta[at + a.sq] : 0.f;
    const float turn = map ? -lam : 1.f;
    asm volatile("" : "+v"(lse1), "+v"(lse2), "+v"(d1), "+v"(d2));
    settle(q1);
    if constexpr (M2) settle(q2);
    settle(g);
    floatx16 dq1[D / 32], dq2[M2 ? D / 32 : 1];
#pragma unroll
    for (auto& x : dq1) x = zero16();
#pragma unroll
    for (auto& x : dq2) x = zero16();

    using KeyCopy = RowCopy<T, D, kKeys, 256, WIDE>;
    using ValueCopy = RowCopy<T, DV, kKeys, 256, WIDE>;
    const KeyCopy key_copy(a.kt, a.d, tid);
    const ValueCopy value_copy(a.vt, a.dv, tid);
    const unsigned base = unsigned(reinterpret_cast<uintptr_t>(lds));
    const unsigned key_row = row_lane<T, D>(lane), key_column = column_lane<T, D>(lane);
    const unsigned value_row = row_lane<T, DV>(lane) + Shape::kMapBytes;
    auto fetch = [&](int key, unsigned buffer) {
        const int left = end - key;
        const T* k = kp + (long long)key * a.kt;
        key_copy.start(buffer, k, a.kt, left, tid);
        if constexpr (M2) key_copy.start(buffer + Shape::kKeyBytes, k + a.km, a.kt, left, tid);
        value_copy.start(buffer + Shape::kMapBytes, vp + (long long)key * a.vt, a.vt, left, tid);
    };
    if (begin < end) fetch(begin, base);
    // of bf16 terms over the keys, or fp32 rows' D2 (once)
    float lam_sum = 0.f;
    if constexpr (sizeof(T) == 4)
        if (valid && hi == 0 && split == 0) lam_sum = a.second[(size_t(b) * a.hq + h) * a.sq + row];
    asm volatile("" : "+v"(lam_sum));
    for (int i = 0, key = begin; key < end; ++i, key += kKeys) {
        const unsigned buffer = base + (i & 1) * Shape::kBufferBytes;
        const unsigned r1 = buffer + key_row, c1 = buffer + key_column;
        const unsigned r2 = r1 + Shape::kKeyBytes, c2 = c1 + Shape::kKeyBytes, rv = buffer + value_row;
        copies_done();
        if (key + kKeys < end) fetch(key + kKeys, base + ((i + 1) & 1) * Shape::kBufferBytes);
        if (key >= wave_end) continue;
        // The products: scores (rows of k1, k2), t (rows of v), then dq (columns of
        // k1, k2), with operands read kAhead before they are used, as on the key side.
        constexpr int kMaps = Shape::kMaps, kT = kMaps * (D / 16), kQ = kT + DV / 16, kEnd = kQ + kMaps * (D / 16), kAhead = kOperandsAhead<D>;
        Operand<T> ring[kAhead + 1];
        auto read = [&](int i) {
            if (i >= kEnd) return;
            Operand<T>& o = ring[i % (kAhead + 1)];
            if (i < kT) {
                o = read_row<T, D>(i % kMaps ? r2 : r1, 0, i / kMaps);
            } else if (i < kQ) {
                o = read_row<T, DV>(rv, 0, i - kT);
            } else {
                const int x = (i - kQ) / kMaps;
                o = read_column<T, D>((i - kQ) % kMaps ? c2 : c1, 0, 32 * (x % (D / 32)), x / (D / 32));
            }
        };
        floatx16 p1 = zero16(), p2 = zero16(), t = zero16();
        Operand<T> s1[2], s2[2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
        for (int i = 0; i < kEnd; ++i) {
            in_order();
            read(i + kAhead);
            in_order();
            const Operand<T>& o = ring[i % (kAhead + 1)];
            if (i == kQ) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    p1[r] = exp2_fast(fmaf(p1[r], a.scale_log2, -lse1));
                    if constexpr (M2) p2[r] = exp2_fast(fmaf(p2[r], a.scale_log2, -lse2));
                }
                if (key + 31 > first_last) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bool hidden = acc_row(r, hi) > last - key;
                        p1[r] = hidden ? 0.f : p1[r];
                        p2[r] = hidden ? 0.f : p2[r];
                    }
                }
                if constexpr (sizeof(T) == 2) {
                    // (a step's terms first, so that the long sum is of few)
                    float step_sum = 0.f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) step_sum = fmaf(ONE ? p1[r] : p2[r], t[r], step_sum);
                    lam_sum += step_sum;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    p1[r] *= ONE ? fmaf(turn, t[r], d1) : t[r] + d1;
                    if constexpr (M2) p2[r] *= fmaf(-lam, t[r], d2);
                }
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    s1[s] = acc_operand<T>(p1, s);
                    s2[s] = acc_operand<T>(p2, s);
                }
            }
            if (i < kT) {
                if (i % kMaps)
                    mma(p2, o, q2[M2 ? i / kMaps : 0]);
                else
                    mma(p1, o, q1[i / kMaps]);
            } else if (i < kQ) {
                mma(t, o, g[i - kT]);
            } else {
                const int x = (i - kQ) / kMaps, d = x % (D / 32), s = x / (D / 32) % 2;
                if ((i - kQ) % kMaps)
                    mma(dq2[M2 ? d : 0], o, s2[s]);
                else
                    mma(dq1[d], o, s1[s]);
            }
        }
    }
    if (last < 0) {      // a row that sees no key: no gradient, whatever q and dO hold
        lam_sum = 0.f;
#pragma unroll
        for (auto& x : dq1) x = zero16();
#pragma unroll
        for (auto& x : dq2) x = zero16();
    }
    if (!ONE || map) {
        // this workgroup's part of dlam, in a fixed order
#pragma unroll
        for (int m = 1; m < 64; m *= 2) lam_sum += __shfl_xor(lam_sum, m, 64);
        __syncthreads();
        float* sums = reinterpret_cast<float*>(lds);
        if (lane == 0) sums[wave] = lam_sum;
        __syncthreads();
        if (tid == 0)
            a.dlam_part[size_t(h) * a.parts + (size_t(b) * tiles + tile) * a.query_splits + split] =
                -(sums[0] + sums[1] + sums[2] + sums[3]);
    }
    if (!valid) return;
    const size_t out = ((size_t(b) * a.sq + row) * a.hq + h) * 2 * a.d;
    const bool whole = a.d % 4 == 0;
    // A part of the sum, unscaled, or the gradient.  (Rows of fp32, parts or not, take
    // one path: of two, the compiler makes code in which the scan for overwritten
    // store data in the tests takes a store's address registers for its data.)
    const bool shared = a.query_splits > 1;
    float* part = a.query_part + (shared ? size_t(split) * a.n * a.sq * a.hq * 2 * a.d + out : 0);
    const float scale = shared ? 1.f : a.scale;
    if (sizeof(T) == 4 || shared) {
        float* to = sizeof(T) == 4 && !shared ? static_cast<float*>(a.dq) + out : part;
        store_row(to + map * a.d, dq1, a.d, whole, scale, hi);
        if constexpr (M2) store_row(to + a.d, dq2, a.d, whole, scale, hi);
        return;
    }
    T* dq = static_cast<T*>(a.dq) + out;
    store_row(dq + map * a.d, dq1, a.d, whole, scale, hi);
    if constexpr (M2) store_row(dq + a.d, dq2, a.d, whole, scale, hi);
}

namespace {

// Sums of the parts of workgroups that shared their steps, in their order: rows
// of `width` values, of which the first `scaled` go to `a0` (times scale), the
// rest to `a1`, by `blocks` workgroups of which this is the one `block`.
template <typename T, int V>
__device__ void add_parts(const float* part, int splits, long long rows, int width, int scaled, float scale, T* a0, T* a1,
                          int block, int blocks) {
    const long long n = rows * (width / V);
    for (long long i = (long long)block * 256 + threadIdx.x; i < n; i += (long long)blocks * 256) {
        float t[V] = {};
        for (int s = 0; s < splits; ++s) {
            if constexpr (V == 4) {
                const float4 x = reinterpret_cast<const float4*>(part)[s * n + i];
                t[0] += x.x;
                t[1] += x.y;
                t[2] += x.z;
                t[3] += x.w;
            } else {
                t[0] += part[s * n + i];
            }
        }
        const int w = width / V;
        const long long row = n < 0x7fffffff ? unsigned(i) / unsigned(w) : i / w;
        const int col = int(i - row * w) * V;
        const long long at = col < scaled ? row * scaled + col : row * (width - scaled) + col - scaled;
        T* const to = col < scaled ? a0 : a1;
        const float f = col < scaled ? scale : 1.f;
        if constexpr (V == 4)
            store4(to + at, 0, 4, true, t[0] * f, t[1] * f, t[2] * f, t[3] * f);
        else
            to[at] = T(t[0] * f);
    }
}
template <typename T>
__device__ void add_parts(const float* part, int splits, long long rows, int width, int scaled, float scale, void* a0, void* a1,
                          int block, int blocks) {
    if (width % 4 == 0 && scaled % 4 == 0)
        add_parts<T, 4>(part, splits, rows, width, scaled, scale, static_cast<T*>(a0), static_cast<T*>(a1), block, blocks);
    else
        add_parts<T, 1>(part, splits, rows, width, scaled, scale, static_cast<T*>(a0), static_cast<T*>(a1), block, blocks);
}

}  // namespace

// What workgroups computed in parts: dlam, by one workgroup a head (or one for
// all heads together), then dk and dv, by `key_blocks`, and dq, by the others.
// Bound by memory, or in small calls by its latency: 13.3 us for the 65 MB of 2 x
// 1999 x 4 keys in two parts (4.9 TB/s), 5 us for dlam alone.
template <typename T>
__global__ __launch_bounds__(256) void attn_finish_kernel(AttnArgs a, int key_blocks, int query_blocks) {
    const int lams = a.lam_step ? a.hq : 1, block = int(blockIdx.x) - lams;
    if (block >= key_blocks) {
        add_parts<T>(a.query_part, a.query_splits, (long long)a.n * a.sq * a.hq, 2 * a.d, 2 * a.d, a.scale, a.dq, nullptr,
                     block - key_blocks, query_blocks);
        return;
    }
    if (block >= 0) {
        add_parts<T>(a.key_part, a.key_splits, (long long)a.n * a.sk * a.hk, 2 * a.d + a.dv, 2 * a.d, a.scale, a.dk, a.dv_out,
                     block, key_blocks);
        return;
    }
    __shared__ float sums[256];
    const int heads = a.lam_step ? 1 : a.hq;
    const float* part = a.dlam_part + size_t(blockIdx.x) * a.parts;
    float t = 0.f;
    for (long long i = threadIdx.x; i < (long long)heads * a.parts; i += 256) t += part[i];
    sums[threadIdx.x] = t;
    __syncthreads();
    for (int m = 128; m > 0; m /= 2) {
        if (int(threadIdx.x) < m) sums[threadIdx.x] += sums[threadIdx.x + m];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        if (a.lam_f32)
            static_cast<float*>(a.dlam)[blockIdx.x] = sums[0];
        else
            static_cast<__bf16*>(a.dlam)[blockIdx.x] = __bf16(sums[0]);
    }
}

namespace {

template <typename T, int D, int DV>
hipError_t launch_key_side(const AttnArgs& a, hipStream_t s) {
    constexpr int kLds = kApart<D> ? std::max(KeySideShape<T, D, DV, kOneMap>::kLds, KeySideShape<T, D, DV, kValues>::kLds)
                                   : KeySideShape<T, D, DV, kAll>::kLds;
    const long long blocks =
        (long long)a.n * a.hk * a.key_splits * ((a.sk + kKeySideKeys - 1) / kKeySideKeys) * (kApart<D> ? 3 : 1);
    auto kernel = a.wide ? attn_key_side_kernel<T, D, DV, true> : attn_key_side_kernel<T, D, DV, false>;
    if (hipError_t e = allow_dynamic_lds(kernel, kLds)) return e;
    return launch_kernel(kernel, dim3(unsigned(blocks)), dim3(256), kLds, s, nullptr, nullptr, a);
}
template <typename T, int D, int DV>
hipError_t launch_query_side(const AttnArgs& a, hipStream_t s) {
    using Shape = QuerySideShape<T, D, DV>;
    const long long blocks =
        (long long)a.n * a.hq * a.query_splits * ((a.sq + kAttnRows - 1) / kAttnRows) * (kApart<D> ? 2 : 1);
    auto kernel = a.wide ? attn_query_side_kernel<T, D, DV, true> : attn_query_side_kernel<T, D, DV, false>;
    if (hipError_t e = allow_dynamic_lds(kernel, Shape::kLds)) return e;
    return launch_kernel(kernel, dim3(unsigned(blocks)), dim3(256), Shape::kLds, s, nullptr, nullptr, a);
}
template <typename T>
hipError_t launch_finish(const AttnArgs& a, hipStream_t s, hipEvent_t stop) {
    // (workgroups of 256 threads with 4 values each, as many as run at once)
    const auto blocks = [](int splits, double values) { return splits > 1 ? int(std::min(2048., values / 1024 + 1)) : 0; };
    const int key_blocks = blocks(a.key_splits, double(a.n) * a.sk * a.hk * (2 * a.d + a.dv));
    const int query_blocks = blocks(a.query_splits, double(a.n) * a.sq * a.hq * 2 * a.d);
    return launch_kernel(attn_finish_kernel<T>, dim3((a.lam_step ? a.hq : 1) + key_blocks + query_blocks), dim3(256), 0, s,
                         nullptr, stop, a, key_blocks, query_blocks);
}

template <typename T, int D, int DV>
hipError_t launch_shaped(const AttnArgs& a, hipStream_t s, const LaunchEvents& ev) {
    const int chunks = (a.sq + kAttnDeltaRows - 1) / kAttnDeltaRows;
    const long long rows = (long long)a.n * a.hq * chunks;
    if (hipError_t e = launch_kernel(attn_delta_kernel<T>, dim3(unsigned(rows)), dim3(256), 0, s, ev.start, nullptr, a))
        return e;
    if (hipError_t e = launch_key_side<T, D, DV>(a, s)) return e;
    if (hipError_t e = launch_query_side<T, D, DV>(a, s)) return e;
    return launch_finish<T>(a, s, ev.stop);
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

hipError_t launch_attn_backward(const fftsplit_attention_plan_s& p, const AttnArgs& a, hipStream_t s,
                                const LaunchEvents& ev) {
    return p.prob.dtype == FFTSPLIT_BF16 ? launch_typed<__bf16>(p, a, s, ev) : launch_typed<float>(p, a, s, ev);
}

}  // namespace fftsplit
