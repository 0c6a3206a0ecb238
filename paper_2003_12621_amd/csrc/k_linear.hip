// Linear attention with a decay for each head, in chunks of 32 tokens.
//
// With S the state (d x dv) before a chunk and D[i][j] = decay^(i - j) for
// j <= i, the chunk's outputs and the state behind it are
//     O = (Q K^T . D) V + diag(decay^(i+1)) Q S
//     S' = decay^32 S + (diag(decay^(31-j)) K)^T V,
// four matrix products.  A wave owns 32 columns of V, O and S; the state stays
// in its accumulators from chunk to chunk.  The scores are computed transposed
// (keys down, queries across the lanes), so that they are in place as the
// operand of the product with V; the state's accumulators are the operand of
// the product with Q as they stand.
//
// The gradients are the same sums with other roles: dq that of (dO, v, k), and
// dk and dv those of (v, dO, q) and (k, q, dO) from the last token to the first.
//
// Sequences with too few heads to fill the chip are cut into segments: a kernel
// that only adds up each segment's own state, one that joins them to the state
// before each, and then all segments side by side.
#include "linear_common.hpp"

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

// An operand's elements times factors.  The state is a sum over all tokens and
// an output in fp32, so bf16 elements are kept as two numbers (rounded, and what
// that left out), together good to 2^-18; fp32 ones as one.
template <typename T>
struct Weighted {
    static constexpr int kParts = sizeof(T) == 2 ? 2 : 1;
    Operand<T> part[kParts];
    __device__ __forceinline__ Weighted(const Operand<T>& x, const float* w) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 8; ++e) part[0].v[e] = x.v[e] * w[e];
        } else {
            u32x4 whole, rest;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = float(x.v[2 * e]) * w[2 * e], b = float(x.v[2 * e + 1]) * w[2 * e + 1];
                whole[e] = pack_bf16(a, b);
                rest[e] = pack_bf16(a - __uint_as_float(whole[e] << 16), b - __uint_as_float(whole[e] & 0xffff0000u));
            }
            part[0].v = __builtin_bit_cast(bf16x8, whole);
            part[1].v = __builtin_bit_cast(bf16x8, rest);
        }
    }
};

template <typename T, int D, int WAVES>
struct ScanShape {
    static constexpr int kThreads = 64 * WAVES;
    static constexpr int kColumns = 32 * WAVES;
    static constexpr int kRowBytes = TileShape<T, D>::bytes(kLinearChunk);          // a chunk of q or k
    static constexpr int kPairBytes = kRowBytes + TileShape<T, kColumns>::bytes(kLinearChunk);   // of k and v
    static constexpr int lds(bool main) { return 2 * (kPairBytes + (main ? kRowBytes : 0)); }
};

}  // namespace

// One workgroup: one segment of one head and 32 WAVES columns.  MAIN: the
// outputs; else only the state that the segment adds, from zero.
template <typename T, int D, int WAVES, bool WIDE, bool MAIN>
__global__ __launch_bounds__(64 * WAVES) void linear_scan_kernel(LinearScan a) {
    using Shape = ScanShape<T, D, WAVES>;
    constexpr int kChunk = kLinearChunk, DT = D / 32, kSteps = D / 16;
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, hi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int slices = (a.dv + Shape::kColumns - 1) / Shape::kColumns, q_heads = MAIN ? a.q_heads : 1;
    // (the columns and query heads of one segment next to one another)
    int id = xcd_logical_block(blockIdx.x, gridDim.x);
    const int slice = id % slices;
    id /= slices;
    const int member = id % q_heads;
    id /= q_heads;
    const int segments = MAIN ? a.segments : a.segments - 1;
    int segment = id % segments;
    const int head = id / segments, h = head % a.hk, b = head / a.hk;
    if (!MAIN && a.reverse) ++segment;               // the last one's own state is not needed
    const int length = linear_length(a.lengths, a.s, b);
    const int begin = segment * a.segment_tokens;
    const int room = int(min((long long)begin + a.segment_tokens, (long long)a.s)), end = min(room, length);
    const int chunks = end > begin ? (end - begin + kChunk - 1) / kChunk : 0;
    const float log2_decay = decay_log2(a.log_decay[h]);
    const int column0 = slice * Shape::kColumns, columns = min(a.dv - column0, Shape::kColumns);

    floatx16 state[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) state[d] = zero16();
    const int column = column0 + 32 * wave + (lane & 31);
    if (MAIN && a.init) {
        const float* p = a.init + head * a.init_head + segment * a.init_segment + column * a.init_column;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = 32 * d + state_row(r, hi);
                if (row < a.d && column < a.dv) state[d][r] = p[row * a.init_row];
            }
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) asm volatile("" : "+v"(state[d]));

    // factors of a pair (key acc_row(r, hi), query lane % 32) and of a token's
    // term of the state, in a chunk of n tokens
    float pair[16], update[16];
    int factors_of = 0;
    float inter = 0.f, carry = 0.f;
    const int query = lane & 31;
    auto set_factors = [&](int n) {
        factors_of = n;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int key = acc_row(r, hi), apart = a.reverse ? key - query : query - key;
            pair[r] = apart >= 0 && key < n ? a.pair_scale * decay_power(log2_decay, apart) : -1.f;
            const int left = a.reverse ? key + 1 : n - 1 - key;
            update[r] = key < n ? a.update_scale * decay_power(log2_decay, left) : 0.f;
        }
        inter = a.inter_scale * decay_power(log2_decay, max(a.reverse ? n - 1 - query : query + 1, 0));
        carry = decay_less_one(log2_decay, n);
    };

    using QueryCopy = RowCopy<T, D, kChunk, Shape::kThreads, WIDE>;
    using ValueCopy = RowCopy<T, Shape::kColumns, kChunk, Shape::kThreads, WIDE>;
    const QueryCopy query_copy(a.q.t, a.d, tid), key_copy(a.k.t, a.d, tid);
    const ValueCopy value_copy(a.v.t, columns, tid);
    const T* q = static_cast<const T*>(a.q.p) + b * a.q.b + (h * a.q_heads + member) * a.q.h;
    const T* k = static_cast<const T*>(a.k.p) + b * a.k.b + (long long)h * a.k_heads * a.k.h;
    const T* v = static_cast<const T*>(a.v.p) + b * a.v.b + (long long)h * a.k_heads * a.v.h + column0;
    const unsigned base = unsigned(reinterpret_cast<uintptr_t>(lds)), queries = base + 2 * Shape::kPairBytes;
    // Chunk and head of step i: the heads of k and v that share a state follow one
    // another within a chunk.
    auto fetch = [&](int chunk, int g, int step) {
        const int row = begin + (a.reverse ? chunks - 1 - chunk : chunk) * kChunk, rows = end - row;
        const unsigned to = base + (step & 1) * Shape::kPairBytes;
        key_copy.start(to, k + g * a.k.h + (long long)row * a.k.t, a.k.t, rows, tid);
        value_copy.start(to + Shape::kRowBytes, v + g * a.v.h + (long long)row * a.v.t, a.v.t, rows, tid);
        if (MAIN && g == 0)
            query_copy.start(queries + (chunk & 1) * Shape::kRowBytes, q + (long long)row * a.q.t, a.q.t, rows, tid);
    };
    const unsigned row_at = row_lane<T, D>(lane), key_column_at = state_column_lane<T, D>(lane);
    const unsigned value_at = column_lane<T, Shape::kColumns>(lane) + Shape::kRowBytes;
    const size_t o_row = size_t(a.hk) * a.q_heads * a.dv;
    T* o = MAIN ? static_cast<T*>(a.o) + size_t(b) * a.s * o_row + (size_t(h) * a.q_heads + member) * a.dv : nullptr;

    floatx16 out = zero16();
    if (chunks > 0) fetch(0, 0, 0);
    copies_done();
    for (int chunk = 0, g = 0, step = 0; chunk < chunks; ++step) {
        const bool last_head = g + 1 == a.k_heads;
        if (!last_head)
            fetch(chunk, g + 1, step + 1);
        else if (chunk + 1 < chunks)
            fetch(chunk + 1, 0, step + 1);
        const int row = begin + (a.reverse ? chunks - 1 - chunk : chunk) * kChunk, n = min(end - row, kChunk);
        if (n != factors_of) set_factors(n);
        const unsigned pairs = base + (step & 1) * Shape::kPairBytes;
        const unsigned tq = queries + (chunk & 1) * Shape::kRowBytes + row_at;
        if (MAIN && g == 0) {
            // what came before the chunk
            out = zero16();
#pragma unroll
            for (int s = 0; s < kSteps; ++s) mma(out, acc_operand<T>(state[s / 2], s % 2), read_row<T, D>(tq, 0, s));
#pragma unroll
            for (int r = 0; r < 16; ++r) out[r] *= inter;
        }
        if (g == 0) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) state[d][r] = fmaf(state[d][r], carry, state[d][r]);
        }
        Operand<T> x[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) x[s] = read_column<T, Shape::kColumns>(pairs + value_at, 0, 32 * wave, s);
        if (MAIN) {
            floatx16 c = zero16();
#pragma unroll
            for (int s = 0; s < kSteps; ++s) mma(c, read_row<T, D>(pairs + row_at, 0, s), read_row<T, D>(tq, 0, s));
#pragma unroll
            for (int r = 0; r < 16; ++r) c[r] = pair[r] < 0.f ? 0.f : c[r] * pair[r];
#pragma unroll
            for (int s = 0; s < 2; ++s) mma(out, x[s], acc_operand<T>(c, s));
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const Weighted<T> w(x[s], update + 8 * s);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const Operand<T> y = read_column<T, D>(pairs + key_column_at, 0, 32 * d, s);
#pragma unroll
                for (int p = 0; p < Weighted<T>::kParts; ++p) mma(state[d], y, w.part[p]);
            }
        }
        // the next stage is there, and all waves are done with this one
        copies_done();
        if (MAIN && last_head && query < n) {
            // (after the wait, so that it is not for these stores)
            T* p = o + size_t(row + query) * o_row;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                store4(p, column0 + 32 * wave + acc_row(4 * r, hi), a.dv, a.o_wide, out[4 * r], out[4 * r + 1], out[4 * r + 2],
                       out[4 * r + 3]);
        }
        g = last_head ? 0 : g + 1;
        chunk += last_head;
    }

    if (MAIN) {
        // tokens behind the last
        for (int row = max(end, begin) + tid / Shape::kColumns; row < room; row += Shape::kThreads / Shape::kColumns) {
            const int c = tid % Shape::kColumns;
            if (c < columns) o[size_t(row) * o_row + column0 + c] = T(0.f);
        }
    }
    float* to = MAIN ? a.last : a.parts;
    if (!to) return;
    if (MAIN) {
        if (member != 0 || segment != (a.reverse ? 0 : a.segments - 1)) return;
        to += size_t(head) * a.d * a.dv;
    } else {
        to += (size_t(head) * a.segments + segment) * a.d * a.dv;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = 32 * d + state_row(r, hi);
            if (row < a.d && column < a.dv) to[size_t(row) * a.dv + column] = state[d][r];
        }
}

// One thread an element: the state before each segment from what each adds.
__global__ __launch_bounds__(256) void linear_join_kernel(LinearJoin a) {
    const int blocks = (a.elements + 255) / 256;
    const int head = blockIdx.x / blocks, i = blockIdx.x % blocks * 256 + threadIdx.x;
    if (i >= a.elements) return;
    const int length = linear_length(a.lengths, a.s, head / a.hk);
    const float log2_decay = decay_log2(a.log_decay[head % a.hk]);
    float* p = a.parts + size_t(head) * a.segments * a.elements + i;
    float state = a.init ? a.init[size_t(head) * a.elements + i] : 0.f;
    constexpr int kAhead = 8;
    for (int m0 = 0; m0 < a.segments; m0 += kAhead) {
        float added[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int m = a.reverse ? a.segments - 1 - (m0 + j) : m0 + j;
            added[j] = m0 + j + 1 < a.segments ? p[size_t(m) * a.elements] : 0.f;   // (the last is not there)
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (m0 + j >= a.segments) break;
            const int m = a.reverse ? a.segments - 1 - (m0 + j) : m0 + j;
            p[size_t(m) * a.elements] = state;
            const int n = max(0, min(length - m * a.segment_tokens, a.segment_tokens));
            state = fmaf(state, decay_less_one(log2_decay, n), state) + added[j];
        }
    }
}

namespace {

template <typename T, int D, int WAVES, bool MAIN>
hipError_t launch_shaped(const LinearScan& a, hipStream_t s, const LaunchEvents& ev) {
    using Shape = ScanShape<T, D, WAVES>;
    const int slices = (a.dv + Shape::kColumns - 1) / Shape::kColumns;
    const long long blocks = (long long)a.n * a.hk * (MAIN ? (long long)a.q_heads * a.segments : a.segments - 1) * slices;
    auto kernel = a.wide ? linear_scan_kernel<T, D, WAVES, true, MAIN> : linear_scan_kernel<T, D, WAVES, false, MAIN>;
    if (hipError_t e = allow_dynamic_lds(kernel, Shape::lds(MAIN))) return e;
    return launch_kernel(kernel, dim3(unsigned(blocks)), dim3(Shape::kThreads), Shape::lds(MAIN), s, ev.start, ev.stop, a);
}

template <typename T, int D, bool MAIN>
hipError_t launch_columns(const LinearScan& a, hipStream_t s, const LaunchEvents& ev) {
    // (fp32 rows of 256: two buffers of 128 columns fill all of a compute unit's LDS)
    if (a.dv > 64 && sizeof(T) * D < 1024) return launch_shaped<T, D, 4, MAIN>(a, s, ev);
    return launch_shaped<T, D, 2, MAIN>(a, s, ev);
}

template <typename T, bool MAIN>
hipError_t launch_typed(const LinearScan& a, hipStream_t s, const LaunchEvents& ev) {
    if (a.d <= 32) return launch_columns<T, 32, MAIN>(a, s, ev);
    if (a.d <= 64) return launch_columns<T, 64, MAIN>(a, s, ev);
    if (a.d <= 128) return launch_columns<T, 128, MAIN>(a, s, ev);
    return launch_columns<T, 256, MAIN>(a, s, ev);
}

}  // namespace

hipError_t launch_linear_scan(const LinearScan& a, int dtype, hipStream_t s, const LaunchEvents& ev) {
    return dtype == FFTSPLIT_BF16 ? launch_typed<__bf16, true>(a, s, ev) : launch_typed<float, true>(a, s, ev);
}

hipError_t launch_linear_parts(const LinearScan& a, int dtype, hipStream_t s, const LaunchEvents& ev) {
    return dtype == FFTSPLIT_BF16 ? launch_typed<__bf16, false>(a, s, ev) : launch_typed<float, false>(a, s, ev);
}

hipError_t launch_linear_join(const LinearJoin& a, hipStream_t s, const LaunchEvents& ev) {
    const long long blocks = (long long)a.heads * ((a.elements + 255) / 256);
    return launch_kernel(linear_join_kernel, dim3(unsigned(blocks)), dim3(256), 0, s, ev.start, ev.stop, a);
}

}  // namespace fftsplit
