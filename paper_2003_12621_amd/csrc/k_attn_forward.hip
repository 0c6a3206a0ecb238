// Differential attention, forward: o = (softmax(q1 k1^T) - lam softmax(q2 k2^T)) v.
//
// Both maps are taken in one pass over the keys with a running maximum and sum
// each, and an output accumulator each: the two softmax denominators are known
// only at the end, where the accumulators are joined.  With values as wide as
// both maps together that costs what a second pass over the keys for the
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

// Scores of 32 keys become terms exp2(score - m); `acc` is rescaled where the
// reference maximum moves.  A row that has seen no key keeps m = -inf.
template <int DT>
__device__ __forceinline__ void softmax_step(floatx16& s, RowState& st, floatx16 (&acc)[DT], float scale_log2) {
    float top = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
    const float2 t2 = both_halves(top);
    top = fmaxf(t2.x, t2.y) * scale_log2;
    if (__ballot(top > st.m + kMaxSlack) != 0) {
        const float m = fmaxf(st.m, top);
        const float alpha = m == -kInf ? 1.f : exp2_fast(st.m - m);
        st.m = m;
        st.l *= alpha;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[d][r] *= alpha;
    }
    const float ref = st.m == -kInf ? 0.f : st.m;
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        s[r] = exp2_fast(fmaf(s[r], scale_log2, -ref));
        sum += s[r];
    }
    st.l += sum;
}

// Hides keys beyond `last` (of the lane's query) in a score tile of keys key0 ...
__device__ __forceinline__ void mask_scores(floatx16& s, int key0, int last, int hi) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
        if (key0 + acc_row(r, hi) > last) s[r] = -kInf;
}

template <typename T, int D, int DV>
struct ForwardShape {
    static constexpr int kKeys = D * sizeof(T) >= 128 * 2 ? 32 : 64;   // keys per stage
    static constexpr int kBlocks = D * sizeof(T) >= 128 * 2 ? 1 : 2;   // workgroups per compute unit aimed at
    static constexpr int kKeyBytes = TileShape<T, D>::bytes(kKeys);
    static constexpr int kBufferBytes = 2 * kKeyBytes + TileShape<T, DV>::bytes(kKeys);
    static constexpr int kLds = 2 * kBufferBytes;
};

// The joined output of the lane's query, and for a backward pass each map's own.
template <typename T, int DT>
__device__ __forceinline__ void store_output(const AttnArgs& a, const floatx16 (&o1)[DT], const floatx16 (&o2)[DT],
                                             float inv1, float inv2, float lam, size_t row, int hi) {
    T* out = static_cast<T*>(a.o) + row * a.dv;
    T* out1 = a.o1 ? static_cast<T*>(a.o1) + row * a.dv : nullptr;
    T* out2 = a.o1 ? static_cast<T*>(a.o2) + row * a.dv : nullptr;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int col = 32 * d + acc_row(4 * g, hi);
            float x[4], y[4], z[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                z[j] = o2[d][4 * g + j] * inv2;
                x[j] = o1[d][4 * g + j] * inv1;
                y[j] = x[j] - lam * z[j];
            }
            store4(out, col, a.dv, a.o_wide, y[0], y[1], y[2], y[3]);
            if (out1) {
                store4(out1, col, a.dv, a.o_wide, x[0], x[1], x[2], x[3]);
                store4(out2, col, a.dv, a.o_wide, z[0], z[1], z[2], z[3]);
            }
        }
}

}  // namespace

// One workgroup: 128 query rows of one head, 32 a wave; the keys pass through
// LDS in double-buffered stages that all four waves read.
template <typename T, int D, int DV>
__global__ __launch_bounds__(256, (ForwardShape<T, D, DV>::kBlocks)) void attn_forward_kernel(AttnArgs a) {
    using Shape = ForwardShape<T, D, DV>;
    constexpr int kKeys = Shape::kKeys, DT = DV / 32;
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, hi = lane >> 5;
    const int tiles = (a.sq + kAttnRows - 1) / kAttnRows;
    const int id = xcd_logical_block(blockIdx.x, gridDim.x);
    const int tile = tiles - 1 - id % tiles;           // under a causal mask the longest first
    const int h = id / tiles % a.hq, b = id / tiles / a.hq;
    const int hkv = h / (a.hq / a.hk);
    const int length = attn_length(a, b);

    const int first = tile * kAttnRows + wave * 32, row = first + (lane & 31);
    const int last = attn_last_key(a, row, length);                  // this lane's query
    const int first_last = attn_last_key(a, first, length);          // the wave's first and last query
    const int wave_end = attn_last_key(a, min(first + 31, a.sq - 1), length) + 1;
    const int end = attn_last_key(a, min(tile * kAttnRows + kAttnRows, a.sq) - 1, length) + 1;

    const T* k1 = static_cast<const T*>(a.k) + b * a.kb + hkv * a.kh;
    const T* v = static_cast<const T*>(a.v) + b * a.vb + hkv * a.vh;

    Operand<T> q1[D / 16], q2[D / 16];
    {
        const T* q = static_cast<const T*>(a.q) + b * a.qb + (long long)row * a.qt + h * a.qh;
        load_row_operands<T, D>(q1, q, a.d, row < a.sq, a.q_wide, lane);
        load_row_operands<T, D>(q2, q + a.qm, a.d, row < a.sq, a.q_wide, lane);
    }
    floatx16 o1[DT], o2[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o1[d] = o2[d] = zero16();
    RowState s1{-kInf, 0.f}, s2{-kInf, 0.f};

    Stage<T, D, kKeys, 256> g1, g2;
    Stage<T, DV, kKeys, 256> gv;
    auto fetch = [&](int key) {
        const int left = end - key;
        g1.load(RowBlock<T>{k1 + (long long)key * a.kt, a.kt, left, a.d, bool(a.k_wide)}, tid);
        g2.load(RowBlock<T>{k1 + a.km + (long long)key * a.kt, a.kt, left, a.d, bool(a.k_wide)}, tid);
        gv.load(RowBlock<T>{v + (long long)key * a.vt, a.vt, left, a.dv, bool(a.v_wide)}, tid);
    };
    auto buffer = [&](int i) { return lds + (i & 1) * Shape::kBufferBytes; };
    if (end > 0) fetch(0);
    for (int i = 0, key = 0; key < end; ++i, key += kKeys) {
        T* t1 = reinterpret_cast<T*>(buffer(i));
        T* t2 = reinterpret_cast<T*>(buffer(i) + Shape::kKeyBytes);
        T* tv = reinterpret_cast<T*>(buffer(i) + 2 * Shape::kKeyBytes);
        g1.store(t1, tid);
        g2.store(t2, tid);
        gv.store(tv, tid);
        // (the buffer's readers of two stages ago passed the last barrier)
        __syncthreads();
        if (key + kKeys < end) fetch(key + kKeys);
#pragma unroll
        for (int sub = 0; sub < kKeys; sub += 32) {
            const int key0 = key + sub;
            if (key0 >= wave_end) break;
            floatx16 c1 = zero16(), c2 = zero16();
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                mma(c1, read_row<T, D>(t1, sub, s, lane), q1[s]);
                mma(c2, read_row<T, D>(t2, sub, s, lane), q2[s]);
            }
            if (key0 + 31 > first_last) {
                mask_scores(c1, key0, last, hi);
                mask_scores(c2, key0, last, hi);
            }
            softmax_step(c1, s1, o1, a.scale_log2);
            softmax_step(c2, s2, o2, a.scale_log2);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const Operand<T> p1 = acc_operand<T>(c1, s), p2 = acc_operand<T>(c2, s);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const Operand<T> x = read_column<T, DV>(tv, sub, 32 * d, s, lane);
                    mma(o1[d], x, p1);
                    mma(o2[d], x, p2);
                }
            }
        }
    }

    const float2 h1 = both_halves(s1.l), h2 = both_halves(s2.l);
    const float l1 = h1.x + h1.y, l2 = h2.x + h2.y;
    if (row >= a.sq) return;
    // (m stays -inf where no key is visible: such a row is zero)
    const bool none = last < 0;
    store_output<T, DT>(a, o1, o2, none ? 0.f : 1.f / l1, none ? 0.f : 1.f / l2, attn_lambda(a, h),
                        (size_t(b) * a.sq + row) * a.hq + h, hi);
    if (a.lse && hi == 0) {
        float* lse = a.lse + (size_t(b) * a.hq + h) * 2 * a.sq + row;
        lse[0] = none ? 0.f : s1.m + log2f(l1);
        lse[a.sq] = none ? 0.f : s2.m + log2f(l2);
    }
}

namespace {
template <typename T, int D, int DV>
hipError_t launch_tiled(const AttnArgs& a, hipStream_t s, const LaunchEvents& ev) {
    using Shape = ForwardShape<T, D, DV>;
    const long long blocks = (long long)a.n * a.hq * ((a.sq + kAttnRows - 1) / kAttnRows);
    if (hipError_t e = allow_dynamic_lds(attn_forward_kernel<T, D, DV>, Shape::kLds)) return e;
    return launch_kernel(attn_forward_kernel<T, D, DV>, dim3(unsigned(blocks)), dim3(256), Shape::kLds, s, ev.start,
                         ev.stop, a);
}

template <typename T>
hipError_t launch_typed(const fftsplit_attention_plan_s& p, const AttnArgs& a, hipStream_t s, const LaunchEvents& ev) {
    switch (p.shape) {
        case 0: return launch_tiled<T, 32, 64>(a, s, ev);
        case 1: return launch_tiled<T, 64, 128>(a, s, ev);
        default: return launch_tiled<T, 128, 256>(a, s, ev);
    }
}
}  // namespace

hipError_t launch_attn_forward(const fftsplit_attention_plan_s& p, const AttnArgs& a, hipStream_t s,
                               const LaunchEvents& ev) {
    return p.prob.dtype == FFTSPLIT_BF16 ? launch_typed<__bf16>(p, a, s, ev) : launch_typed<float>(p, a, s, ev);
}

}  // namespace fftsplit
