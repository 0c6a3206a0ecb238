// Building blocks of the differential-attention kernels: matrix operands in
// registers, tiles in LDS, and the copies between memory and LDS.
//
// Every product is taken on 32x32 tiles in steps of 16 along the contracted
// axis.  A wave's operand of such a step is 8 elements a lane: row (of A) or
// column (of B) lane % 32, and the 8 elements that lane / 32 selects of the
// 16.  Which of the 16 a lane's element stands for does not matter as long as
// A and B agree, and the accumulator's layout
//     column lane % 32, row 8 (r / 4) + 4 (lane / 32) + r % 4 in register r
// makes one half-accumulator (r = 8 s .. 8 s + 7) the B operand of a later
// product over its rows as it stands, with no exchange between lanes.  So the
// kernels compute the transposed score tile where they go on with products
// over keys, and keep everything that belongs to one query (its maximum, sum
// and output scale) in the lane that holds its column.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_runtime.h>

#include "bf16_split.hpp"

namespace fftsplit {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float floatx8 __attribute__((ext_vector_type(8)));

constexpr float kInf = __builtin_inff();

// 8 elements a lane, and the product step.  The fp32 step is 8 instructions
// that each contract one element of either half of the lanes.
template <typename T>
struct Operand;
template <>
struct Operand<__bf16> {
    bf16x8 v;
};
template <>
struct Operand<float> {
    floatx8 v;
};

__device__ __forceinline__ void mma(floatx16& c, const Operand<__bf16>& a, const Operand<__bf16>& b) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ void mma(floatx16& c, const Operand<float>& a, const Operand<float>& b) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
}

__device__ __forceinline__ floatx16 zero16() {
    floatx16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
}

// Row of accumulator register r (lane half `hi`).
__device__ __forceinline__ int acc_row(int r, int hi) { return 8 * (r >> 2) + 4 * hi + (r & 3); }

// Half s of an accumulator as a B operand, rounded to T.
template <typename T>
__device__ __forceinline__ Operand<T> acc_operand(const floatx16& c, int s) {
    Operand<T> o;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o.v[e] = c[8 * s + e];
    } else {
        u32x4 p;
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = pack_bf16(c[8 * s + 2 * e], c[8 * s + 2 * e + 1]);
        o.v = __builtin_bit_cast(bf16x8, p);
    }
    return o;
}

// The value of the lane 32 further (modulo 64) next to a lane's own, in an
// order that is the same for both.
__device__ __forceinline__ float2 both_halves(float x) {
    const unsigned u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <typename T>
__device__ __forceinline__ float to_float(T x) {
    return float(x);
}

// An LDS tile of rows of W elements.  Rows are padded by 16 bytes (bf16) or
// 8 elements (fp32): reads of 16 bytes at one column of 16 rows then fall into
// different banks, and so do the column reads of read_column.
template <typename T, int W>
struct TileShape {
    static constexpr int kStride = W + 8;
    static constexpr int kChunk = 16 / sizeof(T);          // elements per 16 bytes
    static constexpr int kRowChunks = W / kChunk;
    static constexpr int bytes(int rows) { return rows * kStride * int(sizeof(T)); }
};

// Operand whose row (or column) lane % 32 is a row of the tile, contracted
// along the row: elements 16 s + 8 (lane / 32) + e of row row0 + lane % 32.
template <typename T, int W>
__device__ __forceinline__ Operand<T> read_row(const T* tile, int row0, int s, int lane) {
    const T* p = tile + (row0 + (lane & 31)) * TileShape<T, W>::kStride + 16 * s + 8 * (lane >> 5);
    Operand<T> o;
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
        o.v = floatx8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    } else {
        o.v = *reinterpret_cast<const bf16x8*>(p);
    }
    return o;
}

// Operand whose row lane % 32 is column col0 + lane % 32 of the tile,
// contracted along the tile's rows in the order of an accumulator's registers:
// element e stands for row row0 + 16 s + 8 (e / 4) + 4 (lane / 32) + e % 4.
// bf16: a transposing read takes 4 rows of 16 columns per 16 lanes; lane i of
// the 16 gives the address of 4 columns of row i / 4 and gets column i.
template <typename T, int W>
__device__ __forceinline__ Operand<T> read_column(const T* tile, int row0, int col0, int s, int lane) {
    constexpr int kStride = TileShape<T, W>::kStride;
    Operand<T> o;
    if constexpr (sizeof(T) == 4) {
        const T* p = tile + (row0 + 16 * s + 4 * (lane >> 5)) * kStride + col0 + (lane & 31);
#pragma unroll
        for (int e = 0; e < 8; ++e) o.v[e] = p[(8 * (e >> 2) + (e & 3)) * kStride];
    } else {
        const T* p = tile + (row0 + 16 * s + 4 * (lane >> 5) + ((lane >> 2) & 3)) * kStride + col0 +
                     16 * ((lane >> 4) & 1) + 4 * (lane & 3);
        typedef __attribute__((address_space(3))) bf16x4* LdsQuad;
        const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsQuad)(p));
        const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsQuad)(p + 8 * kStride));
        o.v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    return o;
}

// Rows in memory on their way to a tile of ROWS rows of W elements in LDS,
// spread over THREADS threads: chunk i of thread t is chunk t + i THREADS in row
// order.  Loads go through a buffer descriptor of the rows that exist, so rows
// beyond them read as zero and are not touched; so do columns from `cols` on.
// WIDE: base, stride and cols allow 16-byte accesses, else single elements.
template <typename T, int W, int ROWS, int THREADS, bool WIDE>
struct Stage {
    using Shape = TileShape<T, W>;
    static constexpr int kChunks = ROWS * Shape::kRowChunks;
    static constexpr int kPer = (kChunks + THREADS - 1) / THREADS;
    static constexpr bool kWhole = kChunks % THREADS == 0;
    uint4 r[kPer];

    // Byte offsets of a thread's chunks from the tile's first row, the same
    // for all tiles of a tensor.
    struct Map {
        unsigned off[kPer];
        int cols, col;
        __device__ __forceinline__ Map(long long stride, int cols_, int t) : cols(cols_) {
            col = t % Shape::kRowChunks * Shape::kChunk;    // (THREADS is a multiple of kRowChunks)
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int c = t + i * THREADS, row = c / Shape::kRowChunks;
                off[i] = (kWhole || c < kChunks) && col < cols ? unsigned((row * stride + col) * int(sizeof(T))) : kOutOfRange;
            }
        }
    };

    // `rows` (possibly none or more than ROWS) rows exist from `base` on.
    __device__ __forceinline__ void load(const Map& m, const T* base, long long stride, int rows) {
        const int n = min(rows, ROWS);
        const BufRsrc rsrc = make_rsrc(base, n > 0 ? unsigned(((n - 1) * stride + m.cols) * int(sizeof(T))) : 0u);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if constexpr (WIDE) {
                r[i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, m.off[i], 0, 0));
            } else {
                T e[Shape::kChunk];
#pragma unroll
                for (int j = 0; j < Shape::kChunk; ++j) {
                    const unsigned o = m.col + j < m.cols && m.off[i] != kOutOfRange ? m.off[i] + j * unsigned(sizeof(T))
                                                                                    : kOutOfRange;
                    if constexpr (sizeof(T) == 4)
                        e[j] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rsrc, o, 0, 0));
                    else
                        e[j] = __builtin_bit_cast(__bf16, __builtin_amdgcn_raw_buffer_load_b16(rsrc, o, 0, 0));
                }
                __builtin_memcpy(&r[i], e, 16);
            }
        }
    }
    __device__ __forceinline__ void store(T* tile, int t) const {
        T* p = tile + t / Shape::kRowChunks * Shape::kStride + t % Shape::kRowChunks * Shape::kChunk;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (kWhole || t + i * THREADS < kChunks)
                *reinterpret_cast<uint4*>(p + i * (THREADS / Shape::kRowChunks) * Shape::kStride) = r[i];
    }
};

// The operand steps of one row of `cols` elements that lane % 32 holds, from
// memory (p may be anything where `valid` is false).
template <typename T, int W, bool WIDE>
__device__ __forceinline__ void load_row_operands(Operand<T> (&o)[W / 16], const T* p, int cols, bool valid, int lane) {
#pragma unroll
    for (int s = 0; s < W / 16; ++s) {
        const int col = 16 * s + 8 * (lane >> 5);
        T e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = T(0.f);
        if (valid) {
            if constexpr (WIDE) {
#pragma unroll
                for (int j = 0; j < 8; j += 16 / int(sizeof(T)))
                    if (col + j < cols) *reinterpret_cast<uint4*>(e + j) = *reinterpret_cast<const uint4*>(p + col + j);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (col + j < cols) e[j] = p[col + j];
            }
        }
        __builtin_memcpy(&o[s].v, e, sizeof(e));
    }
}

// Four consecutive elements of an output row, elements from `cols` on left out
// (`wide`: cols is a multiple of 4).
template <typename T>
__device__ __forceinline__ void store4(T* p, int col, int cols, bool wide, float a, float b, float c, float d) {
    const float v[4] = {a, b, c, d};
    if (wide) {
        if (col >= cols) return;
        if constexpr (sizeof(T) == 4)
            *reinterpret_cast<float4*>(p + col) = make_float4(a, b, c, d);
        else
            *reinterpret_cast<uint2*>(p + col) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j < cols) p[col + j] = T(v[j]);
    }
}

}  // namespace fftsplit
