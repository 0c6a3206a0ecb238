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

// An LDS tile: rows of W elements in 16-byte chunks, without padding (copies
// from memory fill 1024 consecutive bytes a wave).  Chunk c of row r lies in
// place c ^ swizzle(r) of its row, so that 16 lanes that read one chunk of 16
// rows, or 32 lanes that read 4 neighbouring chunks of 4 consecutive rows, use
// all 64 banks alike: of the rows that start in the same bank, all of 16
// consecutive rows differ in the swizzle, and those of 4 by multiples of 4.
template <typename T, int W>
struct TileShape {
    static constexpr int kChunk = 16 / sizeof(T);          // elements
    static constexpr int kRowChunks = W / kChunk;
    static constexpr int bytes(int rows) { return rows * W * int(sizeof(T)); }
    static __device__ __forceinline__ int swizzle(int row) {
        if constexpr (kRowChunks == 4) return (row >> 2) & 3;
        if constexpr (kRowChunks == 8) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
        return (row & 3) << 2 | ((row >> 2) & 3);
    }
    static __device__ __forceinline__ unsigned at(int row, int chunk) {
        return unsigned(row * kRowChunks + (chunk ^ swizzle(row))) * 16;
    }
};

// LDS is addressed by byte offset.  Tiles start at multiples of 1024, so what a
// step changes of a lane's address is an exclusive or with a constant (its
// chunk) and a constant distance (its row): one register a lane and tile, from
// the two functions below, serves all of a tile's reads.
typedef __attribute__((address_space(3))) const char* LdsBytes;
template <typename V>
__device__ __forceinline__ V lds_at(unsigned address, int distance) {
    return *reinterpret_cast<__attribute__((address_space(3))) const V*>(LdsBytes(address) + distance);
}
// A lane's part of the address of read_row ...
template <typename T, int W>
__device__ __forceinline__ unsigned row_lane(int lane) {
    return TileShape<T, W>::at(lane & 31, 8 * (lane >> 5) / TileShape<T, W>::kChunk);
}
// ... and of read_column.
template <typename T, int W>
__device__ __forceinline__ unsigned column_lane(int lane) {
    using Shape = TileShape<T, W>;
    if constexpr (sizeof(T) == 4) return Shape::at(4 * (lane >> 5), (lane & 31) / 4) + (lane & 3) * 4;
    return Shape::at(4 * (lane >> 5) + ((lane >> 2) & 3), 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) + (lane & 1) * 8;
}

// Operand whose row (or column) lane % 32 is a row of the tile, contracted
// along the row: elements 16 s + 8 (lane / 32) + e of row row0 + lane % 32.
// `at`: the tile's address plus row_lane.  (row0 and col0 below are multiples
// of 32.)
template <typename T, int W>
__device__ __forceinline__ Operand<T> read_row(unsigned at, int row0, int s) {
    using Shape = TileShape<T, W>;
    const int distance = row0 * Shape::kRowChunks * 16;
    const unsigned chunk = 16 * s / Shape::kChunk;
    Operand<T> o;
    if constexpr (sizeof(T) == 4) {
        const floatx4 a = lds_at<floatx4>(at ^ (chunk * 16), distance), b = lds_at<floatx4>(at ^ ((chunk + 1) * 16), distance);
        o.v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
        o.v = lds_at<bf16x8>(at ^ (chunk * 16), distance);
    }
    return o;
}

// Operand whose row lane % 32 is column col0 + lane % 32 of the tile,
// contracted along the tile's rows in the order of an accumulator's registers:
// element e stands for row row0 + 16 s + 8 (e / 4) + 4 (lane / 32) + e % 4.
// `at`: the tile's address plus column_lane.
// bf16: a transposing read takes 4 rows of 16 columns per 16 lanes; lane i of
// the 16 gives the address of 4 columns of row i / 4 and gets column i.
template <typename T, int W>
__device__ __forceinline__ Operand<T> read_column(unsigned at, int row0, int col0, int s) {
    using Shape = TileShape<T, W>;
    constexpr int kRowBytes = Shape::kRowChunks * 16;
    constexpr unsigned kEight = 2;      // what 8 rows further changes of the swizzle
    const int distance = (row0 + 16 * s) * kRowBytes;
    at ^= unsigned(col0 / Shape::kChunk) * 16;
    Operand<T> o;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = e & 3, far = e >> 2;
            const unsigned turned = (Shape::kRowChunks == 8 ? 4 * (j >> 1) : 4 * j) ^ (far * kEight);
            o.v[e] = lds_at<float>(at ^ (turned * 16), distance + (8 * far + j) * kRowBytes);
        }
    } else {
        typedef __attribute__((address_space(3))) bf16x4* LdsQuad;
        const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsQuad)(LdsBytes(at) + distance));
        const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
            (LdsQuad)(LdsBytes(at ^ (kEight * 16)) + distance + 8 * kRowBytes));
        o.v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    return o;
}

// 16 bytes a lane from a buffer straight into LDS: lane l fills LDS bytes
// [lds + 16 l, lds + 16 l + 16), with zeros where its offset is out of range.
// Inline assembly because for the builtin the compiler waits for every
// outstanding load before each LDS read; copies_done waits before the barrier
// that publishes a tile.  The wait states cover a descriptor that a vector
// instruction wrote just before and the M0 write.
__device__ __forceinline__ void copy16(u32x4 rsrc, unsigned off, unsigned lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(rsrc), "s"(lds)
                 : "memory", "m0");
}
// The same of 4 bytes a lane.
__device__ __forceinline__ void copy4(u32x4 rsrc, unsigned off, unsigned lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(off), "s"(rsrc), "s"(lds)
                 : "memory", "m0");
}
__device__ __forceinline__ u32x4 copy_source(const void* base, unsigned bytes) {
    const uint64_t p = reinterpret_cast<uintptr_t>(base);
    u32x4 rsrc;
    rsrc[0] = __builtin_amdgcn_readfirstlane(unsigned(p));
    rsrc[1] = __builtin_amdgcn_readfirstlane(unsigned(p >> 32) & 0xffffu);
    rsrc[2] = __builtin_amdgcn_readfirstlane(bytes);
    rsrc[3] = 0x00020000u;
    return rsrc;
}
// The copies that all waves have started are complete.
__device__ __forceinline__ void copies_done() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// As above for a tile that only this wave copies and reads: all but the last
// LATER copies it has started are complete.
template <int LATER>
__device__ __forceinline__ void own_copies_done() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LATER) : "memory");
}
// This wave's reads of LDS are complete, so that it may copy over what they read.
__device__ __forceinline__ void own_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Copies rows from memory into a tile of ROWS rows of W elements, spread over
// THREADS threads: chunk place i of thread t is place t + i THREADS in row
// order.  Tiles are given by their LDS address.  Memory is read through a
// descriptor that ends with the last row that exists, so nothing beyond it is
// touched, and columns from `cols` on become zero.  What rows beyond the last
// hold is zero only where the stride is at least `cols`: where rows overlap, or are
// one and the same (stride 0), their offsets lie before that end, and the one row
// of a tensor may have any stride, so that they wrap round.  They then hold
// elements of rows that exist, and their terms have to be hidden.
// WIDE: base, stride and cols allow 16-byte accesses, and the copy goes straight
// into LDS; else elements pass through registers one by one.
template <typename T, int W, int ROWS, int THREADS, bool WIDE>
struct RowCopy {
    using Shape = TileShape<T, W>;
    static constexpr int kChunks = ROWS * Shape::kRowChunks;
    static constexpr int kPer = (kChunks + THREADS - 1) / THREADS;
    static constexpr bool kWhole = kChunks % THREADS == 0;
    // Memory operations of a wave in flight after start; of every wave, where all
    // have places.
    static constexpr int kCopies = WIDE ? kPer : 0;
    static_assert(kChunks % 64 == 0, "whole waves");

    // Byte offsets of a thread's chunks from the tile's first row in memory, the
    // same for all tiles of a tensor.
    unsigned off[kPer];
    int cols;

    __device__ __forceinline__ RowCopy(long long stride, int cols_, int t) : cols(cols_) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int row = (t + i * THREADS) / Shape::kRowChunks;
            const int col = ((t % Shape::kRowChunks) ^ Shape::swizzle(row)) * Shape::kChunk;
            off[i] = col < cols ? unsigned((row * stride + col) * int(sizeof(T))) : kOutOfRange;
        }
    }

    // Starts the copy of `rows` (possibly none or more than ROWS) rows from `base` on.
    // (t: the thread's place among the THREADS)
    __device__ __forceinline__ void start(unsigned tile, const T* base, long long stride, int rows, int t) const {
        const int n = min(rows, ROWS);
        const unsigned bytes = n > 0 ? unsigned(((n - 1) * stride + cols) * int(sizeof(T))) : 0u;
        const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
        if constexpr (WIDE) {
            const u32x4 rsrc = copy_source(base, bytes);
            const unsigned lds = tile + wave * 1024;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (kWhole || wave * 64 + i * THREADS < kChunks)
                    copy16(rsrc, off[i], __builtin_amdgcn_readfirstlane(lds + i * THREADS * 16));
        } else {
            const BufRsrc rsrc = make_rsrc(base, bytes);
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (!(kWhole || wave * 64 + i * THREADS < kChunks)) continue;
                const int row = (t + i * THREADS) / Shape::kRowChunks;
                const int col = ((t % Shape::kRowChunks) ^ Shape::swizzle(row)) * Shape::kChunk;
                T e[Shape::kChunk];
#pragma unroll
                for (int j = 0; j < Shape::kChunk; ++j) {
                    const unsigned o = col + j < cols ? off[i] + j * unsigned(sizeof(T)) : kOutOfRange;
                    if constexpr (sizeof(T) == 4)
                        e[j] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rsrc, o, 0, 0));
                    else
                        e[j] = __builtin_bit_cast(__bf16, __builtin_amdgcn_raw_buffer_load_b16(rsrc, o, 0, 0));
                }
                uint4 u;
                __builtin_memcpy(&u, e, 16);
                *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(
                    (__attribute__((address_space(3))) char*)(tile + (t + i * THREADS) * 16)) = __builtin_bit_cast(u32x4, u);
            }
        }
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

// Makes the compiler wait here for the memory that an operand comes from.  It
// does not know of the copies in flight, and a wait of its own inside a loop
// for an operand loaded before it would be one for all of them.
template <typename T, int N>
__device__ __forceinline__ void settle(Operand<T> (&o)[N]) {
#pragma unroll
    for (int s = 0; s < N; ++s) asm volatile("" : "+v"(o[s].v));
}

// No instruction is moved across this.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

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
