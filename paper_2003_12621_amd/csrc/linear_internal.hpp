// Declarations shared by the linear attention entry points and kernels.
#pragma once

#include "fftsplit_internal.hpp"

struct fftsplit_linear_attention_plan_s {
    fftsplit_linear_attention_problem_t prob;
    int device;              // HIP ordinal, or -1 for an architecture-only plan
    float scale;
    int recurrent;           // the forward pass goes token by token
    // Tokens of a segment, within which pairs of tokens are taken one by one
    // and which only a state carries over, and how many make up a sequence.
    int segment_tokens, segments;
    size_t forward_ws, backward_ws;
};

namespace fftsplit {

// Widths of a head (rows of a state) the kernels are compiled for.
constexpr int kLinearMaxDim = 256;
// Tokens of a tile, and query rows of a workgroup (four waves' tiles).
constexpr int kLinearTile = 32, kLinearRows = 128;
// A tile's rows are addressed with 32-bit offsets from its first.
constexpr long long kLinearMaxTokenStride = 1 << 22;

// Tokens up to which the forward pass goes token by token, as where a state goes in and
// out: one launch in place of three.  Measured with states, token by token / by segments
// (us): 16 sequences of 16 heads (4) of 64 / 128 in bf16 1, 4, 8, 12 tokens 6 / 18, 9 / 18,
// 15 / 18, 20 / 18; 64 of 16 heads 8 and 12 tokens 25 / 64, 30 / 65; 16 of 8 heads of 128 / 256
// 15 / 43, 19 / 43; 16 of 8 heads (4) of 32 / 64 in fp32 9 / 20, 12 / 20.  (Without states one
// segment is faster from 4 tokens on in bf16, 6 us in place of 14 for 8 tokens of the first,
// and from 8 on in fp32, 7 in place of 9 of the last.)
constexpr int kLinearRecurrentTokens = 8;

// Rows [batch][token][head][width] of one tensor: strides in elements.
struct LinearRows {
    const void* p;
    long long b, t, h;
};

// One sum over the tokens, which the forward pass and each gradient are:
//   out_i = sum over the j up to i of decay^|i - j| pair_scale (q_i . k_j) v_j
//           + inter_scale q_i^T S,
//   S     = the state before i's segment, times decay to the distance.
// Forwards j is up to i from the segment's first token on; backwards from its
// last, and the state is one step of decay behind (it holds the gradient that the
// tokens behind the segment gave to the state after it).
struct LinearPass {
    LinearRows q, k, v;
    void* o;                         // [n][s][hk q_heads][dv], dense
    int q_heads, k_heads;            // of either, those that share a key head; one of them is 1
    int d, dv;                       // widths of q and k, and of v
    int reverse;
    float pair_scale, update_scale, inter_scale;
    const void* starts;              // operands of the states before the segments, or null: zero
    float* parts;                    // what each segment adds to the state: [n hk][segments][d][dv]
    const float* log_decay;
    const int* lengths;
    int n, s, hk, segments, segment_tokens;
    int first_part, part_count;      // the segments whose parts are needed
    int exact;                       // the caller gets the state, in fp32
    int wide, o_wide;
};

// The state before each segment from the parts, as the operand of the product
// with a tile of queries: [head][segment][column / 32][row / 16][part][lane][8], lane
// = 32 (row / 8 % 2) + column % 32, in the tensors' type, of which bf16 takes two
// parts; rows are those of the state, columns its columns, or (turned) the other way
// round.
struct LinearJoin {
    const float* parts;              // [heads][segments][d][dv]
    const float* init;               // [heads][d][dv] or null
    void* starts;                    // or null
    float* last;                     // [heads][d][dv]: the state behind the last segment, or null
    const float* log_decay;
    const int* lengths;
    int heads, hk, s, segments, segment_tokens, reverse;
    int d, dv, turned;
    int rows, columns;               // of the operands, rounded up to whole tiles
    int first_part, part_count;
};

struct LinearTokens {
    LinearRows q, k, v;
    void* o;                         // [n][s][hq][dv], dense
    const float* state;              // [n][hk][d][dv] or null
    float* state_out;                // likewise, possibly `state`
    const float* log_decay;
    const int* lengths;
    int n, s, hq, hk, d, dv;
    float scale;
    int state_wide;
};

// Widths that the kernels pad a pass's rows and a workgroup's columns to.
constexpr int linear_padded(int width) { return width <= 32 ? 32 : width <= 64 ? 64 : width <= 128 ? 128 : 256; }
constexpr int linear_columns(int width) { return width <= 64 ? 64 : 128; }

// Two passes of the same widths in one launch, or one (b null).
hipError_t launch_linear_pass(const LinearPass& a, const LinearPass* b, int dtype, hipStream_t s, const LaunchEvents& ev);
// The three passes of the gradients, of aligned tensors, in one launch.
hipError_t launch_linear_gradients(const LinearPass& dq, const LinearPass& dk, const LinearPass& dv, int dtype, hipStream_t s,
                                   const LaunchEvents& ev);
hipError_t launch_linear_parts(const LinearPass& a, const LinearPass* b, int dtype, hipStream_t s, const LaunchEvents& ev);
hipError_t launch_linear_join(const LinearJoin* jobs, int count, int dtype, hipStream_t s, const LaunchEvents& ev);
hipError_t launch_linear_tokens(const LinearTokens& a, int dtype, hipStream_t s, const LaunchEvents& ev);

}  // namespace fftsplit
