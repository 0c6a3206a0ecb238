// Declarations shared by the linear attention entry points and kernels.
#pragma once

#include "fftsplit_internal.hpp"

struct fftsplit_linear_attention_plan_s {
    fftsplit_linear_attention_problem_t prob;
    int device;              // HIP ordinal, or -1 for an architecture-only plan
    float scale;
    int recurrent;           // the forward pass goes token by token
    // Parts of a sequence that workgroups take side by side (1: each goes over
    // all of it), and their tokens, in the forward and in the backward pass.
    int segments[2], segment_tokens[2];
    size_t forward_ws, backward_ws;
};

namespace fftsplit {

// Widths of a head (rows of a state) the kernels are compiled for.
constexpr int kLinearMaxDim = 256;
// Tokens of a chunk: one 32 x 32 tile of scores.
constexpr int kLinearChunk = 32;
constexpr int kLinearMaxSegments = 64;
// A chunk's rows are addressed with 32-bit offsets from its first.
constexpr long long kLinearMaxTokenStride = 1 << 22;

// Tokens up to which the forward pass goes token by token.
constexpr int kLinearRecurrentTokens = 8;

// Rows [batch][token][head][width] of one tensor: strides in elements.
struct LinearRows {
    const void* p;
    long long b, t, h;
};

// One scan over the tokens, which the forward pass and each gradient are:
//   out_i = sum over the j up to i of decay^|i - j| pair_scale (q_i . k_j) v_j
//           + inter_scale q_i^T S,
//   S     = the state before i, of the terms update_scale k_j v_j^T.
// Forwards j is up to i from the first token on; backwards from the last, and
// the state is one step of decay behind (it holds the gradient that the tokens
// behind i gave to the state after i).
struct LinearScan {
    LinearRows q, k, v;
    void* o;                         // [n][s][hk q_heads][dv], dense
    int q_heads, k_heads;            // of either, those that share a key head; one of them is 1
    int d, dv;                       // widths of q and k, and of v
    int reverse;
    float pair_scale, update_scale, inter_scale;
    // State at the start of a segment, and after the last: of head g (over all
    // sequences) and segment m element (row, column) is
    //   g * head + m * segment + row * row_step + column * column_step.
    const float* init;               // or null: zero
    long long init_head, init_segment, init_row, init_column;
    float* last;                     // [n hk][d][dv], or null
    float* parts;                    // of the kernel that only computes states: [n hk][segments][d][dv]
    const float* log_decay;
    const int* lengths;
    int n, s, hk, segments, segment_tokens;
    int wide, o_wide;
};

// States at the start of the segments from what each segment adds.
struct LinearJoin {
    float* parts;                    // [heads][segments][elements], in place
    const float* init;               // [heads][elements] or null
    const float* log_decay;
    const int* lengths;
    int heads, hk, s, segments, segment_tokens, reverse;
    int elements;
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

hipError_t launch_linear_scan(const LinearScan& a, int dtype, hipStream_t s, const LaunchEvents& ev);
hipError_t launch_linear_parts(const LinearScan& a, int dtype, hipStream_t s, const LaunchEvents& ev);
hipError_t launch_linear_join(const LinearJoin& a, hipStream_t s, const LaunchEvents& ev);
hipError_t launch_linear_tokens(const LinearTokens& a, int dtype, hipStream_t s, const LaunchEvents& ev);

}  // namespace fftsplit
