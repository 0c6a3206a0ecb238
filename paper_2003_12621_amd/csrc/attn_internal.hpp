// Declarations shared by the attention entry points and kernels.
#pragma once

#include "fftsplit_internal.hpp"

struct fftsplit_attention_plan_s {
    fftsplit_attention_problem_t prob;
    int device;              // HIP ordinal, or -1 for an architecture-only plan
    float scale;             // of the products, before the softmax
    int shape;               // index into kAttnShapes: the kernels' padded head widths
    int splits;              // workgroups that share the keys of one tile of few rows; 0: the tiled kernel runs
    // Workgroups that share the rows of a tile of keys, and the keys of a tile
    // of rows, in the backward pass (1: each goes over all).
    int key_splits, query_splits;
    size_t forward_ws, backward_ws;
};

namespace fftsplit {

// Head widths (of a map's queries and keys, of the values) the kernels are
// compiled for; a plan takes the first pair that holds its own.
struct AttnShape {
    int d, dv;
};
constexpr AttnShape kAttnShapes[] = {{32, 64}, {64, 128}, {128, 256}};
constexpr int kAttnShapeCount = 3;

// Query rows a workgroup of the forward kernel takes (two of 32, each by a wave
// for either map), and of the backward kernels (4 waves of 32).
constexpr int kAttnTiledRows = 64;
constexpr int kAttnRows = 128;
// Query rows, packed over the heads that share a key head, of the kernel for few rows.
constexpr int kAttnFewRows = 32;

// Tiles hold at most 128 rows of at most 4-byte elements: their byte offsets stay
// below 2^31.
constexpr long long kAttnMaxTokenStride = 1 << 22;

// What the attention kernels get.  Strides are in elements.
struct AttnArgs {
    const void *q, *k, *v, *lam;
    const int* lengths;              // keys of each sequence, or null: all sk
    int n, sq, sk, hq, hk, d, dv;
    int causal;
    float scale_log2;                // scale * log2(e)
    float scale;
    int lam_f32, lam_step;           // lam is fp32; 0 if one lam serves all heads
    long long qb, qt, qh, qm;        // batch, token, head, map
    long long kb, kt, kh, km;
    long long vb, vt, vh;
    int wide;                        // 16-byte accesses of all input rows allowed
    void* o;                         // [n][sq][hq][dv]
    float *o1, *o2;                  // the maps' own outputs, same layout, or null
    float* lse;                      // [n][hq][2][sq]: log2 of the sum of exp2, or null
    int o_wide;
    // few rows
    int splits;
    float* part;                     // [batch][key head][packed row][split][2][padded dv]
    float* part_stats;               // [batch][key head][packed row][split][4]: maximum and sum of both maps
    // backward
    const void* dout;
    long long gb, gt, gh;            // batch, token, head strides of dout
    float* delta;                    // [n][hq][2][sq]: - D1, lam D2
    float* second;                   // [n][hq][sq]: D2 (fp32)
    float* dlam_part;                // [hq][parts]
    float* lam32;                    // [hq]: lam in fp32
    int parts;
    int key_splits, query_splits;
    float* key_part;                 // [split][n][sk][hk][2 d + dv]
    float* query_part;               // [split][n][sq][hq][2][d]
    void *dq, *dk, *dv_out, *dlam;
};

hipError_t launch_attn_forward(const fftsplit_attention_plan_s& p, const AttnArgs& a, hipStream_t s,
                               const LaunchEvents& ev);
hipError_t launch_attn_backward(const fftsplit_attention_plan_s& p, const AttnArgs& a, hipStream_t s,
                                const LaunchEvents& ev);
// Rows of one head that a workgroup of the backward's first kernel reduces: two
// for each 16 lanes (four took 6.5 us, not 4.9, at 6 x 301 rows of 6 heads; one
// 15.7, not 14.3, at 4 x 3136 of 8).
constexpr int kAttnDeltaRows = 32;

}  // namespace fftsplit
