/*
 * fftsplit.h -- C ABI of the split-FFT 2-D convolution library for AMD
 * MI355X (gfx950).
 *
 * Method: Chitsaz et al., "Acceleration of Convolutional Neural Network Using
 * FFT-Based Split Convolutions" (arXiv:2003.12621), Section 3.1.  A stride-1
 * 'same' convolution layer (CNN cross-correlation, odd K x K kernel, K//2
 * zeros of padding) is computed by
 *   1. splitting each input plane into T x T patches (eq. 4),
 *   2. padding each patch to L x L, L = T + K - 1 (eqs. 5-6),
 *   3. a 2-D real FFT of every padded patch, and of every zero-padded filter
 *      (eq. 8, done once per layer by fftsplit_transform_weights),
 *   4. the entry-wise product of patch and filter spectra (eq. 9), summed
 *      over input channels: per frequency bin a Cin -> Cout complex matrix
 *      product batched over patches,
 *   5. an inverse FFT per (patch, output channel), crop and concatenation of
 *      the valid T x T tile (eq. 10 and the text after it) -- or, with
 *      FFTSPLIT_OVERLAP_ADD, zero-padded patches whose L x L results are
 *      overlap-added (the discipline of Section 2, Fig. 1, at tile size T),
 *   6. optional bias and ReLU, fused into the inverse stage.
 *
 * Result: y = relu?(conv2d(x, w, bias, stride=1, padding=K//2)) with
 * PyTorch's cross-correlation convention, in fp32.
 *
 * Conventions for every entry point:
 *   - Tensors are fp32 and densely packed (C order).  Pointers marked
 *     "device" are device addresses on the plan's device; "host" pointers
 *     are host memory.  Device buffers must be 16-byte aligned.
 *   - The caller owns every buffer.  The library never allocates device
 *     memory; a plan owns host memory only.
 *   - Work is enqueued asynchronously on the given stream (0 = the null
 *     stream).  The return status covers argument checks and launch errors;
 *     a fault inside a kernel surfaces at the caller's next synchronisation.
 *   - No C++ exception crosses this ABI.  On any status other than
 *     FFTSPLIT_SUCCESS, fftsplit_last_error() returns a message for the
 *     calling thread and nothing has been enqueued.
 *   - A plan is immutable after creation and may be used from several
 *     threads and streams at once, as long as each concurrent call has its
 *     own workspace and output.
 */
#ifndef FFTSPLIT_H
#define FFTSPLIT_H

#include <stddef.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct fftsplit_plan_s* fftsplit_plan_t;   /* opaque, host-side */

typedef enum {
    FFTSPLIT_SUCCESS = 0,
    FFTSPLIT_ERROR_INVALID_VALUE = 1,        /* bad dimension, NULL/misaligned pointer, aliasing */
    FFTSPLIT_ERROR_NOT_SUPPORTED = 2,        /* even K, stride != 1, pad != K/2, unsupported L */
    FFTSPLIT_ERROR_INSUFFICIENT_WORKSPACE = 3,
    FFTSPLIT_ERROR_DEVICE = 4,               /* a HIP runtime call or kernel launch failed */
    FFTSPLIT_ERROR_ARCH = 5                  /* the device is not gfx950 */
} fftsplit_status_t;

/* Problem flags. */
enum {
    FFTSPLIT_OVERLAP_SAVE = 0,   /* halo'd patches, crop + concatenate (Section 3.1); default */
    FFTSPLIT_OVERLAP_ADD  = 1,   /* zero-padded patches, overlap-add of the L x L results */
    FFTSPLIT_BIAS         = 2,   /* add bias[co] in the inverse stage */
    FFTSPLIT_RELU         = 4,   /* apply max(., 0) after the bias */
    FFTSPLIT_MAXPOOL      = 8    /* then a 2x2 stride-2 max-pool (floor): y is
                                  * [n][cout][h/2][w/2] (the VGG stage ends);
                                  * needs h, w >= 2 */
};

/* The layer, as the paper states the problem: batch n, channels cin -> cout,
 * an h x w input, a k x k filter, the patch (tile) size, stride 1 and zero
 * padding of k/2 (Section 2, eq. 1; Section 3.1). */
typedef struct {
    int n, cin, h, w, cout, k;
    int tile;        /* T; 0 lets the plan choose among L = 8, 16, 32.  With
                      * FFTSPLIT_OVERLAP_ADD, tile = k (k = 3, 5, 7) selects the
                      * OaAConv configuration the paper compares against
                      * (Section 2, Fig. 1): patches of the filter's size,
                      * L = 2k - 1 = 5, 9, 13 */
    int stride;      /* must be 1 */
    int pad;         /* must be k/2 ('same') */
    unsigned flags;  /* FFTSPLIT_* flags above */
} fftsplit_problem_t;

/* What a plan decided.  Spectra are complex64 (re, im float pairs).
 *
 * Frequency bins: the 2-D real transform S of an L x L patch has
 * L*(L/2+1) bins (k1 in [0,L), k2 in [0,L/2]); columns k2 = 0 and k2 = L/2
 * are Hermitian in k1, so only their k1 <= L/2 halves are kept, and the
 * four of those that are real (k1, k2 in {0, L/2}) share two slots, leaving
 * bins = L*L/2 slots.  Slot f holds
 *   f = (k2-1)*L + k1             S(k1, k2)   for k2 in [1, L/2-1], k1 in [0, L)
 *   f = L*(L/2-1) + k1 - 1        S(k1, 0)    for k1 in [1, L/2-1]
 *   f = L*(L/2-1) + L/2-2 + k1    S(k1, L/2)  for k1 in [1, L/2-1]
 *   f = L*L/2 - 2                 (S(0, 0), S(L/2, 0))     as (re, im)
 *   f = L*L/2 - 1                 (S(0, L/2), S(L/2, L/2)) as (re, im)
 * The two last slots are multiplied part by part in the per-bin product
 * (a product of two real bins is real), the others as complex numbers.
 * For odd L (the OaAConv configuration) only S(0, 0) is real, nothing is
 * packed, and bins = (L*L+1)/2:
 *   f = (k2-1)*L + k1             S(k1, k2)   for k2 in [1, (L-1)/2], k1 in [0, L)
 *   f = (L-1)/2*L + k1            S(k1, 0)    for k1 in [0, (L-1)/2]
 *
 * Patch index t = (img * tiles_h + a) * tiles_w + b for the patch whose
 * top-left output pixel is (a*T, b*T); t in [tiles, tiles_padded) are zero
 * padding.
 *
 * Layouts (all complex64, innermost index last):
 *   weight spectra  W[bins][cin][cout_padded]        (wspec, wspec_bytes)
 *       = conj(DFT of w[co][ci] zero-padded top-left to L x L) / L^2,
 *         zero for co >= cout
 *   patch spectra   X[cin16/16][bins][16][tiles_padded]  (workspace + xspec_offset)
 *       channel-blocked: channel c of bin f is row c % 16 of block c / 16
 *       (cin16 = cin rounded up to a multiple of 16), so the slots of one
 *       channel are 16 * tiles_padded elements apart
 *   output spectra  Y[cout_padded][tiles_padded/G][bins][G] (workspace + yspec_offset)
 *       patch-group-major, G = spec_group (64, 32, 16 for L = 8, 16, 32):
 *       all slots of one channel and G consecutive patches are one
 *       contiguous run (the unit of work of the inverse transform)
 * The DFT is unnormalised, exp(-2 pi i (m k1 + q k2) / L). */
typedef struct {
    int tile;            /* T */
    int nfft;            /* L = T + k - 1 */
    int tiles_h, tiles_w;/* ceil(h/T), ceil(w/T) */
    int tiles;           /* n * tiles_h * tiles_w */
    int tiles_padded;    /* tiles rounded up to the contraction's tile granularity */
    int bins;            /* L*L/2 ((L*L+1)/2 for odd L) */
    int cout_padded;     /* cout rounded up to the contraction's tile granularity */
    unsigned flags;
    size_t wspec_bytes;
    size_t workspace_bytes;
    size_t xspec_offset, xspec_bytes;
    size_t yspec_offset, yspec_bytes;
    size_t aux_offset, aux_bytes;   /* overlap-add seam partials, room for a patch's whole
                                     * L x L result each, of which the inverse uses at most
                                     * the seams (0 for overlap-save) */
    /* The contraction on the fp32 matrix instruction: output tile
     * contract_tile_m channels x contract_tile_n patches, input channels in
     * stages of contract_stage_k, and 3 (Gauss) or 4 real matrix products
     * per complex multiply-add.  It runs where the environment variable
     * FFTSPLIT_CONTRACT_TILE=[g3:|g4:]MxNxK (which overrides the choice),
     * FFTSPLIT_CONTRACT_PREFETCH=1..3 or FFTSPLIT_CONTRACT_SPLIT=0 asks for it
     * at plan time, where the patches are padded to an odd multiple of 32, and
     * for three or four whole channel blocks in a small grid; otherwise the
     * same product runs on the bf16 matrix instruction with every fp32
     * operand, subnormal ones too, split exactly into three bf16 parts, and is
     * no less precise.  Where operands or sums are not finite, or operands
     * reach 2^104 or sums 2^80, the affected part of the product is computed
     * on the fp32 instruction.  fftsplit_plan_kernels tells which one a plan
     * runs. */
    int contract_tile_m, contract_tile_n, contract_stage_k, contract_real_products;
    int spec_group;      /* G of the output-spectra layout */
    /* 1 if fftsplit_conv2d sums the input channels inside the inverse stage
     * (layers of at most 4 input channels at L = 8, 3 at L = 16, on the
     * overlap-save band path): no contraction launch, and the output
     * spectra region of the workspace is left untouched.  The stage entry
     * points are unaffected. */
    int fused_channel_sum;
    /* Bytes of the filter layout of the direct (spatial) convolution,
     * fftsplit_direct_transform_weights. */
    size_t direct_wspec_bytes;
    /* Input-channel stages the fp32 contraction loads ahead of the one it
     * multiplies: 1 (through registers), or 2 or 3 straight into LDS (2 the
     * default where the tile has that variant, 3 with the 8-channel stages
     * the plan picks for layers of at most 128 input channels and at least
     * 8192 workgroups).  The environment variable
     * FFTSPLIT_CONTRACT_PREFETCH=1..3 overrides it at plan time. */
    int contract_prefetch;
    /* The plan's cost model for the chosen L (Section 3.2 weighs the
     * operations and memory accesses of a patch size; here they are priced
     * at an effective HBM rate and matrix-core rate):
     *   model_contract_flops  = 8 * bins * cin * cout_padded * tiles_padded
     *                           (8 flops per complex multiply-add),
     *   model_transform_bytes = forward bytes (x read once, patch spectra
     *                           written once) + inverse bytes (output spectra
     *                           read once, y written once),
     *   model_seconds         = the modelled time the tile choice minimises. */
    double model_contract_flops;
    double model_transform_bytes;
    double model_seconds;
    /* Transform kernel variants: 1 if the forward / inverse stage runs the
     * row-band kernel (overlap-save, image width a multiple of 4 and at most
     * 256), else the general one; forward_sweep is 1 if the row-band forward
     * spaces each workgroup's work items a grid apart (chosen where the
     * input and the patch spectra together exceed 256 MB;
     * FFTSPLIT_FORWARD_SWEEP=1 / 0 forces it at plan time). */
    int forward_band, forward_sweep, inverse_band;
    /* 1 if the row-band forward reads its input non-temporally (an input
     * larger than the 256 MB last-level cache). */
    int forward_stream;
} fftsplit_plan_info_t;

/* Validate `prob` (host) and create a plan for `device` (a HIP ordinal).
 * The paper leaves the patch size free, to be chosen from the resources of
 * the hardware (Section 3.1, first paragraph), and weighs a patch size by
 * its operation count and memory accesses (Section 3.2, eqs. 13-14).  Here
 * the choice is among the FFT sizes the kernels implement.
 * Queries the device: its gcnArchName must start with "gfx950", else
 * FFTSPLIT_ERROR_ARCH.  With prob->tile == 0 the plan picks T from a cost
 * model over L = 8, 16, 32 (the model_* fields of fftsplit_plan_info_t);
 * the environment variable FFTSPLIT_TILE forces a tile size.  No device memory is touched.  *out is set only on success.
 * Other environment variables read here (for experiments; the defaults are
 * the measured best): FFTSPLIT_CONTRACT_TILE (see contract_tile_m),
 * FFTSPLIT_CONTRACT_PREFETCH (see contract_prefetch),
 * FFTSPLIT_CONTRACT_SPLIT=0 / FFTSPLIT_DIRECT_SPLIT=0 (the contraction / the
 * direct convolution on the fp32 matrix instruction),
 * FFTSPLIT_FORWARD_BAND=0 / FFTSPLIT_INVERSE_BAND=0 (general forward /
 * inverse kernels instead of the row-band ones), FFTSPLIT_FORWARD_SWEEP=1 / 0
 * (the row-band forward's workgroups run items a grid apart, or contiguous
 * runs; by default the former where input and patch spectra exceed 256 MB),
 * FFTSPLIT_FUSE_CIN=0 (no channel sum in the inverse), FFTSPLIT_LOG=1 (print
 * the plan to stderr). */
fftsplit_status_t fftsplit_plan(const fftsplit_problem_t* prob, int device, fftsplit_plan_t* out);

/* As fftsplit_plan, but for a named architecture string (host-only, no HIP
 * call).  The resulting plan can be queried but not executed: the entry
 * points that launch work return FFTSPLIT_ERROR_INVALID_VALUE for it. */
fftsplit_status_t fftsplit_plan_for_arch(const fftsplit_problem_t* prob, const char* arch,
                                         fftsplit_plan_t* out);

/* What the plan decided (Section 3.1: patch size T and FFT size
 * L = T + K - 1; Section 3.2: the cost that chose them), the buffer sizes
 * and layouts the caller must provide, and the kernel variants.  Fails with
 * FFTSPLIT_ERROR_INVALID_VALUE on a NULL argument. */
fftsplit_status_t fftsplit_plan_info(fftsplit_plan_t plan, fftsplit_plan_info_t* out /* host */);

/* The matrix kernels that a plan's entry points launch (fftsplit_plan_info_t
 * describes the fp32 contraction kernel, also for a plan that does not run
 * it). */
typedef struct {
    /* fftsplit_contract (and fftsplit_conv2d, unless fused_channel_sum): 1 if
     * on the bf16 matrix instruction with fp32 operands split into three parts,
     * 0 if on the fp32 one.  A workgroup's output tile is contract_tile_m
     * channels x contract_tile_n patches; the input channels are taken in
     * stages of contract_stage_k, contract_prefetch of them loaded ahead, by
     * contract_wave_groups groups of waves in turn.  A complex multiply-add
     * takes contract_real_products real matrix products of
     * contract_part_products instructions' work each. */
    int contract_split;
    int contract_tile_m, contract_tile_n, contract_stage_k, contract_prefetch, contract_wave_groups;
    int contract_real_products, contract_part_products;
    /* fftsplit_direct_conv2d: 1 if on the bf16 matrix instruction, in blocks
     * of 64 pixels that are direct_block_w wide; 0 (and 0) if on the fp32 one,
     * in runs of pixels. */
    int direct_split, direct_block_w;
    /* The OaAConv configuration's inverse: patch rows (of one plane) and images
     * whose results a workgroup adds up in LDS; 0 and 0 where they go through
     * the aux buffer (planes too wide) and for other configurations. */
    int oaaconv_strip_rows, oaaconv_strip_images;
} fftsplit_plan_kernels_t;

/* Fails with FFTSPLIT_ERROR_INVALID_VALUE on a NULL argument. */
fftsplit_status_t fftsplit_plan_kernels(fftsplit_plan_t plan, fftsplit_plan_kernels_t* out /* host */);

/* Frees a plan's host memory.  NULL is ignored. */
void fftsplit_plan_destroy(fftsplit_plan_t plan);

/* Eq. (8) and the filter half of eq. (9), once per layer:
 * w (device) [cout][cin][k][k] -> wspec (device, info.wspec_bytes).  The
 * spectra are evaluated in double precision and rounded once to fp32. */
fftsplit_status_t fftsplit_transform_weights(fftsplit_plan_t plan, const float* w, void* wspec,
                                             hipStream_t stream);

/* The hot path, Section 3.1 steps 1-6:
 *   x (device) [n][cin][h][w], wspec from fftsplit_transform_weights,
 *   bias (device) [cout] or NULL (required iff FFTSPLIT_BIAS),
 *   y (device) [n][cout][h][w] (must not overlap x),
 *   workspace (device) of at least info.workspace_bytes.
 * Enqueues the forward patch transform, the per-bin contraction and the
 * inverse transform with placement on `stream`. */
fftsplit_status_t fftsplit_conv2d(fftsplit_plan_t plan, const float* x, const void* wspec,
                                  const float* bias, float* y, void* workspace,
                                  size_t workspace_bytes, hipStream_t stream);

/* Bytes of the static device scratch behind fftsplit_conv2d_noalloc. */
#define FFTSPLIT_NOALLOC_MAX_WORKSPACE (256u << 20)

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc):
 * fftsplit_conv2d with the workspace taken from a static device array of
 * FFTSPLIT_NOALLOC_MAX_WORKSPACE bytes (256 MiB) that the library holds on
 * each device it runs on until the process ends.  Same arguments, layouts,
 * kernels and results as fftsplit_conv2d, minus the workspace; calls no
 * allocating routine.  Plans whose info.workspace_bytes exceed the limit
 * get FFTSPLIT_ERROR_INSUFFICIENT_WORKSPACE (nothing enqueued).  Every call
 * on a device shares that device's array: calls that overlap on one device
 * (concurrent streams, or threads) race and must be serialised by the
 * caller.  The array needs no clearing between calls.  The first call on a
 * device looks up the array's device address (hipGetSymbolAddress). */
fftsplit_status_t fftsplit_conv2d_noalloc(fftsplit_plan_t plan, const float* x, const void* wspec,
                                          const float* bias, float* y, hipStream_t stream);

/* The three stages of fftsplit_conv2d, separately (same arguments and
 * workspace layout; running them in order is exactly fftsplit_conv2d).
 * They exist for stage-by-stage testing and per-kernel timing.
 *   forward:  x -> patch spectra at workspace + xspec_offset (eqs. 4-6, FFT)
 *   contract: patch spectra, wspec -> output spectra at yspec_offset (eq. 9)
 *   inverse:  output spectra -> y, with crop/concatenate or overlap-add,
 *             bias and ReLU (eq. 10). */
fftsplit_status_t fftsplit_forward(fftsplit_plan_t plan, const float* x, void* workspace,
                                   size_t workspace_bytes, hipStream_t stream);
fftsplit_status_t fftsplit_contract(fftsplit_plan_t plan, const void* wspec, void* workspace,
                                    size_t workspace_bytes, hipStream_t stream);
fftsplit_status_t fftsplit_inverse(fftsplit_plan_t plan, const float* bias, float* y,
                                   void* workspace, size_t workspace_bytes, hipStream_t stream);

/* The spatial convolution the paper compares the split method against
 * (Section 2, eq. 1 computed directly; Section 4): the same layer as the
 * plan's, as an implicit matrix product in fp32 (on the fp32 matrix
 * instruction, or where that is faster on the bf16 one with every operand,
 * subnormal ones too, split exactly into three parts: no less precise, and
 * back on the fp32 one where a sum is not finite), with the plan's bias and
 * ReLU flags.  The filters are first rearranged once per layer:
 *   fftsplit_direct_transform_weights: w (device) [cout][cin][k][k] ->
 *     wd (device, info.direct_wspec_bytes) = [k*k][cin16][cout_padded],
 *     zero for padded channels;
 *   fftsplit_direct_conv2d: x (device) [n][cin][h][w], wd, bias (device,
 *     [cout] or NULL; required iff FFTSPLIT_BIAS), y (device)
 *     [n][cout][h][w] (must not overlap x or wd).  No workspace.  x must be
 *     under 2 GiB (FFTSPLIT_ERROR_NOT_SUPPORTED otherwise).
 * The plan's tile size and overlap mode do not apply. */
fftsplit_status_t fftsplit_direct_transform_weights(fftsplit_plan_t plan, const float* w, float* wd,
                                                    hipStream_t stream);
fftsplit_status_t fftsplit_direct_conv2d(fftsplit_plan_t plan, const float* x, const float* wd, const float* bias,
                                         float* y, hipStream_t stream);

/* 2x2, stride-2 max-pool (floor), used between the stages of a VGG-16
 * stack; not part of the method.  x (device) [n][c][h][w] ->
 * y (device) [n][c][h/2][w/2].  x and y must not overlap. */
fftsplit_status_t fftsplit_maxpool2x2(const float* x, float* y, int n, int c, int h, int w,
                                      hipStream_t stream);

/* ---------------------------------------------------------------------
 * Operators of the attention blocks that follow a convolution backbone:
 * layer norm, rotary positions over several axes, differential attention,
 * norms of query and key heads with their rotation, linear attention.
 * They are not part of the paper's method.  The conventions above hold,
 * except that tensors may also be bf16 and that attention and the rotation
 * take strides where they say so.
 * ------------------------------------------------------------------- */

typedef enum {
    FFTSPLIT_F32 = 0,
    FFTSPLIT_BF16 = 1
} fftsplit_dtype_t;

/* Differential attention.  Every head holds two softmax maps over the same
 * values; for sequence b, query row i and query head h with key head
 * g = h / (heads_q / heads_k),
 *   o[b][i][h] = sum_j (P1[j] - lam[h] P2[j]) v[b][j][g],
 *   Pm[j] = softmax_j(scale <q[b][i][h][m], k[b][j][g][m]>)  over the visible j.
 * Key j is visible to row i if j < key_lengths[b] and, with causal set, if
 * j <= i + key_lengths[b] - queries (the last row sees every key).  A row
 * that sees no key gives o = 0 and contributes to no gradient, whatever it
 * holds.  What lies in k and v from row key_lengths[b] on is not read.  What
 * causal hides from a row that sees other keys is: it has to be finite, as the
 * row takes zero times it (and in the backward pass the keys take zero times
 * the row's q and dout).
 * Scores, the softmax statistics and all sums are fp32; with bf16 tensors the
 * terms of the softmax (and the score gradients) are rounded to bf16 as
 * operands of the matrix products, those of the forward pass by each map: what
 * that leaves out, 1.7e-3 of either map's output, stays where the maps cancel
 * (plans with key_splits keep it).  fp32 tensors are rounded nowhere. */
typedef struct {
    int batch;            /* sequences */
    int queries, keys;    /* query rows; room for keys (each sequence may fill less); at most 2^28 */
    int heads_q, heads_k; /* heads_k divides heads_q */
    int dim;              /* width of one map's queries and keys, at most 128 */
    int dim_v;            /* width of the values, at most 256 */
    int dtype;            /* fftsplit_dtype_t of q, k, v, o and their gradients */
    int causal;           /* 0 or 1 */
    float scale;          /* factor of the scores; 0: 1 / sqrt(dim) */
} fftsplit_attention_problem_t;

typedef struct fftsplit_attention_plan_s* fftsplit_attention_plan_t;   /* opaque, host-side */

typedef struct {
    size_t forward_workspace_bytes, backward_workspace_bytes;
    size_t lse_bytes;     /* of the statistics saved for the backward pass */
    /* Kernel choice: head widths the tiles are padded to, and how many
     * workgroups share the keys of a tile of few rows (0: the kernel for
     * many rows, whose workgroups each go over all keys). */
    int tile_dim, tile_dim_v, key_splits;
} fftsplit_attention_info_t;

/* Input tensors (device).  Strides are in elements, of the dimensions
 *   q [batch][queries][heads_q][2][dim], k [batch][keys][heads_k][2][dim]:
 *     batch, token, head, map;
 *   v [batch][keys][heads_k][dim_v]: batch, token, head;
 * the last dimension is dense, no stride is negative and those of tokens are at
 * most 2^22.  q, k and v may be slices of one tensor, and rows of each may
 * overlap or be one row for all (stride 0).  Pointers need only their type's alignment; where
 * pointers, strides and widths allow 16-byte accesses those are used.
 *   lam: one value for all heads or one per query head (lam_count 1 or
 *     heads_q), of type lam_dtype;
 *   key_lengths: [batch], or NULL: every sequence has `keys` keys.  Values
 *     outside [0, keys] are taken as the nearest of the two. */
typedef struct {
    const void *q, *k, *v, *lam;
    const int* key_lengths;
    long long q_stride[4], k_stride[4], v_stride[3];
    int lam_dtype, lam_count;
} fftsplit_attention_inputs_t;

/* Validate `prob` and create a plan for `device`, as fftsplit_plan does; the
 * _for_arch form makes one that can be queried but not run. */
fftsplit_status_t fftsplit_attention_plan(const fftsplit_attention_problem_t* prob, int device,
                                          fftsplit_attention_plan_t* out);
fftsplit_status_t fftsplit_attention_plan_for_arch(const fftsplit_attention_problem_t* prob, const char* arch,
                                                   fftsplit_attention_plan_t* out);
fftsplit_status_t fftsplit_attention_plan_info(fftsplit_attention_plan_t plan, fftsplit_attention_info_t* out /* host */);
void fftsplit_attention_plan_destroy(fftsplit_attention_plan_t plan);   /* NULL is ignored */

/* o (device) [batch][queries][heads_q][dim_v], dense, 16-byte aligned.
 * For a backward pass also o1 and o2 (device, the maps' own outputs: fp32
 * whatever o is, laid out as o, 16-byte aligned) and lse (device,
 * info.lse_bytes: fp32 [batch][heads_q][2][queries], log2 of the sum of
 * exp2 of the scaled scores); all NULL otherwise.  Outputs must not
 * overlap the inputs or the workspace (of info.forward_workspace_bytes; NULL
 * allowed if that is 0).  The result does not depend on what runs beside it:
 * no atomics are used. */
fftsplit_status_t fftsplit_attention_forward(fftsplit_attention_plan_t plan, const fftsplit_attention_inputs_t* in /* host */,
                                             void* o, float* o1, float* o2, float* lse, void* workspace, size_t workspace_bytes,
                                             hipStream_t stream);

/* Gradients of fftsplit_attention_forward's inputs from that of o.
 *   dout (device): [batch][queries][heads_q][dim_v], strides batch, token,
 *     head in elements, last dimension dense;
 *   o1, o2, lse: as the forward pass left them;
 *   dq, dk, dv (device): dense, laid out as q, k and v are declared above;
 *     gradients of keys that no query sees (those past key_lengths among
 *     them) are zero; a key head's sums over its query heads;
 *   dlam (device): like lam (type and count; one value sums over heads). */
fftsplit_status_t fftsplit_attention_backward(fftsplit_attention_plan_t plan, const fftsplit_attention_inputs_t* in /* host */,
                                              const void* dout, const long long dout_stride[3], const float* o1,
                                              const float* o2, const float* lse, void* dq, void* dk, void* dv,
                                              void* dlam, void* workspace, size_t workspace_bytes,
                                              hipStream_t stream);

/* Layer norm over the channels of each position of each image or sequence:
 *   y = (x - mean) * rstd * weight + bias,  rstd = 1 / sqrt(var + eps),
 * statistics in fp32 (the mean first, then the squared deviations from it). */
enum {
    FFTSPLIT_CHANNELS_LAST = 0,    /* [batch][positions][channels]: tokens */
    FFTSPLIT_CHANNELS_FIRST = 1    /* [batch][channels][positions]: a feature map */
};
typedef struct {
    /* At most 8192 channels, with x channels first 2048 and 2^22 positions.
     * batch * positions: below 2^25 (2^23 above 1024 channels); with x
     * channels first batch * ceil(positions / 16) below 2^21. */
    int batch, positions, channels;
    int x_dtype, y_dtype;             /* fftsplit_dtype_t; both the same, or fp32 to bf16 */
    int x_layout, y_layout;           /* both the same, or a feature map to tokens */
    float eps;
} fftsplit_layer_norm_t;

/* x (device, x_dtype, x_layout) -> y (device, y_dtype, y_layout); weight and
 * bias (device, fp32 [channels]) or NULL (1 and 0); mean and rstd (device,
 * fp32 [batch][positions], for the backward pass) or both NULL.  Runs on the
 * current device. */
fftsplit_status_t fftsplit_layer_norm(const fftsplit_layer_norm_t* desc /* host */, const void* x, const float* weight,
                                      const float* bias, void* y, float* mean, float* rstd, hipStream_t stream);

/* Gradients: dy (like y), x, mean, rstd, weight as in the forward pass ->
 * dx (like x), dweight and dbias (device, fp32 [channels]; sums over all
 * positions in a fixed order).  workspace: device, of the bytes that
 * fftsplit_layer_norm_workspace gives. */
fftsplit_status_t fftsplit_layer_norm_workspace(const fftsplit_layer_norm_t* desc /* host */, size_t* bytes /* host */);
fftsplit_status_t fftsplit_layer_norm_backward(const fftsplit_layer_norm_t* desc /* host */, const void* dy,
                                               const void* x, const float* mean, const float* rstd,
                                               const float* weight, void* dx, float* dweight, float* dbias,
                                               void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Rotary positions over several axes (row and column of an image's tokens,
 * and time).  The first sections[0] pairs of a head's elements follow the
 * token's first coordinate, the next sections[1] its second, and so on: pair
 * i = (a, b) at coordinate p becomes
 *   (a cos t - b sin t, b cos t + a sin t),  t = p * freqs[i]
 * (inverse: -t, which is also the gradient).  With r pairs in all, pair i is
 * elements (i, i + r), or (2 i, 2 i + 1) where interleaved; elements from 2 r
 * on are passed on.  The angle's whole turns are taken off in 64 bits. */
#define FFTSPLIT_ROTARY_MAX_AXES 4
typedef struct {
    int batch, tokens, dim;        /* dim: elements of a head, at most 1024; batch * tokens at most 2^26 */
    int heads0, heads1;            /* heads of the two tensors; heads1 0: only the first */
    int dtype;                     /* fftsplit_dtype_t */
    int axes;                      /* 1 to FFTSPLIT_ROTARY_MAX_AXES */
    int sections[FFTSPLIT_ROTARY_MAX_AXES];   /* pairs of each axis */
    int positions_per_batch;       /* positions are [batch][tokens][axes], else [tokens][axes] */
    int inverse, interleaved;
} fftsplit_rotary_t;

/* positions (device, int), freqs (device, fp32, one per pair).  x0 -> y0 and,
 * with heads1, x1 -> y1 (device): strides of batch, token and head in
 * elements, last dimension dense.  y may be x (in place, with equal strides)
 * and must not overlap it otherwise.  Runs on the current device. */
fftsplit_status_t fftsplit_rotary(const fftsplit_rotary_t* desc /* host */, const int* positions, const float* freqs,
                                  const void* x0, const long long x0_stride[3], void* y0, const long long y0_stride[3],
                                  const void* x1, const long long x1_stride[3], void* y1, const long long y1_stride[3],
                                  hipStream_t stream);

/* Norm of every head and rotation in one pass, as for queries and keys between
 * a projection and attention.  Of a head x of a token:
 *   y = R (weight * x * rstd),  rstd = 1 / sqrt(mean(x^2) + eps),
 * with the mean over all `dim` elements and the rotation R of fftsplit_rotary
 * (rotary.inverse must be 0).  Everything is fp32 until y is rounded. */
typedef struct {
    fftsplit_rotary_t rotary;
    float eps;                     /* finite, not negative */
} fftsplit_head_norm_t;

/* One of the two tensors (strides as for fftsplit_rotary). */
typedef struct {
    const void* x;                 /* device */
    void* y;                       /* device; may be x (in place, with equal strides), no other overlap */
    long long x_stride[3], y_stride[3];
    const float* weight;           /* device, fp32 [dim], or NULL: 1 */
} fftsplit_head_norm_tensor_t;

/* t1 is NULL unless rotary.heads1.  Runs on the current device. */
fftsplit_status_t fftsplit_head_norm_rotary(const fftsplit_head_norm_t* desc /* host */, const int* positions,
                                            const float* freqs, const fftsplit_head_norm_tensor_t* t0 /* host */,
                                            const fftsplit_head_norm_tensor_t* t1 /* host */, hipStream_t stream);

/* Gradients of one tensor's input and weight; x and weight as in the forward
 * pass, nothing else is saved from it. */
typedef struct {
    const void *dy, *x;            /* device */
    void* dx;                      /* device; may be dy (in place, with equal strides), no other overlap */
    long long dy_stride[3], x_stride[3], dx_stride[3];
    const float* weight;
    float* dweight;                /* device, fp32 [dim]: the sum over all tokens and heads, in a fixed order;
                                    * NULL: not computed */
} fftsplit_head_norm_gradient_t;

/* workspace: device, of the bytes that fftsplit_head_norm_rotary_workspace gives. */
fftsplit_status_t fftsplit_head_norm_rotary_workspace(const fftsplit_head_norm_t* desc /* host */, size_t* bytes /* host */);
fftsplit_status_t fftsplit_head_norm_rotary_backward(const fftsplit_head_norm_t* desc /* host */, const int* positions,
                                                     const float* freqs,
                                                     const fftsplit_head_norm_gradient_t* t0 /* host */,
                                                     const fftsplit_head_norm_gradient_t* t1 /* host */, void* workspace,
                                                     size_t workspace_bytes, hipStream_t stream);

/* Linear attention with a decay for each head: causal, with a state of fixed
 * size in place of a cache.  For sequence b and key head g, with
 * decay = exp(log_decay[g]),
 *   S_t = decay S_(t-1) + k_t v_t^T              (dim x dim_v),
 *   o_t = scale S_t^T q_t                        for the query heads h of g = h / (heads_q / heads_k),
 * from the state that the caller gives, or zero.  Tokens from lengths[b] on are
 * not read; their outputs and gradients are zero, and the state is the one after
 * the last token that is there.
 * Values are taken to be finite.  What takes an infinity or a NaN is not finite, and
 * which of the two it is is not specified: a value's column (a key's row) of the state
 * from its token on, and the outputs of that token, of those behind it and, in calls of
 * more than a few tokens, of up to 31 before it, which the order of tokens hides it
 * from but which are multiplied by zero.  Backwards likewise.
 * States, products and sums are fp32.  With bf16 tensors the scores q k^T (with
 * their decay) and the state that a segment begins with are good to 2^-14 as operands,
 * in calls of more than a few tokens, and only outputs are rounded; what a call returns
 * of a state or its gradient is a sum of unrounded products.  fp32 tensors are rounded
 * nowhere. */
typedef struct {
    int batch;                     /* sequences */
    int tokens;                    /* of the longest; at most 2^28 */
    int heads_q, heads_k;          /* heads_k divides heads_q; v has heads_k heads */
    int dim, dim_v;                /* widths of q and k, and of v and o; at most 256 */
    int dtype;                     /* fftsplit_dtype_t of q, k, v, o and their gradients */
    float scale;                   /* 0: 1 / sqrt(dim) */
} fftsplit_linear_attention_problem_t;

typedef struct fftsplit_linear_attention_plan_s* fftsplit_linear_attention_plan_t;   /* opaque, host-side */

typedef struct {
    size_t forward_workspace_bytes, backward_workspace_bytes;
    size_t state_bytes;            /* fp32 [batch][heads_k][dim][dim_v] */
    /* Kernel choice: 1 if the forward pass goes token by token, else 0; tokens of
     * a segment, within which pairs of tokens are taken one by one and between
     * which a state is carried, and how many a sequence is cut into (one that is not
     * long is taken as one segment where no state is returned). */
    int recurrent, segment_tokens, segments;
} fftsplit_linear_attention_info_t;

/* Input tensors (device).  Strides are in elements, of the dimensions
 *   q [batch][tokens][heads_q][dim], k [batch][tokens][heads_k][dim],
 *   v [batch][tokens][heads_k][dim_v]: batch, token, head;
 * the last dimension is dense, no stride is negative and those of tokens are at
 * most 2^22.  q, k and v may be slices of one tensor and overlap.  Pointers need
 * only their type's alignment; where pointers, strides and widths allow 16-byte
 * accesses those are used.
 *   log_decay: fp32 [heads_k]; values above 0 are taken as 0.  No gradient of it
 *     is computed: decays are constants of a model.
 *   lengths: [batch], or NULL: every sequence has `tokens` tokens.  Values
 *     outside [0, tokens] are taken as the nearest of the two.
 *   state: fp32 [batch][heads_k][dim][dim_v], dense, 16-byte aligned, or NULL: zero. */
typedef struct {
    const void *q, *k, *v;
    const float* log_decay;
    const int* lengths;
    const float* state;
    long long q_stride[3], k_stride[3], v_stride[3];
} fftsplit_linear_attention_inputs_t;

/* Validate `prob` and create a plan for `device`, as fftsplit_plan does; the
 * _for_arch form makes one that can be queried but not run. */
fftsplit_status_t fftsplit_linear_attention_plan(const fftsplit_linear_attention_problem_t* prob, int device,
                                                 fftsplit_linear_attention_plan_t* out);
fftsplit_status_t fftsplit_linear_attention_plan_for_arch(const fftsplit_linear_attention_problem_t* prob,
                                                          const char* arch, fftsplit_linear_attention_plan_t* out);
fftsplit_status_t fftsplit_linear_attention_plan_info(fftsplit_linear_attention_plan_t plan,
                                                      fftsplit_linear_attention_info_t* out /* host */);
void fftsplit_linear_attention_plan_destroy(fftsplit_linear_attention_plan_t plan);   /* NULL is ignored */

/* o (device) [batch][tokens][heads_q][dim_v], dense, 16-byte aligned; state_out
 * (device): laid out as state, the state after each sequence's last token, or
 * NULL.  It may be `state` (in place); outputs and the workspace (of
 * info.forward_workspace_bytes; NULL allowed if that is 0) must not overlap
 * anything else.  No atomics are used. */
fftsplit_status_t fftsplit_linear_attention_forward(fftsplit_linear_attention_plan_t plan,
                                                    const fftsplit_linear_attention_inputs_t* in /* host */, void* o,
                                                    float* state_out, void* workspace, size_t workspace_bytes,
                                                    hipStream_t stream);

/* Gradients of fftsplit_linear_attention_forward's inputs.
 *   dout (device): the gradient of o, strides batch, token, head in elements,
 *     last dimension dense; dstate_out (device): that of state_out, laid out as
 *     state, or NULL: zero;
 *   dq, dk, dv (device): dense, 16-byte aligned, laid out as q, k and v are
 *     declared above; a key head's are sums over its query heads;
 *   dstate (device): the gradient of state, or NULL: not computed. */
fftsplit_status_t fftsplit_linear_attention_backward(fftsplit_linear_attention_plan_t plan,
                                                     const fftsplit_linear_attention_inputs_t* in /* host */,
                                                     const void* dout, const long long dout_stride[3],
                                                     const float* dstate_out, void* dq, void* dk, void* dv, float* dstate,
                                                     void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Benchmark hook (host, per calling thread): until called again with
 * NULL, NULL, every later fftsplit_transform_weights / fftsplit_conv2d /
 * stage call made by this thread records `start` (if non-NULL) when its
 * first kernel begins executing and `stop` (if non-NULL) when its last
 * kernel ends, using the kernels' own dispatch timestamps
 * (hipExtLaunchKernel) rather than separate event packets; the two
 * measurement probes below are timed the same way.  The events
 * must be valid hipEvents created with timing enabled, on the plan's
 * device.  Always returns FFTSPLIT_SUCCESS. */
fftsplit_status_t fftsplit_set_timing_events(hipEvent_t start, hipEvent_t stop);

/* Measurement hooks: the practical ceilings the path's kernels are
 * measured against, on the device they run on.  Neither computes anything
 * of the method.
 *
 * fftsplit_probe_matrix: enqueues on `stream` (on the plan's device) one
 * kernel with the launch of the plan's fp32 contraction kernel (the
 * contract_* fields of fftsplit_plan_info_t, also for a plan whose
 * fftsplit_contract runs on the bf16 instruction) -- the same grid of
 * 256-thread workgroups and the same dynamic LDS, hence the same workgroups
 * per compute unit -- in which every wave issues as many fp32 matrix
 * operations (v_mfma_f32_32x32x2f32) as a wave of that kernel does, with
 * operands in registers and no other memory traffic.  Its duration is the
 * time the fp32 matrix cores need for those operations at this launch
 * shape.  `sink` (device, one float) is written
 * only if the sum of a wave's accumulators is exactly -1, which it never
 * is.  INVALID_VALUE for a NULL plan or sink or an architecture-only plan;
 * NOT_SUPPORTED for a plan whose channel sum runs inside the inverse (it
 * has no contraction).
 *
 * fftsplit_probe_stream: enqueues on `stream` (current device) a plain
 * streaming kernel that loads `read_bytes` from src and stores
 * `write_bytes` to dst, 16 bytes per lane, from 8192 workgroups of 256
 * threads: dst[i] = src[i] for the first min(read_bytes, write_bytes)
 * bytes, zero for the rest of dst.  Its duration is what HBM needs for
 * that read/write mix (e.g. a transform's bytes).  Both pointers device,
 * 16-byte aligned, sizes multiples of 16, not overlapping; INVALID_VALUE
 * otherwise. */
fftsplit_status_t fftsplit_probe_matrix(fftsplit_plan_t plan, float* sink, hipStream_t stream);
fftsplit_status_t fftsplit_probe_stream(const void* src, void* dst, size_t read_bytes, size_t write_bytes,
                                        hipStream_t stream);

/* Static description of a status code. */
const char* fftsplit_status_string(fftsplit_status_t status);

/* Detail of the calling thread's last failure (empty string if none).
 * Valid until the thread's next call into the library. */
const char* fftsplit_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* FFTSPLIT_H */
