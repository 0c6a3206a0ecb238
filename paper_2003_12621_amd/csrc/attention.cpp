// Differential attention: plans, argument checks and launches.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <new>
#include <string>

#include "attn_internal.hpp"
#include "entry_checks.hpp"
#include "launch_util.hpp"

using namespace fftsplit;

namespace {

// Bytes from the first element of a strided tensor to the end of its last.
size_t extent(const int* dims, const long long* strides, int nd, int width, int bytes) {
    size_t last = 0;
    for (int i = 0; i < nd; ++i) last += size_t(dims[i] - 1) * size_t(strides[i]);
    return (last + size_t(width)) * size_t(bytes);
}

// Whether 16-byte accesses of rows are aligned and whole.
bool wide(const void* p, const int* dims, const long long* strides, int nd, int width, int bytes) {
    const int per = 16 / bytes;
    bool ok = reinterpret_cast<uintptr_t>(p) % 16 == 0 && width % per == 0;
    for (int i = 0; i < nd; ++i) ok = ok && (dims[i] == 1 || strides[i] % per == 0);
    return ok;
}

fftsplit_status_t check_strides(const int* dims, const long long* strides, int nd, const char* name) {
    for (int i = 0; i < nd; ++i) {
        if (strides[i] < 0) return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(name) + " has a negative stride");
        if (dims[i] > 1 && size_t(strides[i]) > (size_t(1) << 58) / size_t(dims[i]))
            return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(name) + " has a stride out of range");
        // (a tile's rows are addressed with 32-bit offsets from its first)
        if (i == 1 && dims[i] > 1 && strides[i] > kAttnMaxTokenStride)
            return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, std::string(name) + ": token strides above 2^22 elements");
    }
    return FFTSPLIT_SUCCESS;
}

int shape_index(int d, int dv) {
    for (int i = 0; i < kAttnShapeCount; ++i)
        if (d <= kAttnShapes[i].d && dv <= kAttnShapes[i].dv) return i;
    return -1;
}

size_t round256(size_t v) { return (v + 255) / 256 * 256; }

size_t output_bytes(const fftsplit_attention_problem_t& p) {
    return size_t(p.batch) * p.queries * p.heads_q * p.dim_v * type_bytes(p.dtype);
}
size_t map_output_bytes(const fftsplit_attention_problem_t& p) {
    return size_t(p.batch) * p.queries * p.heads_q * p.dim_v * 4;
}
size_t lse_bytes(const fftsplit_attention_problem_t& p) { return size_t(p.batch) * p.heads_q * 2 * p.queries * 4; }

// How many workgroups share the keys of a tile of the kernel for few rows, or
// 0 for the kernel that takes kAttnTiledRows rows of one head.
//
// The kernel for few rows pays a second launch and reads the keys once for every
// 32 rows, but uses the whole chip for a handful of rows.  Which is faster, and
// with how many workgroups, is taken from what a step of either was measured to
// take (us), the tiled kernel's of 32 keys, the other's of 128; 12 and 3 us are
// the launches, 0.02 us a workgroup the join.  Measured, tiled / few rows: 128
// rows x 4096 keys, 4 heads 94 / 22 us; 1024 x 1024, 4 heads 28 / 24; 100 x 100,
// 8 heads 8 / 12; 784 x 784, 16 heads 25 / 53.
int choose_splits(const fftsplit_attention_problem_t& p, int shape) {
    static const double kTiledStep[2][kAttnShapeCount] = {{2.2, 3.3, 6.6}, {0.55, 0.72, 1.0}};      // fp32, bf16
    static const double kFewStep[2][kAttnShapeCount] = {{3.8, 13.4, 27.0}, {0.75, 1.65, 3.8}};
    const int type = p.dtype == FFTSPLIT_BF16;
    const long long group = p.heads_q / p.heads_k, heads = (long long)p.batch * p.heads_k;
    const long long tiled = heads * group * ((p.queries + kAttnTiledRows - 1) / kAttnTiledRows);
    const long long few = heads * ((group * p.queries + kAttnFewRows - 1) / kAttnFewRows);
    if (tiled > 512 || few > 256) return 0;
    double best = 3 + kTiledStep[type][shape] * ((p.keys + 31) / 32);
    int splits = 0;
    for (int s = 1; s <= 32 && few * s <= 256; s *= 2) {
        const double t = 12 + kFewStep[type][shape] * ((p.keys + 128LL * s - 1) / (128 * s)) + 0.02 * double(few * s);
        if (t < best) {
            best = t;
            splits = s;
        }
    }
    return splits;
}

// Workgroups that share the steps of a tile of 128 keys or rows in the backward
// pass: as many as run at once, of at least 8 steps each (bf16; an fp32 step
// takes four times as long).  Two run at once on a compute unit up to bf16 heads
// of 64 / 128.  Wider heads have two or three workgroups a tile as it is, and
// one of fp32 keeps a unit's matrix instructions busy: two took 39 and 31 us for
// the two sides of 6 x 301 tokens of 6 heads of 32 / 64, one takes 35 and 28.
// Their parts are added up by another launch.
int choose_backward_splits(const fftsplit_attention_problem_t& p, int shape, long long tiles, long long steps) {
    const bool two = p.dtype == FFTSPLIT_BF16 && shape < 2;
    const long long least = p.dtype == FFTSPLIT_F32 ? 2 : 8;
    long long splits = (two ? 512 : 256) / tiles;
    if (splits > steps / least) splits = steps / least;
    if (splits > 8) splits = 8;
    return splits < 1 ? 1 : int(splits);
}
// fp32 plans keep every row's D2 for dlam.
size_t second_bytes(const fftsplit_attention_problem_t& p) {
    return p.dtype == FFTSPLIT_F32 ? round256(size_t(p.batch) * p.heads_q * p.queries * 4) : 0;
}
size_t key_part_bytes(const fftsplit_attention_problem_t& p, int splits) {
    return splits > 1 ? round256(size_t(splits) * p.batch * p.keys * p.heads_k * (2 * p.dim + p.dim_v) * 4) : 0;
}
size_t query_part_bytes(const fftsplit_attention_problem_t& p, int splits) {
    return splits > 1 ? round256(size_t(splits) * p.batch * p.queries * p.heads_q * 2 * p.dim * 4) : 0;
}

// Parts of dlam of a head: one from each workgroup of the query side.
int dlam_parts(const fftsplit_attention_problem_t& p, int query_splits) {
    return p.batch * ((p.queries + kAttnRows - 1) / kAttnRows) * query_splits;
}

fftsplit_status_t build(const fftsplit_attention_problem_t* prob, int device, const char* arch,
                        fftsplit_attention_plan_t* out) {
    if (!prob || !out) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "problem and output pointers must be non-NULL");
    const fftsplit_attention_problem_t p = *prob;
    if (p.batch <= 0 || p.queries <= 0 || p.keys <= 0 || p.heads_q <= 0 || p.heads_k <= 0 || p.dim <= 0 || p.dim_v <= 0)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "all dimensions must be positive");
    if (p.heads_q % p.heads_k) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "heads_k must divide heads_q");
    if (!known_type(p.dtype))
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "attention: fp32 and bf16 only");
    if (p.causal != 0 && p.causal != 1) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "causal must be 0 or 1");
    if (!(p.scale >= 0.f) || !std::isfinite(p.scale))
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "scale must be finite and positive, or 0 for 1 / sqrt(dim)");
    const int shape = shape_index(p.dim, p.dim_v);
    if (shape < 0) return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "attention: dim at most 128 and dim_v at most 256");
    // Token counts and launch sizes stay below 2^30; element offsets are 64-bit.
    const double rows = double(p.batch) * p.heads_q * p.queries, keys = double(p.batch) * p.heads_q * p.keys;
    if (p.queries > (1 << 28) || p.keys > (1 << 28) || rows > double(1u << 30) || keys > double(1u << 30))
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "attention: at most 2^28 queries and keys, and 2^30 of them over all heads and sequences");

    char archbuf[64] = {0};
    if (device >= 0) {
        hipDeviceProp_t prop;
        const hipError_t e = hipGetDeviceProperties(&prop, device);
        if (e != hipSuccess)
            return fail(FFTSPLIT_ERROR_DEVICE, std::string("hipGetDeviceProperties: ") + hipGetErrorString(e));
        std::snprintf(archbuf, sizeof(archbuf), "%s", prop.gcnArchName);
    } else {
        std::snprintf(archbuf, sizeof(archbuf), "%s", arch);
    }
    if (std::strncmp(archbuf, "gfx950", 6) != 0)
        return fail(FFTSPLIT_ERROR_ARCH, std::string("device architecture '") + archbuf + "' is not gfx950");

    auto* plan = new (std::nothrow) fftsplit_attention_plan_s();
    if (!plan) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "out of host memory");
    plan->prob = p;
    plan->device = device;
    plan->scale = p.scale > 0.f ? p.scale : float(1.0 / std::sqrt(double(p.dim)));
    plan->shape = shape;
    plan->splits = choose_splits(p, shape);
    const size_t parts = size_t(rows) * plan->splits;
    plan->forward_ws = plan->splits ? round256(parts * 2 * kAttnShapes[shape].dv * 4) + round256(parts * 4 * 4) : 0;
    const long long group = p.heads_q / p.heads_k;
    plan->key_splits = choose_backward_splits(p, shape, (long long)p.batch * p.heads_k * ((p.keys + 127LL) / 128),
                                              group * ((p.queries + 31LL) / 32));
    plan->query_splits = choose_backward_splits(p, shape, (long long)p.batch * p.heads_q * ((p.queries + 127LL) / 128),
                                                (p.keys + 31LL) / 32);
    plan->backward_ws = round256(lse_bytes(p)) + round256(size_t(p.heads_q) * (dlam_parts(p, plan->query_splits) + 1) * 4) +
                        key_part_bytes(p, plan->key_splits) + query_part_bytes(p, plan->query_splits) + second_bytes(p);
    // workgroups of the largest launches (a dimension of a grid holds below 2^32 threads)
    const double heads = double(p.batch) * p.heads_q;
    const double groups[] = {heads * ((p.queries + 63) / 64), heads * ((p.keys + 127) / 128) * plan->key_splits,
                             heads * ((p.queries + 127) / 128) * plan->query_splits};
    for (double g : groups)
        if (g > double(1 << 22)) {
            delete plan;
            return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "attention: too many tiles of queries or keys (2^22)");
        }
    *out = plan;
    return FFTSPLIT_SUCCESS;
}

fftsplit_status_t check_plan(fftsplit_attention_plan_t plan) {
    if (!plan) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "plan is NULL");
    if (plan->device < 0)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "plan was created for an architecture name only and cannot run");
    return FFTSPLIT_SUCCESS;
}

// Checks the inputs and fills the kernels' arguments with them.
fftsplit_status_t check_inputs(fftsplit_attention_plan_t plan, const fftsplit_attention_inputs_t* in, AttnArgs& a,
                               Spans& spans) {
    if (!in) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "inputs is NULL");
    const fftsplit_attention_problem_t& p = plan->prob;
    const int es = type_bytes(p.dtype);
    if (fftsplit_status_t s = check_device_ptr(in->q, "q", es)) return s;
    if (fftsplit_status_t s = check_device_ptr(in->k, "k", es)) return s;
    if (fftsplit_status_t s = check_device_ptr(in->v, "v", es)) return s;
    if (!known_type(in->lam_dtype))
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "lam: fp32 and bf16 only");
    if (in->lam_count != 1 && in->lam_count != p.heads_q)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "lam_count must be 1 or heads_q");
    if (fftsplit_status_t s = check_device_ptr(in->lam, "lam", type_bytes(in->lam_dtype))) return s;
    if (reinterpret_cast<uintptr_t>(in->key_lengths) % 4)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "key_lengths is not 4-byte aligned");
    const int qd[4] = {p.batch, p.queries, p.heads_q, 2}, kd[4] = {p.batch, p.keys, p.heads_k, 2};
    const int vd[3] = {p.batch, p.keys, p.heads_k};
    if (fftsplit_status_t s = check_strides(qd, in->q_stride, 4, "q")) return s;
    if (fftsplit_status_t s = check_strides(kd, in->k_stride, 4, "k")) return s;
    if (fftsplit_status_t s = check_strides(vd, in->v_stride, 3, "v")) return s;

    a.q = in->q;
    a.k = in->k;
    a.v = in->v;
    a.lam = in->lam;
    a.lengths = in->key_lengths;
    a.n = p.batch;
    a.sq = p.queries;
    a.sk = p.keys;
    a.hq = p.heads_q;
    a.hk = p.heads_k;
    a.d = p.dim;
    a.dv = p.dim_v;
    a.causal = p.causal;
    a.scale = plan->scale;
    a.scale_log2 = float(double(plan->scale) * 1.4426950408889634);
    a.lam_f32 = in->lam_dtype == FFTSPLIT_F32;
    a.lam_step = in->lam_count == 1 ? 0 : 1;
    a.qb = in->q_stride[0];
    a.qt = in->q_stride[1];
    a.qh = in->q_stride[2];
    a.qm = in->q_stride[3];
    a.kb = in->k_stride[0];
    a.kt = in->k_stride[1];
    a.kh = in->k_stride[2];
    a.km = in->k_stride[3];
    a.vb = in->v_stride[0];
    a.vt = in->v_stride[1];
    a.vh = in->v_stride[2];
    a.wide = wide(in->q, qd, in->q_stride, 4, p.dim, es) && wide(in->k, kd, in->k_stride, 4, p.dim, es) &&
             wide(in->v, vd, in->v_stride, 3, p.dim_v, es);
    a.o_wide = p.dim_v % 4 == 0;
    spans.add(in->q, extent(qd, in->q_stride, 4, p.dim, es), "q");
    spans.add(in->k, extent(kd, in->k_stride, 4, p.dim, es), "k");
    spans.add(in->v, extent(vd, in->v_stride, 3, p.dim_v, es), "v");
    spans.add(in->lam, size_t(in->lam_count) * type_bytes(in->lam_dtype), "lam");
    spans.add(in->key_lengths, size_t(p.batch) * 4, "key_lengths");
    return FFTSPLIT_SUCCESS;
}

}  // namespace

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_attention_plan(const fftsplit_attention_problem_t* prob, int device,
                                                          fftsplit_attention_plan_t* out) {
    return guarded([&] {
        if (device < 0) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "device ordinal must be >= 0");
        return build(prob, device, nullptr, out);
    });
}

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_attention_plan_for_arch(const fftsplit_attention_problem_t* prob,
                                                                   const char* arch, fftsplit_attention_plan_t* out) {
    return guarded([&] {
        if (!arch) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "architecture string must be non-NULL");
        return build(prob, -1, arch, out);
    });
}

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_attention_plan_info(fftsplit_attention_plan_t plan,
                                                               fftsplit_attention_info_t* out) {
    return guarded([&] {
        if (!plan || !out) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "plan and output must be non-NULL");
        fftsplit_attention_info_t i{};
        i.forward_workspace_bytes = plan->forward_ws;
        i.backward_workspace_bytes = plan->backward_ws;
        i.lse_bytes = lse_bytes(plan->prob);
        i.tile_dim = kAttnShapes[plan->shape].d;
        i.tile_dim_v = kAttnShapes[plan->shape].dv;
        i.key_splits = plan->splits;
        *out = i;
        return FFTSPLIT_SUCCESS;
    });
}

FFTSPLIT_EXPORT void fftsplit_attention_plan_destroy(fftsplit_attention_plan_t plan) { delete plan; }

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_attention_forward(fftsplit_attention_plan_t plan,
                                                             const fftsplit_attention_inputs_t* in, void* o, float* o1,
                                                             float* o2, float* lse, void* workspace, size_t workspace_bytes,
                                                             hipStream_t stream) {
    return guarded([&] {
        if (fftsplit_status_t s = check_plan(plan)) return s;
        AttnArgs a{};
        Spans ins, outs;
        if (fftsplit_status_t s = check_inputs(plan, in, a, ins)) return s;
        if (fftsplit_status_t s = check_device_ptr(o, "o", 16)) return s;
        if (!o1 != !lse || !o2 != !lse)
            return fail(FFTSPLIT_ERROR_INVALID_VALUE, "o1, o2 and lse must all be given or all be NULL");
        if (lse) {
            if (fftsplit_status_t s = check_device_ptr(o1, "o1", 16)) return s;
            if (fftsplit_status_t s = check_device_ptr(o2, "o2", 16)) return s;
            if (fftsplit_status_t s = check_device_ptr(lse, "lse", 16)) return s;
        }
        if (fftsplit_status_t s = check_scratch(workspace, workspace_bytes, plan->forward_ws)) return s;
        outs.add(o, output_bytes(plan->prob), "o");
        outs.add(o1, map_output_bytes(plan->prob), "o1");
        outs.add(o2, map_output_bytes(plan->prob), "o2");
        outs.add(lse, lse_bytes(plan->prob), "lse");
        outs.add(workspace, plan->forward_ws, "the workspace");
        if (fftsplit_status_t s = check_apart(ins, outs)) return s;
        a.o = o;
        a.o1 = o1;
        a.o2 = o2;
        a.lse = lse;
        a.splits = plan->splits;
        if (plan->splits) {
            const size_t parts = size_t(a.n) * a.hq * a.sq * plan->splits;
            a.part = static_cast<float*>(workspace);
            a.part_stats = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                                    round256(parts * 2 * kAttnShapes[plan->shape].dv * 4));
        }
        DeviceGuard g(plan->device);
        if (!g.ok()) return fail(FFTSPLIT_ERROR_DEVICE, "cannot select the plan's device");
        return launched_ok(launch_attn_forward(*plan, a, stream, timing_events()), "attention launch");
    });
}

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_attention_backward(fftsplit_attention_plan_t plan,
                                                              const fftsplit_attention_inputs_t* in, const void* dout,
                                                              const long long dout_stride[3], const float* o1,
                                                              const float* o2, const float* lse, void* dq, void* dk,
                                                              void* dv, void* dlam, void* workspace,
                                                              size_t workspace_bytes, hipStream_t stream) {
    return guarded([&] {
        if (fftsplit_status_t s = check_plan(plan)) return s;
        AttnArgs a{};
        Spans ins, outs;
        if (fftsplit_status_t s = check_inputs(plan, in, a, ins)) return s;
        const fftsplit_attention_problem_t& p = plan->prob;
        const int es = type_bytes(p.dtype);
        if (fftsplit_status_t s = check_device_ptr(dout, "dout", es)) return s;
        if (!dout_stride) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "dout_stride is NULL");
        const int gd[3] = {p.batch, p.queries, p.heads_q};
        if (fftsplit_status_t s = check_strides(gd, dout_stride, 3, "dout")) return s;
        if (fftsplit_status_t s = check_device_ptr(o1, "o1", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(o2, "o2", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(lse, "lse", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(dq, "dq", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(dk, "dk", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(dv, "dv", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(dlam, "dlam", type_bytes(in->lam_dtype))) return s;
        if (fftsplit_status_t s = check_scratch(workspace, workspace_bytes, plan->backward_ws)) return s;
        ins.add(dout, extent(gd, dout_stride, 3, p.dim_v, es), "dout");
        ins.add(o1, map_output_bytes(p), "o1");
        ins.add(o2, map_output_bytes(p), "o2");
        ins.add(lse, lse_bytes(p), "lse");
        outs.add(dq, size_t(p.batch) * p.queries * p.heads_q * 2 * p.dim * es, "dq");
        outs.add(dk, size_t(p.batch) * p.keys * p.heads_k * 2 * p.dim * es, "dk");
        outs.add(dv, size_t(p.batch) * p.keys * p.heads_k * p.dim_v * es, "dv");
        outs.add(dlam, size_t(in->lam_count) * type_bytes(in->lam_dtype), "dlam");
        outs.add(workspace, plan->backward_ws, "the workspace");
        if (fftsplit_status_t s = check_apart(ins, outs)) return s;
        a.o1 = const_cast<float*>(o1);
        a.o2 = const_cast<float*>(o2);
        a.lse = const_cast<float*>(lse);
        a.dout = dout;
        a.gb = dout_stride[0];
        a.gt = dout_stride[1];
        a.gh = dout_stride[2];
        a.wide = a.wide && wide(dout, gd, dout_stride, 3, p.dim_v, es);
        a.parts = dlam_parts(p, plan->query_splits);
        a.delta = static_cast<float*>(workspace);
        a.dlam_part = reinterpret_cast<float*>(static_cast<char*>(workspace) + round256(lse_bytes(p)));
        a.key_splits = plan->key_splits;
        a.query_splits = plan->query_splits;
        a.lam32 = a.dlam_part + size_t(p.heads_q) * a.parts;
        a.key_part = a.dlam_part + round256(size_t(p.heads_q) * (a.parts + 1) * 4) / 4;
        a.query_part = a.key_part + key_part_bytes(p, plan->key_splits) / 4;
        a.second = a.query_part + query_part_bytes(p, plan->query_splits) / 4;
        a.dq = dq;
        a.dk = dk;
        a.dv_out = dv;
        a.dlam = dlam;
        DeviceGuard g(plan->device);
        if (!g.ok()) return fail(FFTSPLIT_ERROR_DEVICE, "cannot select the plan's device");
        return launched_ok(launch_attn_backward(*plan, a, stream, timing_events()), "attention gradient launch");
    });
}
