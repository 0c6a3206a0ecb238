// Linear attention: plans, argument checks and launches.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <new>
#include <string>

#include "entry_checks.hpp"
#include "launch_util.hpp"
#include "linear_internal.hpp"

using namespace fftsplit;

namespace {

size_t extent(const int* dims, const long long* strides, int width, int bytes) {
    size_t last = 0;
    for (int i = 0; i < 3; ++i) last += size_t(dims[i] - 1) * size_t(strides[i]);
    return (last + size_t(width)) * size_t(bytes);
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Whether 16-byte accesses of rows are aligned and whole.
bool wide_rows(const void* p, const int* dims, const long long* strides, int width, int bytes) {
    const int per = 16 / bytes;
    bool ok = aligned16(p) && width % per == 0;
    for (int i = 0; i < 3; ++i) ok = ok && (dims[i] == 1 || strides[i] % per == 0);
    return ok;
}

// One strided input: checks it, notes its extent and describes its rows.
fftsplit_status_t check_rows(const void* p, const long long* strides, int n, int s, int heads, int width, int dtype,
                             const char* name, LinearRows& rows, int& wide, Spans& spans) {
    const int es = type_bytes(dtype), dims[3] = {n, s, heads};
    if (fftsplit_status_t st = check_device_ptr(p, name, unsigned(es))) return st;
    for (int i = 0; i < 3; ++i) {
        if (strides[i] < 0) return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(name) + " has a negative stride");
        if (dims[i] > 1 && size_t(strides[i]) > (size_t(1) << 58) / size_t(dims[i]))
            return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(name) + " has a stride out of range");
    }
    if (s > 1 && strides[1] > kLinearMaxTokenStride)
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, std::string(name) + ": token strides above 2^22 elements");
    // (the stride of a dimension of one does not matter)
    rows = LinearRows{p, n > 1 ? strides[0] : 0, s > 1 ? strides[1] : 0, heads > 1 ? strides[2] : 0};
    const long long used[3] = {rows.b, rows.t, rows.h};
    wide = wide && wide_rows(p, dims, used, width, es);
    spans.add(p, extent(dims, used, width, es), name);
    return FFTSPLIT_SUCCESS;
}

size_t round256(size_t v) { return (v + 255) / 256 * 256; }

size_t state_bytes(const fftsplit_linear_attention_problem_t& p) {
    return size_t(p.batch) * p.heads_k * p.dim * p.dim_v * 4;
}

// Into how many parts to cut the sequences so that the waves of `workgroups` of
// them fill the chip.
void choose_segments(const fftsplit_linear_attention_problem_t& p, long long waves, int& segments, int& tokens) {
    const long long chunks = (p.tokens + kLinearChunk - 1) / kLinearChunk;
    long long want = (1024 + waves - 1) / waves;
    if (want > chunks / 4) want = chunks / 4;
    if (want > kLinearMaxSegments) want = kLinearMaxSegments;
    if (want < 1) want = 1;
    const long long per = (chunks + want - 1) / want;
    segments = int((chunks + per - 1) / per);
    tokens = int(per * kLinearChunk < p.tokens ? per * kLinearChunk : p.tokens);
}

long long slices(int width) { return (width + 31) / 32; }

fftsplit_status_t build(const fftsplit_linear_attention_problem_t* prob, int device, const char* arch,
                        fftsplit_linear_attention_plan_t* out) {
    if (!prob || !out) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "problem and output pointers must be non-NULL");
    const fftsplit_linear_attention_problem_t p = *prob;
    if (p.batch <= 0 || p.tokens <= 0 || p.heads_q <= 0 || p.heads_k <= 0 || p.dim <= 0 || p.dim_v <= 0)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "all dimensions must be positive");
    if (p.heads_q % p.heads_k) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "heads_k must divide heads_q");
    if (!known_type(p.dtype)) return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "linear attention: fp32 and bf16 only");
    if (!(p.scale >= 0.f) || !std::isfinite(p.scale))
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "scale must be finite and positive, or 0 for 1 / sqrt(dim)");
    if (p.dim > kLinearMaxDim || p.dim_v > kLinearMaxDim)
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "linear attention: dim and dim_v at most 256");
    // Row numbers of all sequences and heads stay below 2^30; element offsets are 64-bit.
    if (p.tokens > (1 << 28) || double(p.batch) * p.heads_q * p.tokens > double(1u << 30))
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED,
                    "linear attention: at most 2^28 tokens, and 2^30 of them over all heads and sequences");

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

    auto* plan = new (std::nothrow) fftsplit_linear_attention_plan_s();
    if (!plan) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "out of host memory");
    plan->prob = p;
    plan->device = device;
    plan->scale = p.scale > 0.f ? p.scale : float(1.0 / std::sqrt(double(p.dim)));
    plan->recurrent = p.tokens <= kLinearRecurrentTokens;
    const long long heads_k = (long long)p.batch * p.heads_k, heads_q = (long long)p.batch * p.heads_q;
    choose_segments(p, heads_q * slices(p.dim_v), plan->segments[0], plan->segment_tokens[0]);
    choose_segments(p, heads_k * slices(p.dim), plan->segments[1], plan->segment_tokens[1]);
    // (one segment of several query heads: the state that all of them start from
    // has to stay while one of them writes the last)
    const bool shared = p.heads_q > p.heads_k;
    plan->forward_ws = plan->recurrent || (plan->segments[0] == 1 && !shared)
                           ? 0 : round256(state_bytes(p) * size_t(plan->segments[0]));
    plan->backward_ws = plan->segments[1] == 1 ? 0 : 2 * round256(state_bytes(p) * size_t(plan->segments[1]));
    // workgroups of the largest launches (a dimension of a grid holds below 2^32 threads)
    const double most = double(heads_q) * slices(p.dim > p.dim_v ? p.dim : p.dim_v) *
                        (plan->segments[0] > plan->segments[1] ? plan->segments[0] : plan->segments[1]);
    const double joined = double(heads_k) * ((double(p.dim) * p.dim_v + 255) / 256);
    if (most > double(1 << 22) || joined > double(1 << 22)) {
        delete plan;
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "linear attention: too many heads over all sequences");
    }
    *out = plan;
    return FFTSPLIT_SUCCESS;
}

fftsplit_status_t check_plan(fftsplit_linear_attention_plan_t plan) {
    if (!plan) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "plan is NULL");
    if (plan->device < 0)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "plan was created for an architecture name only and cannot run");
    return FFTSPLIT_SUCCESS;
}

struct Inputs {
    LinearRows q, k, v;
    int wide = 1;
};

fftsplit_status_t check_inputs(fftsplit_linear_attention_plan_t plan, const fftsplit_linear_attention_inputs_t* in,
                               Inputs& x, Spans& spans) {
    if (!in) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "inputs is NULL");
    const fftsplit_linear_attention_problem_t& p = plan->prob;
    if (fftsplit_status_t s = check_rows(in->q, in->q_stride, p.batch, p.tokens, p.heads_q, p.dim, p.dtype, "q", x.q, x.wide,
                                         spans))
        return s;
    if (fftsplit_status_t s = check_rows(in->k, in->k_stride, p.batch, p.tokens, p.heads_k, p.dim, p.dtype, "k", x.k, x.wide,
                                         spans))
        return s;
    if (fftsplit_status_t s = check_rows(in->v, in->v_stride, p.batch, p.tokens, p.heads_k, p.dim_v, p.dtype, "v", x.v,
                                         x.wide, spans))
        return s;
    if (fftsplit_status_t s = check_device_ptr(in->log_decay, "log_decay", 4)) return s;
    spans.add(in->log_decay, size_t(p.heads_k) * 4, "log_decay");
    if (reinterpret_cast<uintptr_t>(in->lengths) % 4)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "lengths is not 4-byte aligned");
    spans.add(in->lengths, size_t(p.batch) * 4, "lengths");
    if (in->state)
        if (fftsplit_status_t s = check_device_ptr(in->state, "state", 16)) return s;
    return FFTSPLIT_SUCCESS;
}

// What all scans of a call share; the caller sets their rows, widths and factors.
LinearScan scan_of(fftsplit_linear_attention_plan_t plan, const fftsplit_linear_attention_inputs_t* in, int pass) {
    const fftsplit_linear_attention_problem_t& p = plan->prob;
    LinearScan a{};
    a.log_decay = in->log_decay;
    a.lengths = in->lengths;
    a.n = p.batch;
    a.s = p.tokens;
    a.hk = p.heads_k;
    a.segments = plan->segments[pass];
    a.segment_tokens = plan->segment_tokens[pass];
    return a;
}

LinearJoin join_of(const LinearScan& a, float* parts, const float* init, int reverse, int elements) {
    LinearJoin j{};
    j.parts = parts;
    j.init = init;
    j.log_decay = a.log_decay;
    j.lengths = a.lengths;
    j.heads = a.n * a.hk;
    j.hk = a.hk;
    j.s = a.s;
    j.segments = a.segments;
    j.segment_tokens = a.segment_tokens;
    j.reverse = reverse;
    j.elements = elements;
    return j;
}

// The states that a scan starts its segments from: `p` [head][segment][dim][dim_v],
// with rows along dim (or, turned, along dim_v).
void start_from(LinearScan& a, const float* p, int segments, int dim, int dim_v, bool turned) {
    a.init = p;
    a.init_segment = (long long)dim * dim_v;
    a.init_head = a.init_segment * segments;
    a.init_row = turned ? 1 : dim_v;
    a.init_column = turned ? dim_v : 1;
}

}  // namespace

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_linear_attention_plan(const fftsplit_linear_attention_problem_t* prob, int device,
                                                                 fftsplit_linear_attention_plan_t* out) {
    return guarded([&] {
        if (device < 0) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "device ordinal must be >= 0");
        return build(prob, device, nullptr, out);
    });
}

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_linear_attention_plan_for_arch(const fftsplit_linear_attention_problem_t* prob,
                                                                          const char* arch,
                                                                          fftsplit_linear_attention_plan_t* out) {
    return guarded([&] {
        if (!arch) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "architecture string must be non-NULL");
        return build(prob, -1, arch, out);
    });
}

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_linear_attention_plan_info(fftsplit_linear_attention_plan_t plan,
                                                                      fftsplit_linear_attention_info_t* out) {
    return guarded([&] {
        if (!plan || !out) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "plan and output must be non-NULL");
        fftsplit_linear_attention_info_t i{};
        i.forward_workspace_bytes = plan->forward_ws;
        i.backward_workspace_bytes = plan->backward_ws;
        i.state_bytes = state_bytes(plan->prob);
        i.recurrent = plan->recurrent;
        i.forward_segments = plan->recurrent ? 1 : plan->segments[0];
        i.backward_segments = plan->segments[1];
        *out = i;
        return FFTSPLIT_SUCCESS;
    });
}

FFTSPLIT_EXPORT void fftsplit_linear_attention_plan_destroy(fftsplit_linear_attention_plan_t plan) { delete plan; }

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_linear_attention_forward(fftsplit_linear_attention_plan_t plan,
                                                                    const fftsplit_linear_attention_inputs_t* in, void* o,
                                                                    float* state_out, void* workspace,
                                                                    size_t workspace_bytes, hipStream_t stream) {
    return guarded([&] {
        if (fftsplit_status_t s = check_plan(plan)) return s;
        const fftsplit_linear_attention_problem_t& p = plan->prob;
        Inputs x;
        Spans ins, outs;
        if (fftsplit_status_t s = check_inputs(plan, in, x, ins)) return s;
        if (fftsplit_status_t s = check_device_ptr(o, "o", 16)) return s;
        if (state_out)
            if (fftsplit_status_t s = check_device_ptr(state_out, "state_out", 16)) return s;
        if (fftsplit_status_t s = check_scratch(workspace, workspace_bytes, plan->forward_ws)) return s;
        if (in->state != state_out) ins.add(in->state, state_bytes(p), "state");
        outs.add(o, size_t(p.batch) * p.tokens * p.heads_q * p.dim_v * type_bytes(p.dtype), "o");
        outs.add(state_out, state_bytes(p), "state_out");
        outs.add(workspace, plan->forward_ws, "the workspace");
        if (fftsplit_status_t s = check_apart(ins, outs)) return s;
        DeviceGuard g(plan->device);
        if (!g.ok()) return fail(FFTSPLIT_ERROR_DEVICE, "cannot select the plan's device");
        const LaunchEvents ev = timing_events();

        if (plan->recurrent) {
            LinearTokens a{};
            a.q = x.q;
            a.k = x.k;
            a.v = x.v;
            a.o = o;
            a.state = in->state;
            a.state_out = state_out;
            a.log_decay = in->log_decay;
            a.lengths = in->lengths;
            a.n = p.batch;
            a.s = p.tokens;
            a.hq = p.heads_q;
            a.hk = p.heads_k;
            a.d = p.dim;
            a.dv = p.dim_v;
            a.scale = plan->scale;
            a.state_wide = p.dim_v % 4 == 0;
            return launched_ok(launch_linear_tokens(a, p.dtype, stream, ev), "linear attention launch");
        }

        LinearScan a = scan_of(plan, in, 0);
        a.q = x.q;
        a.k = x.k;
        a.v = x.v;
        a.wide = x.wide;
        a.o = o;
        a.o_wide = p.dim_v % 4 == 0;
        a.q_heads = p.heads_q / p.heads_k;
        a.k_heads = 1;
        a.d = p.dim;
        a.dv = p.dim_v;
        a.pair_scale = a.inter_scale = plan->scale;
        a.update_scale = 1.f;
        a.last = state_out;
        // the states before the segments, where they are more than one or the
        // only one's is shared
        const bool parts = a.segments > 1 || (a.q_heads > 1 && in->state && in->state == state_out);
        LaunchEvents first = ev, last = ev;
        if (parts) {
            first.stop = last.start = nullptr;
            LaunchEvents middle{a.segments > 1 ? nullptr : ev.start, nullptr};
            a.parts = static_cast<float*>(workspace);
            if (a.segments > 1)
                if (fftsplit_status_t s = launched_ok(launch_linear_parts(a, p.dtype, stream, first), "linear attention launch"))
                    return s;
            if (fftsplit_status_t s = launched_ok(
                    launch_linear_join(join_of(a, a.parts, in->state, 0, p.dim * p.dim_v), stream, middle),
                    "linear attention launch"))
                return s;
            start_from(a, a.parts, a.segments, p.dim, p.dim_v, false);
        } else if (in->state) {
            start_from(a, in->state, 1, p.dim, p.dim_v, false);
        }
        return launched_ok(launch_linear_scan(a, p.dtype, stream, last), "linear attention launch");
    });
}

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_linear_attention_backward(
    fftsplit_linear_attention_plan_t plan, const fftsplit_linear_attention_inputs_t* in, const void* dout,
    const long long dout_stride[3], const float* dstate_out, void* dq, void* dk, void* dv, float* dstate, void* workspace,
    size_t workspace_bytes, hipStream_t stream) {
    return guarded([&] {
        if (fftsplit_status_t s = check_plan(plan)) return s;
        const fftsplit_linear_attention_problem_t& p = plan->prob;
        const int es = type_bytes(p.dtype);
        Inputs x;
        Spans ins, outs;
        if (fftsplit_status_t s = check_inputs(plan, in, x, ins)) return s;
        if (!dout_stride) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "dout_stride is NULL");
        LinearRows g;
        if (fftsplit_status_t s = check_rows(dout, dout_stride, p.batch, p.tokens, p.heads_q, p.dim_v, p.dtype, "dout", g,
                                             x.wide, ins))
            return s;
        if (dstate_out)
            if (fftsplit_status_t s = check_device_ptr(dstate_out, "dstate_out", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(dq, "dq", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(dk, "dk", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(dv, "dv", 16)) return s;
        if (dstate)
            if (fftsplit_status_t s = check_device_ptr(dstate, "dstate", 16)) return s;
        if (fftsplit_status_t s = check_scratch(workspace, workspace_bytes, plan->backward_ws)) return s;
        ins.add(in->state, state_bytes(p), "state");
        ins.add(dstate_out, state_bytes(p), "dstate_out");
        const size_t rows = size_t(p.batch) * p.tokens;
        outs.add(dq, rows * p.heads_q * p.dim * es, "dq");
        outs.add(dk, rows * p.heads_k * p.dim * es, "dk");
        outs.add(dv, rows * p.heads_k * p.dim_v * es, "dv");
        outs.add(dstate, state_bytes(p), "dstate");
        outs.add(workspace, plan->backward_ws, "the workspace");
        if (fftsplit_status_t s = check_apart(ins, outs)) return s;
        DeviceGuard guard(plan->device);
        if (!guard.ok()) return fail(FFTSPLIT_ERROR_DEVICE, "cannot select the plan's device");
        const LaunchEvents ev = timing_events(), none;
        auto launched = [](hipError_t e) { return launched_ok(e, "linear attention gradient launch"); };

        // The forward pass's state, of (k, v), serves dq; its gradient, of (q,
        // dout) from the last token on, dk and dv.
        const int group = p.heads_q / p.heads_k;
        LinearScan a = scan_of(plan, in, 1);
        a.wide = x.wide;
        LinearScan sq = a, sk = a, sv = a;
        sq.q = g;                       // dq = scan(dout, v, k)
        sq.k = x.v;
        sq.v = x.k;
        sq.o = dq;
        sq.q_heads = group;
        sq.k_heads = 1;
        sq.pair_scale = sq.inter_scale = plan->scale;
        sq.update_scale = 1.f;
        sv.q = x.k;                     // dv = scan back(k, q, dout)
        sv.k = x.q;
        sv.v = g;
        sv.o = dv;
        sk.q = x.v;                     // dk = scan back(v, dout, q)
        sk.k = g;
        sk.v = x.q;
        sk.o = dk;
        for (LinearScan* s : {&sk, &sv}) {
            s->q_heads = 1;
            s->k_heads = group;
            s->reverse = 1;
            s->pair_scale = s->update_scale = plan->scale;
            s->inter_scale = 1.f;
        }
        sv.d = p.dim;
        sv.dv = p.dim_v;
        sq.d = sk.d = p.dim_v;
        sq.dv = sk.dv = p.dim;
        sv.o_wide = p.dim_v % 4 == 0;
        sq.o_wide = sk.o_wide = p.dim % 4 == 0;
        sv.last = dstate;
        const int segments = a.segments;
        if (segments > 1) {
            float* forward = static_cast<float*>(workspace);
            float* backward = forward + plan->backward_ws / 8;
            LinearScan pf = sv;          // the state's own parts: of (k, v), d x dv
            pf.q = LinearRows{};
            pf.k = x.k;
            pf.v = x.v;
            pf.k_heads = 1;
            pf.reverse = 0;
            pf.update_scale = 1.f;
            pf.parts = forward;
            if (fftsplit_status_t s = launched(launch_linear_parts(pf, p.dtype, stream, LaunchEvents{ev.start, nullptr}))) return s;
            LinearScan pb = sv;
            pb.parts = backward;
            if (fftsplit_status_t s = launched(launch_linear_parts(pb, p.dtype, stream, none))) return s;
            if (fftsplit_status_t s = launched(launch_linear_join(join_of(a, forward, in->state, 0, p.dim * p.dim_v), stream, none)))
                return s;
            if (fftsplit_status_t s = launched(launch_linear_join(join_of(a, backward, dstate_out, 1, p.dim * p.dim_v), stream, none)))
                return s;
            start_from(sq, forward, segments, p.dim, p.dim_v, true);
            start_from(sk, backward, segments, p.dim, p.dim_v, true);
            start_from(sv, backward, segments, p.dim, p.dim_v, false);
        } else {
            if (in->state) start_from(sq, in->state, 1, p.dim, p.dim_v, true);
            if (dstate_out) {
                start_from(sk, dstate_out, 1, p.dim, p.dim_v, true);
                start_from(sv, dstate_out, 1, p.dim, p.dim_v, false);
            }
        }
        if (fftsplit_status_t s =
                launched(launch_linear_scan(sq, p.dtype, stream, LaunchEvents{segments > 1 ? nullptr : ev.start, nullptr})))
            return s;
        if (fftsplit_status_t s = launched(launch_linear_scan(sk, p.dtype, stream, none))) return s;
        return launched(launch_linear_scan(sv, p.dtype, stream, LaunchEvents{nullptr, ev.stop}));
    });
}
