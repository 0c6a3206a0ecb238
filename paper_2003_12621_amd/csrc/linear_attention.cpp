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

// Whether 16-byte accesses of rows are aligned and whole.  Where they are not, elements pass
// through registers one by one: 8 x 784 tokens of 8 heads of 64 / 128 in bf16 off by an element
// 32 us forwards and 58 backwards, so 62 and 153; 2 x 1999 of 8 heads (4) of 128 / 256 41 and
// 76, so 77 and 195; 6 x 301 of 6 heads (3) of 32 / 64 in fp32 20 and 41, so 27 and 84.
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

// Tokens of a segment, a multiple of a workgroup's rows.  Long segments cost pairs of
// tokens, short ones states, written and read.  Measured (us of forward + backward passes,
// segments of 128 / 256 / 384) where the short segments' states take up to 16 MiB, bf16:
// 8192 tokens of 16 heads (4) of 64 / 128 50 + 80 / 56 + 101 / 62 + 122, 16384 of 32 heads (4)
// 112 + 237 / 119 + 271 / 135 + 333, 2 x 1999 tokens of 8 heads (4) of 128 / 256 42 + 79 / 49 +
// 82 / 54 + 91; and where they take more: 4 x 16384 tokens of 16 heads 493 + 1335 / 413 + 1082 /
// 409 + 1053, 4 x 3136 tokens of 8 heads 56 + 116 / 55 + 98 / 58 + 103, 2 x 4000 tokens of 16
// heads (8) of 256 220 + 568 / 173 + 450 / 183 + 446.  Products of fp32 take 16 times as long
// as those of bf16, so that pairs weigh more: 6 x 301 tokens of 6 heads (3) of 32 / 64 26 + 43 /
// 38 + 67 / 42 + 79, 4 x 3000 tokens of 8 heads of 64 93 + 195 / 115 + 248 / 120 + 250.
void choose_segments(const fftsplit_linear_attention_problem_t& p, int& tokens, int& segments) {
    const double states = double(state_bytes(p)) * ((p.tokens + kLinearRows - 1) / kLinearRows);
    tokens = p.dtype == FFTSPLIT_F32 || states <= 16 << 20 ? kLinearRows : 2 * kLinearRows;
    segments = (p.tokens + tokens - 1) / tokens;
}

// us that a wave takes for a tile of 32 rows by 32 tokens and a slice of columns (whose
// elements pass through registers one by one where accesses of 16 bytes are not aligned).
double tile_us(const fftsplit_linear_attention_problem_t& p, int width, int width_v, bool wide) {
    const int rows = linear_padded(width), columns = linear_columns(width_v);
    const double products = p.dtype == FFTSPLIT_F32 ? 0.015 * (rows + columns) : 0.25 + 0.0012 * (rows + 2 * columns);
    return products + (wide ? 0 : 0.0035 * type_bytes(p.dtype) * (rows + columns));
}

// Whether a call that returns no state takes a sequence as one segment, which saves two
// launches and the states, for pairs of all its tokens: by an estimate of both, from the
// tiles of the longest wave and of all waves of a SIMD (which hardly overlap), the states'
// bytes (written, read, and the same as operands; backwards for both sums) and what the
// first two launches cost besides.  Measured, in segments / as one (us):
//   bf16, forward, 8 heads of 64 / 128, one sequence of 300, 600, 900 tokens 21 / 12, 21 /
//   19, 22 / 26, 32 sequences 47 / 24, 70 / 55, 97 / 105; 16 heads (4) of 64, 32 sequences 38
//   / 29, 54 / 65, 75 / 127; 8 heads of 128 / 256, 8 sequences 46 / 17, 60 / 37, 76 / 73;
//   backward, 8 heads of 64 / 128, one sequence 22 / 13, 25 / 20, 28 / 27, 32 sequences of 32
//   / 32 43 / 33, 64 / 74, 91 / 158, 16 heads (4) of 64, 8 sequences 40 / 32, 47 / 65, 57 / 125;
//   fp32, 8 heads of 64 / 128, 8 sequences of 160, 300, 600 tokens: forward 41 / 21, 45 / 38,
//   66 / 99, backward 58 / 38, 82 / 77, 121 / 195; 6 heads (3) of 32 / 64 backward 37 / 30, 46 /
//   55, 53 / 112.
// The estimate's numbers are fitted to 168 such calls, of which it takes the slower way by up
// to 12 % and by 0.3 % in the mean (a bound on the tokens alone: 74 % and 2.5 %); of 48 other
// calls by up to 19 % and by 1 % in the mean.
// Rows that are not aligned, bf16, 8 heads of 64 / 128: forward, one sequence of 300, 600 tokens
// 36 / 26, 37 / 46, 8 sequences of 784 62 / 82, backward (in two launches) 58 / 60, 61 / 96, 153 /
// 209.
bool one_segment(const fftsplit_linear_attention_plan_s& plan, bool backward, bool wide) {
    const fftsplit_linear_attention_problem_t& p = plan.prob;
    if (plan.segments == 1) return true;
    const int group = p.heads_q / p.heads_k;
    double longest = 0, all = 0;            // of a wave with one tile, and of all of them with one each
    auto add = [&](int width, int width_v, int heads, int k_heads) {
        const double us = tile_us(p, width, width_v, wide) * k_heads;
        const int columns = linear_columns(width_v);
        all += us * p.batch * heads * ((width_v + columns - 1) / columns);
        return us;
    };
    if (backward) {
        const double dq = add(p.dim_v, p.dim, p.heads_q, 1), dk = add(p.dim_v, p.dim, p.heads_k, group);
        const double dv = add(p.dim, p.dim_v, p.heads_k, group), first = dq > dk ? dq : dk;
        longest = !wide ? first + dv : first > dv ? first : dv;
    } else {
        longest = add(p.dim, p.dim_v, p.heads_q, 1);
    }
    const double tiles = (p.tokens + kLinearTile - 1) / kLinearTile, own = plan.segment_tokens / kLinearTile;
    constexpr double kSimds = 1024, kBytesPerUs = 4.5e6;
    auto pairs = [&](double of) {           // rows that each see `of` tiles at most
        const double chain = longest * of, work = all / kSimds * tiles * of / 2;
        return chain > work ? chain : work;
    };
    const double states = double(state_bytes(p)) * plan.segments * (backward ? 11 : 4) / kBytesPerUs;
    const double before = p.dtype == FFTSPLIT_F32 ? 6 : 8;
    return pairs(tiles) <= pairs(tiles < own ? tiles : own) + 4 * longest + before + states;
}

int padded32(int width) { return (width + 31) / 32 * 32; }

// Bytes of the parts of the segments' states, and of the operands made of them
// (rows padded as the passes that read them pad their widths; of fp32 one operand of
// 4 bytes a value, of bf16 two of 2).
size_t parts_bytes(const fftsplit_linear_attention_problem_t& p, int segments) {
    return round256(state_bytes(p) * size_t(segments));
}
size_t starts_bytes(const fftsplit_linear_attention_problem_t& p, int segments, bool turned) {
    const size_t rows = linear_padded(turned ? p.dim_v : p.dim), columns = padded32(turned ? p.dim : p.dim_v);
    return round256(size_t(p.batch) * p.heads_k * segments * rows * columns * 4);
}

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
    choose_segments(p, plan->segment_tokens, plan->segments);
    plan->forward_ws = plan->recurrent ? 0 : parts_bytes(p, plan->segments) + starts_bytes(p, plan->segments, false);
    plan->backward_ws = 2 * parts_bytes(p, plan->segments) + starts_bytes(p, plan->segments, false) +
                        2 * starts_bytes(p, plan->segments, true);
    // workgroups of the largest launches (a dimension of a grid holds below 2^32 threads)
    const double heads_q = double(p.batch) * p.heads_q, heads_k = double(p.batch) * p.heads_k;
    auto slices = [](int width) { return (width + linear_columns(width) - 1) / linear_columns(width); };
    const int wider = slices(p.dim) > slices(p.dim_v) ? slices(p.dim) : slices(p.dim_v);
    const double groups[] = {(heads_q + 2 * heads_k) * wider * ((p.tokens + kLinearRows - 1) / kLinearRows),
                             2 * heads_k * wider * plan->segments,
                             6 * heads_k * (double(linear_padded(p.dim)) * linear_padded(p.dim_v) / 512)};
    for (double g : groups)
        if (g > double(1 << 23)) {
            delete plan;
            return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "linear attention: too many tokens and heads over all sequences");
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

// What all passes of a call share; the caller sets their rows, widths and factors.
LinearPass pass_of(fftsplit_linear_attention_plan_t plan, const fftsplit_linear_attention_inputs_t* in, int wide, bool one) {
    const fftsplit_linear_attention_problem_t& p = plan->prob;
    LinearPass a{};
    a.log_decay = in->log_decay;
    a.lengths = in->lengths;
    a.n = p.batch;
    a.s = p.tokens;
    a.hk = p.heads_k;
    a.segments = one ? 1 : plan->segments;
    a.segment_tokens = one ? (p.tokens + kLinearRows - 1) / kLinearRows * kLinearRows : plan->segment_tokens;
    a.wide = wide;
    return a;
}

// The join of the parts of `a`, of states dim x dim_v.
LinearJoin join_of(const LinearPass& a, int dim, int dim_v, bool turned, const float* init, void* starts, float* last) {
    LinearJoin j{};
    j.parts = a.parts;
    j.init = init;
    j.starts = starts;
    j.last = last;
    j.log_decay = a.log_decay;
    j.lengths = a.lengths;
    j.heads = a.n * a.hk;
    j.hk = a.hk;
    j.s = a.s;
    j.segments = a.segments;
    j.segment_tokens = a.segment_tokens;
    j.reverse = a.reverse;
    j.d = dim;
    j.dv = dim_v;
    j.turned = turned;
    j.rows = linear_padded(turned ? dim_v : dim);
    j.columns = padded32(turned ? dim : dim_v);
    j.first_part = a.first_part;
    j.part_count = a.part_count;
    return j;
}

// The launches of a call: only the first records when the call begins, and only
// the last when it ends.
struct Launches {
    LaunchEvents ev;
    LaunchEvents next(bool last) {
        const LaunchEvents e{ev.start, last ? ev.stop : nullptr};
        ev.start = nullptr;
        return e;
    }
};

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
        i.segment_tokens = plan->segment_tokens;
        i.segments = plan->segments;
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

        LinearPass a = pass_of(plan, in, x.wide, !state_out && one_segment(*plan, false, x.wide));
        a.q = x.q;
        a.k = x.k;
        a.v = x.v;
        a.o = o;
        a.o_wide = p.dim_v % 4 == 0;
        a.q_heads = p.heads_q / p.heads_k;
        a.k_heads = 1;
        a.d = p.dim;
        a.dv = p.dim_v;
        a.pair_scale = a.inter_scale = plan->scale;
        a.update_scale = 1.f;
        a.part_count = state_out ? a.segments : a.segments - 1;
        a.exact = state_out != nullptr;
        a.parts = static_cast<float*>(workspace);
        auto launched = [](hipError_t e) { return launched_ok(e, "linear attention launch"); };
        Launches launches{ev};
        if (a.part_count)
            if (fftsplit_status_t s = launched(launch_linear_parts(a, nullptr, p.dtype, stream, launches.next(false))))
                return s;
        const bool before = a.segments > 1 || in->state;
        if (before || state_out) {
            void* starts = before ? static_cast<char*>(workspace) + parts_bytes(p, a.segments) : nullptr;
            const LinearJoin j = join_of(a, p.dim, p.dim_v, false, in->state, starts, state_out);
            if (fftsplit_status_t s = launched(launch_linear_join(&j, 1, p.dtype, stream, launches.next(false)))) return s;
            a.starts = starts;
        }
        return launched(launch_linear_pass(a, nullptr, p.dtype, stream, launches.next(true)));
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
        auto launched = [](hipError_t e) { return launched_ok(e, "linear attention gradient launch"); };
        Launches launches{timing_events()};

        // The forward pass's state, of (k, v), serves dq; its gradient, of (q,
        // dout) from the last token on, dk and dv.
        const int group = p.heads_q / p.heads_k;
        const LinearPass a = pass_of(plan, in, x.wide, !dstate && one_segment(*plan, true, x.wide));
        LinearPass pq = a, pk = a, pv = a;
        pq.q = g;                       // dq: (dout, v, k)
        pq.k = x.v;
        pq.v = x.k;
        pq.o = dq;
        pq.q_heads = group;
        pq.k_heads = 1;
        pq.pair_scale = pq.inter_scale = plan->scale;
        pv.q = x.k;                     // dv: back (k, q, dout)
        pv.k = x.q;
        pv.v = g;
        pv.o = dv;
        pk.q = x.v;                     // dk: back (v, dout, q)
        pk.k = g;
        pk.v = x.q;
        pk.o = dk;
        for (LinearPass* b : {&pk, &pv}) {
            b->q_heads = 1;
            b->k_heads = group;
            b->reverse = 1;
            b->pair_scale = plan->scale;
            b->inter_scale = 1.f;
        }
        pv.d = p.dim;
        pv.dv = p.dim_v;
        pq.d = pk.d = p.dim_v;
        pq.dv = pk.dv = p.dim;
        pv.o_wide = p.dim_v % 4 == 0;
        pq.o_wide = pk.o_wide = p.dim % 4 == 0;

        const int segments = a.segments;
        char* ws = static_cast<char*>(workspace);
        LinearPass state = a, gradient = pv;      // what adds to the state, and to its gradient
        state.k = x.k;
        state.v = x.v;
        state.k_heads = 1;
        state.d = p.dim;
        state.dv = p.dim_v;
        state.update_scale = 1.f;
        state.parts = reinterpret_cast<float*>(ws);
        state.part_count = segments - 1;
        gradient.update_scale = plan->scale;
        gradient.parts = reinterpret_cast<float*>(ws + parts_bytes(p, segments));
        gradient.first_part = dstate ? 0 : 1;
        gradient.part_count = segments - gradient.first_part;
        gradient.exact = dstate != nullptr;
        ws += 2 * parts_bytes(p, segments);
        if (state.part_count) {
            if (fftsplit_status_t s = launched(launch_linear_parts(state, &gradient, p.dtype, stream, launches.next(false))))
                return s;
        } else if (gradient.part_count) {
            if (fftsplit_status_t s = launched(launch_linear_parts(gradient, nullptr, p.dtype, stream, launches.next(false))))
                return s;
        }
        LinearJoin jobs[3];
        int count = 0;
        if (segments > 1 || in->state) {
            jobs[count++] = join_of(state, p.dim, p.dim_v, true, in->state, ws, nullptr);
            pq.starts = ws;
        }
        ws += starts_bytes(p, segments, true);
        if (segments > 1 || dstate_out) {
            jobs[count++] = join_of(gradient, p.dim, p.dim_v, true, dstate_out, ws, nullptr);
            pk.starts = ws;
            pv.starts = ws + starts_bytes(p, segments, true);
        }
        ws += starts_bytes(p, segments, true);
        if (pv.starts || dstate)
            jobs[count++] = join_of(gradient, p.dim, p.dim_v, false, dstate_out, const_cast<void*>(pv.starts), dstate);
        if (count)
            if (fftsplit_status_t s = launched(launch_linear_join(jobs, count, p.dtype, stream, launches.next(false))))
                return s;
        if (x.wide) return launched(launch_linear_gradients(pq, pk, pv, p.dtype, stream, launches.next(true)));
        if (fftsplit_status_t s = launched(launch_linear_pass(pq, &pk, p.dtype, stream, launches.next(false)))) return s;
        return launched(launch_linear_pass(pv, nullptr, p.dtype, stream, launches.next(true)));
    });
}
