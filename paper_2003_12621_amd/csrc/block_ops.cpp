// Layer norm, rotary positions and head norms: argument checks and launches.
#include <cmath>

#include "entry_checks.hpp"
#include "head_norm.hpp"
#include "launch_util.hpp"
#include "norm.hpp"
#include "rotary.hpp"

using namespace fftsplit;

namespace {

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

fftsplit_status_t check_norm(const fftsplit_layer_norm_t* d, NormArgs& a) {
    if (!d) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "layer norm: description is NULL");
    if (d->batch <= 0 || d->positions <= 0 || d->channels <= 0)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "layer norm: all dimensions must be positive");
    if (!known_type(d->x_dtype) || !known_type(d->y_dtype) || (d->x_dtype == FFTSPLIT_BF16 && d->y_dtype == FFTSPLIT_F32))
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "layer norm: x and y fp32 or bf16, y not wider than x");
    if ((d->x_layout != FFTSPLIT_CHANNELS_LAST && d->x_layout != FFTSPLIT_CHANNELS_FIRST) ||
        (d->y_layout != FFTSPLIT_CHANNELS_LAST && d->y_layout != FFTSPLIT_CHANNELS_FIRST))
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "layer norm: unknown layout");
    if (d->x_layout == FFTSPLIT_CHANNELS_LAST && d->y_layout == FFTSPLIT_CHANNELS_FIRST)
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "layer norm: from tokens to a map is not supported");
    const bool first = d->x_layout == FFTSPLIT_CHANNELS_FIRST;
    if (d->channels > (first ? kNormMaxFirst : kNormMaxLast))
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "layer norm: at most 8192 channels, 2048 with channels first");
    if (!(d->eps >= 0.f) || !std::isfinite(d->eps))
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "layer norm: eps must be finite and not negative");
    // a grid holds below 2^32 threads: channels first, 8 positions or more a workgroup of up to 1024 threads
    const long long rows = (long long)d->batch * d->positions;
    if (first ? (long long)d->batch * ((d->positions + 15) / 16) >= (1 << 21) : rows * (d->channels > 1024 ? 256 : 64) > 0x7fffffffLL)
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "layer norm: too many positions");
    if (first && d->positions > (1 << 22))
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "layer norm: at most 2^22 positions of a feature map");
    a.n = d->batch;
    a.s = d->positions;
    a.c = d->channels;
    a.x_type = d->x_dtype;
    a.y_type = d->y_dtype;
    a.x_first = first;
    a.y_first = d->y_layout == FFTSPLIT_CHANNELS_FIRST;
    a.eps = d->eps;
    a.blocks = norm_backward_blocks(a.n, a.s, first);
    return FFTSPLIT_SUCCESS;
}

size_t elements(const NormArgs& a) { return size_t(a.n) * a.s * a.c; }
size_t part_bytes(const NormArgs& a) { return size_t(a.blocks) * 2 * a.c * 4; }
// Whether rows are whole 16-byte pieces of 8 elements (channels last), or four
// positions can be accessed at once (channels first; of fp32 tensors always).
// A map's bf16 output beside an fp32 input is written in fours, too.
bool norm_wide(const NormArgs& a) {
    if (a.x_first) return a.s % 4 == 0 || (a.x_type == FFTSPLIT_F32 && (a.y_type == FFTSPLIT_F32 || !a.y_first));
    return a.c % 8 == 0 && aligned16(a.weight) && aligned16(a.bias);
}

}  // namespace

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_layer_norm(const fftsplit_layer_norm_t* desc, const void* x,
                                                      const float* weight, const float* bias, void* y, float* mean,
                                                      float* rstd, hipStream_t stream) {
    return guarded([&] {
        NormArgs a{};
        if (fftsplit_status_t s = check_norm(desc, a)) return s;
        if (fftsplit_status_t s = check_device_ptr(x, "x", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(y, "y", 16)) return s;
        if (!mean != !rstd) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "mean and rstd must both be given or both be NULL");
        const size_t rows = size_t(a.n) * a.s;
        Spans in, out;
        in.add(x, elements(a) * type_bytes(a.x_type), "x");
        if (weight) {
            if (fftsplit_status_t s = check_device_ptr(weight, "weight", 4)) return s;
            in.add(weight, size_t(a.c) * 4, "weight");
        }
        if (bias) {
            if (fftsplit_status_t s = check_device_ptr(bias, "bias", 4)) return s;
            in.add(bias, size_t(a.c) * 4, "bias");
        }
        out.add(y, elements(a) * type_bytes(a.y_type), "y");
        if (mean) {
            if (fftsplit_status_t s = check_device_ptr(mean, "mean", 4)) return s;
            if (fftsplit_status_t s = check_device_ptr(rstd, "rstd", 4)) return s;
            out.add(mean, rows * 4, "mean");
            out.add(rstd, rows * 4, "rstd");
        }
        if (fftsplit_status_t s = check_apart(in, out)) return s;
        a.x = x;
        a.y = y;
        a.weight = weight;
        a.bias = bias;
        a.mean = mean;
        a.rstd = rstd;
        a.wide = norm_wide(a);
        return launched_ok(launch_norm_forward(a, stream, timing_events()), "layer norm launch");
    });
}

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_layer_norm_workspace(const fftsplit_layer_norm_t* desc, size_t* bytes) {
    return guarded([&] {
        NormArgs a{};
        if (!bytes) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "bytes is NULL");
        if (fftsplit_status_t s = check_norm(desc, a)) return s;
        *bytes = part_bytes(a);
        return FFTSPLIT_SUCCESS;
    });
}

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_layer_norm_backward(const fftsplit_layer_norm_t* desc, const void* dy,
                                                               const void* x, const float* mean, const float* rstd,
                                                               const float* weight, void* dx, float* dweight,
                                                               float* dbias, void* workspace, size_t workspace_bytes,
                                                               hipStream_t stream) {
    return guarded([&] {
        NormArgs a{};
        if (fftsplit_status_t s = check_norm(desc, a)) return s;
        if (fftsplit_status_t s = check_device_ptr(dy, "dy", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(x, "x", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(mean, "mean", 4)) return s;
        if (fftsplit_status_t s = check_device_ptr(rstd, "rstd", 4)) return s;
        if (fftsplit_status_t s = check_device_ptr(dx, "dx", 16)) return s;
        if (fftsplit_status_t s = check_device_ptr(dweight, "dweight", 4)) return s;
        if (fftsplit_status_t s = check_device_ptr(dbias, "dbias", 4)) return s;
        if (fftsplit_status_t s = check_scratch(workspace, workspace_bytes, part_bytes(a))) return s;
        const size_t rows = size_t(a.n) * a.s;
        Spans in, out;
        in.add(dy, elements(a) * type_bytes(a.y_type), "dy");
        in.add(x, elements(a) * type_bytes(a.x_type), "x");
        in.add(mean, rows * 4, "mean");
        in.add(rstd, rows * 4, "rstd");
        if (weight) {
            if (fftsplit_status_t s = check_device_ptr(weight, "weight", 4)) return s;
            in.add(weight, size_t(a.c) * 4, "weight");
        }
        out.add(dx, elements(a) * type_bytes(a.x_type), "dx");
        out.add(dweight, size_t(a.c) * 4, "dweight");
        out.add(dbias, size_t(a.c) * 4, "dbias");
        out.add(workspace, part_bytes(a), "the workspace");
        if (fftsplit_status_t s = check_apart(in, out)) return s;
        a.dy = dy;
        a.x = x;
        a.mean = const_cast<float*>(mean);
        a.rstd = const_cast<float*>(rstd);
        a.weight = weight;
        a.dx = dx;
        a.dweight = dweight;
        a.dbias = dbias;
        a.part = static_cast<float*>(workspace);
        a.wide = norm_wide(a);
        return launched_ok(launch_norm_backward(a, stream, timing_events()), "layer norm gradient launch");
    });
}

namespace {

// A [batch][tokens][heads][dim] tensor of the rotation, in bytes.
struct Heads {
    const char* name;
    uintptr_t p;
    size_t count[3], stride[3];   // batch, token, head
    size_t row, span;             // from a head's first byte to its last, from the tensor's
};

// Bytes that a tensor takes up modulo `period`, from its first on: dimensions
// that step by whole periods add none.
size_t extent_modulo(const Heads& a, size_t period) {
    size_t bytes = a.row;
    for (int i = 0; i < 3; ++i)
        if (a.stride[i] % period) bytes += (a.count[i] - 1) * a.stride[i];
    return bytes;
}

// Whether two tensors share no byte: apart as a whole, or side by side modulo
// one of their strides, as slices of one tensor are (in every token, in every
// head, ...).
bool apart(const Heads& a, const Heads& b) {
    if (a.p + a.span <= b.p || b.p + b.span <= a.p) return true;
    for (const Heads* x : {&a, &b})
        for (int i = 0; i < 3; ++i) {
            const size_t t = x->stride[i];
            if (x->count[i] == 1 || t == 0) continue;
            const size_t delta = b.p >= a.p ? (b.p - a.p) % t : (t - (a.p - b.p) % t) % t;
            if (delta >= extent_modulo(a, t) && delta + extent_modulo(b, t) <= t) return true;
        }
    return false;
}

// Checks the address and strides of a tensor of the rotation, and describes it.
fftsplit_status_t describe_heads(const fftsplit_rotary_t* d, int heads, const char* name, const void* p,
                                 const long long* strides, Heads& h) {
    const int es = type_bytes(d->dtype), dims[3] = {d->batch, d->tokens, heads};
    if (fftsplit_status_t s = check_device_ptr(p, name, es)) return s;
    h.name = name;
    h.p = reinterpret_cast<uintptr_t>(p);
    h.row = h.span = size_t(d->dim) * es;
    for (int i = 0; i < 3; ++i) {
        if (strides[i] < 0 || (dims[i] > 1 && size_t(strides[i]) > (size_t(1) << 58) / size_t(dims[i])))
            return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(name) + " has a stride out of range");
        // (the stride of a dimension of one does not matter)
        h.count[i] = size_t(dims[i]);
        h.stride[i] = dims[i] > 1 ? size_t(strides[i]) * es : 0;
        h.span += (h.count[i] - 1) * h.stride[i];
    }
    return FFTSPLIT_SUCCESS;
}

// Checks one tensor pair of the rotation and describes its two tensors.
fftsplit_status_t check_rotary_tensor(const fftsplit_rotary_t* d, int which, const void* x, const long long* xs, void* y,
                                      const long long* ys, RotaryArgs& a, Heads* desc) {
    const char* names[2] = {which ? "x1" : "x0", which ? "y1" : "y0"};
    const int per = 16 / type_bytes(d->dtype);
    const int dims[3] = {d->batch, d->tokens, a.heads[which]};
    if (fftsplit_status_t s = check_device_ptr(x, names[0], type_bytes(d->dtype))) return s;
    if (fftsplit_status_t s = check_device_ptr(y, names[1], type_bytes(d->dtype))) return s;
    if (!xs || !ys) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "rotary: strides are NULL");
    for (int t = 0; t < 2; ++t) {
        const long long* st = t ? ys : xs;
        if (fftsplit_status_t s = describe_heads(d, a.heads[which], names[t], t ? y : x, st, desc[2 * which + t])) return s;
        for (int i = 0; i < 3; ++i) {
            a.wide = a.wide && (dims[i] == 1 || st[i] % per == 0);
            (t ? a.ys : a.xs)[which][i] = st[i];
            if (dims[i] > 1 && x == y && xs[i] != ys[i])
                return fail(FFTSPLIT_ERROR_INVALID_VALUE, "rotary: in place needs equal strides");
        }
    }
    // no two elements of the output coincide: each dimension steps over the smaller ones
    long long order[3] = {0, 1, 2};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j)
            if (ys[order[j]] > ys[order[j + 1]]) {
                const long long o = order[j];
                order[j] = order[j + 1];
                order[j + 1] = o;
            }
    long long filled = d->dim;
    for (int i = 0; i < 3; ++i)
        if (dims[order[i]] > 1) {
            if (ys[order[i]] < filled)
                return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(names[1]) + " overlaps itself");
            filled += (dims[order[i]] - 1) * ys[order[i]];
        }
    a.x[which] = x;
    a.y[which] = y;
    a.wide = a.wide && aligned16(x) && aligned16(y);
    if (x != y) a.copy_rest = a.copy_rest || 2 * a.pairs < d->dim;
    return FFTSPLIT_SUCCESS;
}

// Checks the description of a rotation.
fftsplit_status_t check_rotation(const fftsplit_rotary_t* d, RotaryArgs& a) {
    if (!d) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "rotary: description is NULL");
    if (d->batch <= 0 || d->tokens <= 0 || d->heads0 <= 0 || d->heads1 < 0 || d->dim <= 0)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "rotary: all dimensions must be positive");
    if (!known_type(d->dtype)) return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "rotary: fp32 and bf16 only");
    if (d->axes < 1 || d->axes > FFTSPLIT_ROTARY_MAX_AXES)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "rotary: 1 to 4 axes");
    long long pairs = 0;
    for (int i = 0; i < d->axes; ++i) {
        if (d->sections[i] < 0) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "rotary: a section is negative");
        pairs += d->sections[i];
        a.section_end[i] = int(pairs < 0x7fffffff ? pairs : 0x7fffffff);
    }
    if (pairs < 1 || 2 * pairs > d->dim)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "rotary: the sections must hold 1 to dim / 2 pairs");
    if (d->dim > 1024 || d->heads0 > 65536 || d->heads1 > 65536 ||
        (long long)d->batch * d->tokens > (1 << 26))
        return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "rotary: dim at most 1024, 65536 heads, 2^26 tokens");
    a.n = d->batch;
    a.s = d->tokens;
    a.d = d->dim;
    a.pairs = int(pairs);
    a.axes = d->axes;
    a.pos_batch = d->positions_per_batch ? (long long)d->tokens * d->axes : 0;
    a.inverse = d->inverse != 0;
    a.interleaved = d->interleaved != 0;
    a.dtype = d->dtype;
    a.heads[0] = d->heads0;
    a.heads[1] = d->heads1;
    const int per = 16 / type_bytes(d->dtype);
    a.wide = d->dim % per == 0 && (a.interleaved ? 2 * a.pairs % per == 0 : a.pairs % per == 0);
    // Eight tokens share a workgroup's sines where that leaves four
    // workgroups a compute unit, fewer tokens in smaller calls (196 tokens:
    // 3.9 us with one, 5.9 with eight; 65536: 139 us with one, 135 with eight).
    const long long tokens = (long long)a.n * a.s;
    a.block_tokens = int(tokens / 1024 < 1 ? 1 : (tokens / 1024 > 8 ? 8 : tokens / 1024));
    return FFTSPLIT_SUCCESS;
}

// Checks its tables.
fftsplit_status_t check_tables(const fftsplit_rotary_t* d, const int* positions, const float* freqs, RotaryArgs& a,
                               Spans& tables) {
    if (fftsplit_status_t s = check_device_ptr(positions, "positions", 4)) return s;
    if (fftsplit_status_t s = check_device_ptr(freqs, "freqs", 4)) return s;
    a.positions = positions;
    a.freqs = freqs;
    tables.add(positions, size_t(d->positions_per_batch ? d->batch : 1) * d->tokens * d->axes * 4, "positions");
    tables.add(freqs, size_t(a.pairs) * 4, "freqs");
    return FFTSPLIT_SUCCESS;
}

// No output shares an element with another tensor (but with the one at `pair`
// less than its own place, in place) or a byte with a dense buffer.
fftsplit_status_t check_heads_apart(const Heads* desc, int tensors, int step, int pair, const Spans& dense) {
    for (int i = step - 1; i < tensors; i += step) {
        for (int j = 0; j < tensors; ++j) {
            const bool in_place = j == i - pair && desc[i].p == desc[j].p;
            if (j != i && !in_place && !apart(desc[i], desc[j]))
                return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(desc[i].name) + " overlaps " + desc[j].name);
        }
        for (int j = 0; j < dense.count; ++j)
            if (desc[i].p < reinterpret_cast<uintptr_t>(dense.p[j]) + dense.n[j] &&
                reinterpret_cast<uintptr_t>(dense.p[j]) < desc[i].p + desc[i].span)
                return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(desc[i].name) + " overlaps " + dense.name[j]);
    }
    return FFTSPLIT_SUCCESS;
}

}  // namespace

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_rotary(const fftsplit_rotary_t* d, const int* positions, const float* freqs,
                                                  const void* x0, const long long x0_stride[3], void* y0,
                                                  const long long y0_stride[3], const void* x1,
                                                  const long long x1_stride[3], void* y1,
                                                  const long long y1_stride[3], hipStream_t stream) {
    return guarded([&] {
        RotaryArgs a{};
        Spans tables;
        if (fftsplit_status_t s = check_rotation(d, a)) return s;
        if (fftsplit_status_t s = check_tables(d, positions, freqs, a, tables)) return s;
        Heads desc[4];
        if (fftsplit_status_t s = check_rotary_tensor(d, 0, x0, x0_stride, y0, y0_stride, a, desc)) return s;
        if (d->heads1)
            if (fftsplit_status_t s = check_rotary_tensor(d, 1, x1, x1_stride, y1, y1_stride, a, desc)) return s;
        if (fftsplit_status_t s = check_heads_apart(desc, d->heads1 ? 4 : 2, 2, 1, tables)) return s;
        return launched_ok(launch_rotary(a, stream, timing_events()), "rotary launch");
    });
}

namespace {

fftsplit_status_t check_head_norm(const fftsplit_head_norm_t* d, HeadNormArgs& a) {
    if (!d) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "head norm: description is NULL");
    if (fftsplit_status_t s = check_rotation(&d->rotary, a.r)) return s;
    if (d->rotary.inverse) return fail(FFTSPLIT_ERROR_NOT_SUPPORTED, "head norm: only rotated forwards");
    if (!(d->eps >= 0.f) || !std::isfinite(d->eps))
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, "head norm: eps must be finite and not negative");
    a.eps = d->eps;
    a.access = 16 / type_bytes(d->rotary.dtype);
    const long long groups = ((long long)a.r.n * a.r.s + a.r.block_tokens - 1) / a.r.block_tokens;
    // (each with the same number of token groups, or one less)
    const long long rounds = (groups + kHeadNormBlocks - 1) / kHeadNormBlocks;
    a.blocks = int((groups + rounds - 1) / rounds);
    return FFTSPLIT_SUCCESS;
}

size_t part_bytes(const HeadNormArgs& a) { return size_t(a.blocks) * 2 * a.r.d * 4; }

// Narrows the accesses to what a tensor's address and strides allow.
void fit_access(HeadNormArgs& a, const void* p, const long long* strides, int heads) {
    const int es = type_bytes(a.r.dtype), dims[3] = {a.r.n, a.r.s, heads};
    while (a.access > 1) {
        bool ok = reinterpret_cast<uintptr_t>(p) % size_t(a.access * es) == 0;
        for (int i = 0; i < 3; ++i) ok = ok && (dims[i] == 1 || strides[i] % a.access == 0);
        if (ok) return;
        a.access /= 2;
    }
}

// Deals a head out to lanes once the accesses are known.
void share_heads(HeadNormArgs& a) {
    const RotaryArgs& r = a.r;
    while (a.access > 1 && (r.d % a.access || (r.interleaved ? 2 * r.pairs : r.pairs) % a.access)) a.access /= 2;
    const int n = a.access;
    const int turned = r.interleaved && n > 1 ? (2 * r.pairs / n + 1) / 2 : r.pairs / n;
    const int pieces = turned + (r.d - 2 * r.pairs + 2 * n - 1) / (2 * n);
    a.row_lanes = 0;
    for (int lanes = 1; lanes <= 64 && !a.row_lanes; lanes *= 2)
        if (pieces <= lanes) a.row_lanes = lanes;
}

}  // namespace

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_head_norm_rotary(const fftsplit_head_norm_t* d, const int* positions,
                                                            const float* freqs, const fftsplit_head_norm_tensor_t* t0,
                                                            const fftsplit_head_norm_tensor_t* t1, hipStream_t stream) {
    return guarded([&] {
        HeadNormArgs a{};
        Spans dense;
        if (fftsplit_status_t s = check_head_norm(d, a)) return s;
        if (fftsplit_status_t s = check_tables(&d->rotary, positions, freqs, a.r, dense)) return s;
        const int tensors = d->rotary.heads1 ? 2 : 1;
        const fftsplit_head_norm_tensor_t* t[2] = {t0, t1};
        Heads desc[4];
        for (int i = 0; i < tensors; ++i) {
            if (!t[i]) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "head norm: a tensor is NULL");
            if (fftsplit_status_t s = check_rotary_tensor(&d->rotary, i, t[i]->x, t[i]->x_stride, t[i]->y, t[i]->y_stride,
                                                          a.r, desc))
                return s;
            if (t[i]->weight) {
                if (fftsplit_status_t s = check_device_ptr(t[i]->weight, i ? "weight of x1" : "weight of x0", 4)) return s;
                dense.add(t[i]->weight, size_t(a.r.d) * 4, i ? "weight of x1" : "weight of x0");
            }
            a.weight[i] = t[i]->weight;
            fit_access(a, t[i]->x, t[i]->x_stride, a.r.heads[i]);
            fit_access(a, t[i]->y, t[i]->y_stride, a.r.heads[i]);
        }
        if (fftsplit_status_t s = check_heads_apart(desc, 2 * tensors, 2, 1, dense)) return s;
        share_heads(a);
        return launched_ok(launch_head_norm(a, stream, timing_events()), "head norm launch");
    });
}

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_head_norm_rotary_workspace(const fftsplit_head_norm_t* d, size_t* bytes) {
    return guarded([&] {
        HeadNormArgs a{};
        if (!bytes) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "bytes is NULL");
        if (fftsplit_status_t s = check_head_norm(d, a)) return s;
        *bytes = part_bytes(a);
        return FFTSPLIT_SUCCESS;
    });
}

FFTSPLIT_EXPORT fftsplit_status_t fftsplit_head_norm_rotary_backward(const fftsplit_head_norm_t* d, const int* positions,
                                                                     const float* freqs,
                                                                     const fftsplit_head_norm_gradient_t* t0,
                                                                     const fftsplit_head_norm_gradient_t* t1,
                                                                     void* workspace, size_t workspace_bytes,
                                                                     hipStream_t stream) {
    return guarded([&] {
        HeadNormArgs a{};
        Spans dense, outs;
        if (fftsplit_status_t s = check_head_norm(d, a)) return s;
        if (fftsplit_status_t s = check_tables(&d->rotary, positions, freqs, a.r, dense)) return s;
        const int tensors = d->rotary.heads1 ? 2 : 1;
        const fftsplit_head_norm_gradient_t* t[2] = {t0, t1};
        Heads desc[6];      // of each: x, dy, dx
        size_t need = 0;
        for (int i = 0; i < tensors; ++i) {
            if (!t[i]) return fail(FFTSPLIT_ERROR_INVALID_VALUE, "head norm: a tensor is NULL");
            const int heads = a.r.heads[i];
            Heads pair[4];
            if (fftsplit_status_t s = describe_heads(&d->rotary, heads, i ? "x1" : "x0", t[i]->x, t[i]->x_stride, desc[3 * i]))
                return s;
            if (fftsplit_status_t s = check_rotary_tensor(&d->rotary, i, t[i]->dy, t[i]->dy_stride, t[i]->dx,
                                                          t[i]->dx_stride, a.r, pair))
                return s;
            desc[3 * i + 1] = pair[2 * i];
            desc[3 * i + 1].name = i ? "dy1" : "dy0";
            desc[3 * i + 2] = pair[2 * i + 1];
            desc[3 * i + 2].name = i ? "dx1" : "dx0";
            a.x[i] = t[i]->x;
            for (int j = 0; j < 3; ++j) a.xs[i][j] = t[i]->x_stride[j];
            if (t[i]->weight) {
                if (fftsplit_status_t s = check_device_ptr(t[i]->weight, i ? "weight of x1" : "weight of x0", 4)) return s;
                dense.add(t[i]->weight, size_t(a.r.d) * 4, i ? "weight of x1" : "weight of x0");
            }
            a.weight[i] = t[i]->weight;
            if (t[i]->dweight) {
                if (fftsplit_status_t s = check_device_ptr(t[i]->dweight, i ? "dweight1" : "dweight0", 4)) return s;
                outs.add(t[i]->dweight, size_t(a.r.d) * 4, i ? "dweight1" : "dweight0");
                need = part_bytes(a);
            }
            a.dweight[i] = t[i]->dweight;
            fit_access(a, t[i]->x, t[i]->x_stride, heads);
            fit_access(a, t[i]->dy, t[i]->dy_stride, heads);
            fit_access(a, t[i]->dx, t[i]->dx_stride, heads);
        }
        if (fftsplit_status_t s = check_scratch(workspace, workspace_bytes, need)) return s;
        outs.add(workspace, need, "the workspace");
        if (fftsplit_status_t s = check_apart(dense, outs)) return s;
        // the dense outputs count as buffers that no tensor may touch
        for (int j = 0; j < outs.count; ++j) {
            for (int i = 0; i < 3 * tensors; ++i)
                if (desc[i].p < reinterpret_cast<uintptr_t>(outs.p[j]) + outs.n[j] &&
                    reinterpret_cast<uintptr_t>(outs.p[j]) < desc[i].p + desc[i].span)
                    return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(outs.name[j]) + " overlaps " + desc[i].name);
        }
        if (fftsplit_status_t s = check_heads_apart(desc, 3 * tensors, 3, 1, dense)) return s;
        a.part = static_cast<float*>(workspace);
        share_heads(a);
        return launched_ok(launch_head_norm_backward(a, stream, timing_events()), "head norm gradient launch");
    });
}
