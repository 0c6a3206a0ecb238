// Argument checks shared by the entry points of the attention block.
#pragma once

#include <cstdint>
#include <string>

#include "fftsplit_internal.hpp"

namespace fftsplit {

inline int type_bytes(int dtype) { return dtype == FFTSPLIT_F32 ? 4 : 2; }
inline bool known_type(int dtype) { return dtype == FFTSPLIT_F32 || dtype == FFTSPLIT_BF16; }

inline fftsplit_status_t check_device_ptr(const void* p, const char* name, unsigned align) {
    if (!p) return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(name) + " is NULL");
    if (reinterpret_cast<uintptr_t>(p) % align)
        return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(name) + " is not " + std::to_string(align) + "-byte aligned");
    return FFTSPLIT_SUCCESS;
}

inline fftsplit_status_t check_scratch(const void* ws, size_t bytes, size_t need) {
    if (need == 0) return FFTSPLIT_SUCCESS;
    if (fftsplit_status_t s = check_device_ptr(ws, "workspace", 16)) return s;
    if (bytes < need)
        return fail(FFTSPLIT_ERROR_INSUFFICIENT_WORKSPACE,
                    "workspace has " + std::to_string(bytes) + " bytes, " + std::to_string(need) + " are needed");
    return FFTSPLIT_SUCCESS;
}

inline fftsplit_status_t launched_ok(hipError_t e, const char* what) {
    if (e != hipSuccess) return fail(FFTSPLIT_ERROR_DEVICE, std::string(what) + ": " + hipGetErrorString(e));
    return FFTSPLIT_SUCCESS;
}

// The buffers of a call.
struct Spans {
    static constexpr int kMost = 12;
    const void* p[kMost];
    size_t n[kMost];
    const char* name[kMost];
    int count = 0;
    void add(const void* ptr, size_t bytes, const char* what) {
        if (!ptr || !bytes || count == kMost) return;
        p[count] = ptr;
        n[count] = bytes;
        name[count++] = what;
    }
};

// No output overlaps an input or another output.
inline fftsplit_status_t check_apart(const Spans& in, const Spans& out) {
    auto overlap = [](const void* a, size_t an, const void* b, size_t bn) {
        const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
        return a0 < b0 + bn && b0 < a0 + an;
    };
    for (int i = 0; i < out.count; ++i) {
        for (int j = 0; j < in.count; ++j)
            if (overlap(out.p[i], out.n[i], in.p[j], in.n[j]))
                return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(out.name[i]) + " overlaps " + in.name[j]);
        for (int j = 0; j < i; ++j)
            if (overlap(out.p[i], out.n[i], out.p[j], out.n[j]))
                return fail(FFTSPLIT_ERROR_INVALID_VALUE, std::string(out.name[i]) + " overlaps " + out.name[j]);
    }
    return FFTSPLIT_SUCCESS;
}

// Runs an entry point's body; an exception (a message that found no memory)
// becomes a status.
template <typename F>
inline fftsplit_status_t guarded(F&& body) noexcept {
    try {
        set_error("");
        return body();
    } catch (...) {
        return FFTSPLIT_ERROR_INVALID_VALUE;
    }
}

}  // namespace fftsplit
