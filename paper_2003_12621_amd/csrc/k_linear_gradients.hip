// The gradients of linear attention in one launch: dq and dk are the sums of rows as
// wide as v with values as wide as q, dv the other way round.  Side by side, the
// workgroups of one fill what those of the other leave idle.  Measured against two
// launches (us): training of 2 x 1999 tokens of 8 heads (4) of 128 / 256 in bf16 50 -> 40,
// of 6 x 301 tokens of 6 heads (3) of 32 / 64 in fp32 45 -> 25, of 4 x 3136 tokens of 8
// heads of 64 / 128 in bf16 78 -> 65.  (Aligned tensors; k_linear.hip has the rest.)
#include "linear_pass.hpp"

namespace fftsplit {

namespace {

struct Gradients {
    LinearPass pass[3];              // dq, dk, dv
    int end[2];                      // workgroups up to and including dq, and dk
};

}  // namespace

// DIM, DIM_V: what the widths of q and k, and of v, are padded to.
template <typename T, int DIM, int DIM_V>
struct GradientShape {
    static constexpr int kColumns = linear_columns(DIM), kColumnsV = linear_columns(DIM_V);
    using Rows = PassShape<T, DIM_V, kColumns>;          // of dq and dk
    using Values = PassShape<T, DIM, kColumnsV>;         // of dv
    static constexpr int kOccupancy =
        Rows::kPassOccupancy < Values::kPassOccupancy ? Rows::kPassOccupancy : Values::kPassOccupancy;
    static constexpr int kLds = (Rows::kLds > Values::kLds ? Rows::kLds : Values::kLds) + kDiagonalBytes;
    static_assert(kOccupancy * kLds <= kLinearLds, "the workgroups aimed at fit");
};

template <typename T, int DIM, int DIM_V>
__global__ __launch_bounds__(64 * kPassWaves, (GradientShape<T, DIM, DIM_V>::kOccupancy))
void linear_gradients_kernel(Gradients g) {
    using Shape = GradientShape<T, DIM, DIM_V>;
    const int id = blockIdx.x, which = id < g.end[0] ? 0 : id < g.end[1] ? 1 : 2;
    const int first = which ? g.end[which - 1] : 0, end = which < 2 ? g.end[which] : int(gridDim.x);
    if constexpr (DIM == DIM_V) {
        linear_pass<T, DIM, Shape::kColumns, true>(g.pass[which], id - first, end - first);
    } else if (which < 2) {
        linear_pass<T, DIM_V, Shape::kColumns, true>(g.pass[which], id - first, end - first);
    } else {
        linear_pass<T, DIM, Shape::kColumnsV, true>(g.pass[2], id - first, end - first);
    }
}

namespace {

template <typename T, int DIM, int DIM_V>
hipError_t launch_shaped(const LinearPass (&p)[3], hipStream_t s, const LaunchEvents& ev) {
    using Shape = GradientShape<T, DIM, DIM_V>;
    const long long q = pass_blocks(p[0], Shape::kColumns), k = pass_blocks(p[1], Shape::kColumns);
    const Gradients g{{p[0], p[1], p[2]}, {int(q), int(q + k)}};
    auto kernel = linear_gradients_kernel<T, DIM, DIM_V>;
    if (hipError_t e = allow_dynamic_lds(kernel, Shape::kLds)) return e;
    return launch_kernel(kernel, dim3(unsigned(q + k + pass_blocks(p[2], Shape::kColumnsV))), dim3(64 * kPassWaves), Shape::kLds,
                         s, ev.start, ev.stop, g);
}

template <typename T, int DIM>
hipError_t launch_dim(const LinearPass (&p)[3], hipStream_t s, const LaunchEvents& ev) {
    switch (linear_padded(p[0].d)) {
        case 32: return launch_shaped<T, DIM, 32>(p, s, ev);
        case 64: return launch_shaped<T, DIM, 64>(p, s, ev);
        case 128: return launch_shaped<T, DIM, 128>(p, s, ev);
        default: return launch_shaped<T, DIM, 256>(p, s, ev);
    }
}

template <typename T>
hipError_t launch_typed(const LinearPass (&p)[3], hipStream_t s, const LaunchEvents& ev) {
    switch (linear_padded(p[0].dv)) {
        case 32: return launch_dim<T, 32>(p, s, ev);
        case 64: return launch_dim<T, 64>(p, s, ev);
        case 128: return launch_dim<T, 128>(p, s, ev);
        default: return launch_dim<T, 256>(p, s, ev);
    }
}

}  // namespace

hipError_t launch_linear_gradients(const LinearPass& dq, const LinearPass& dk, const LinearPass& dv, int dtype, hipStream_t s,
                                   const LaunchEvents& ev) {
    const LinearPass p[3] = {dq, dk, dv};
    return dtype == FFTSPLIT_BF16 ? launch_typed<__bf16>(p, s, ev) : launch_typed<float>(p, s, ev);
}

}  // namespace fftsplit
