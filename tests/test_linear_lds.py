"""Host check of the LDS that the passes of linear attention take: as many
workgroups of every shape as their launch bounds aim at have to fit a compute
unit, the gradients' as well, which share one launch."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2003_12621_amd", "csrc")
HIPCC = "/opt/rocm/bin/hipcc"
LDS = 160 * 1024

SRC = r"""
#include <cstdio>
#include "linear_pass.hpp"
using namespace fftsplit;

template <typename T, int D, int COLUMNS>
void print() {
    using Shape = PassShape<T, D, COLUMNS>;
    std::printf("%d %d %d %d %d\n", int(sizeof(T)), D, COLUMNS, Shape::kPassOccupancy, Shape::kLds + kDiagonalBytes);
}
template <typename T, int D>
void columns() {
    print<T, D, 64>();
    print<T, D, 128>();
}
template <typename T>
void widths() {
    columns<T, 32>();
    columns<T, 64>();
    columns<T, 128>();
    columns<T, 256>();
}
int main() {
    widths<__bf16>();
    widths<float>();
}
"""


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_workgroups_fit(tmp_path):
    src = tmp_path / "lds.hip"
    src.write_text(SRC)
    exe = tmp_path / "lds"
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
                    "-packed-fp32-ops", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True, capture_output=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    shapes = {tuple(map(int, line.split()[:3])): tuple(map(int, line.split()[3:])) for line in out.splitlines()}
    assert len(shapes) == 16
    for shape, (workgroups, lds) in shapes.items():
        assert workgroups * lds <= LDS, shape
    slice_of = lambda width: 64 if width <= 64 else 128
    for size in (2, 4):
        for dim in (32, 64, 128, 256):
            for dim_v in (32, 64, 128, 256):
                pair = shapes[size, dim_v, slice_of(dim)], shapes[size, dim, slice_of(dim_v)]
                assert min(p[0] for p in pair) * max(p[1] for p in pair) <= LDS, (size, dim, dim_v)
