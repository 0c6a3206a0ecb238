"""Static check of the registers of the linear attention and head norm kernels:
their waits are hidden by other workgroups of the compute unit, and a kernel that
needs more registers than the number aimed at, or scratch, loses that silently.
(The variants for aligned tensors, which run in the usual case.)"""
import os
import re
import shutil
import tempfile

import pytest

from test_kernel_resources import BUILD, LLVM, _metadata

BUDGETS = [
    # three workgroups of four waves per compute unit: three waves per SIMD
    ("k_linear.o", r"linear_pass_kernelIDF16bLi(32|64)ELi(64|128)ELb1E", 168),
    ("k_linear.o", r"linear_pass_kernelIDF16bLi128ELi64ELb1E", 168),
    ("k_linear_gradients.o", r"linear_gradients_kernelIDF16bLi(32|64|128)ELi(32|64)E", 168),
    ("k_linear_gradients.o", r"linear_gradients_kernelIDF16bLi(32|64)ELi128E", 168),
    # two
    ("k_linear.o", r"linear_pass_kernelIDF16bLi\d+ELi\d+ELb1E", 256),
    ("k_linear.o", r"linear_pass_kernelIfLi(32|64|128)ELi\d+ELb1E", 256),
    ("k_linear.o", r"linear_parts_kernelI(DF16b|f)Li(32|64|128)ELi\dELb1E", 256),
    ("k_linear_gradients.o", r"linear_gradients_kernelIDF16bLi\d+ELi\d+E", 256),
    ("k_linear_gradients.o", r"linear_gradients_kernelIfLi(32|64|128)ELi(32|64|128)E", 256),
    # one: all of a lane's registers, no scratch
    ("k_linear.o", r"linear_(pass|parts)_kernel", 512),
    ("k_linear_gradients.o", r"linear_gradients_kernel", 512),
    # eight waves of the join, four of each of the others
    ("k_linear.o", r"linear_join_kernel", 128),
    ("k_linear_tokens.o", r"linear_tokens_kernel", 128),
    # six and four waves per SIMD
    ("k_head_norm.o", r"head_norm_kernelI(DF16bLi8|fLi4)ELb\dELb1ELb0E", 80),
    ("k_head_norm.o", r"head_norm_kernelI(DF16bLi8|fLi4)ELb\dELb1ELb1E", 128),
]
# (rows that are not aligned: one or two registers of the pass, outside its loops)
UNALIGNED = r"linear_pass_kernelIDF16bLi(32|64)ELi128ELb0E"


@pytest.mark.skipif(not os.path.isdir(BUILD) or not shutil.which(f"{LLVM}/llvm-readelf"),
                    reason="library not built here, or no LLVM tools")
def test_linear_kernels_keep_their_occupancy():
    with tempfile.TemporaryDirectory() as tmp:
        cache = {}
        for obj, pattern, budget in BUDGETS:
            if obj not in cache:
                cache[obj] = _metadata(os.path.join(BUILD, obj), tmp)
            hits = {k: v for k, v in cache[obj].items() if re.search(pattern, k)}
            assert hits, f"{pattern} not found in {obj}"
            for name, res in hits.items():
                spills = 4 if re.search(UNALIGNED, name) else 0
                assert res.get("spill", 0) <= spills, f"{name} spills {res['spill']} registers"
                assert res.get("vgpr", 0) <= budget, f"{name}: {res.get('vgpr')} registers > {budget}"
