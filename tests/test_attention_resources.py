"""Static check of the attention kernels' registers: their waits are hidden by
other workgroups of the compute unit, and a kernel that needs more registers
than the number aimed at, or scratch, loses that silently.  (The variants for
aligned tensors, which run in the usual case.)"""
import os
import re
import shutil
import tempfile

import pytest

from test_kernel_resources import BUILD, LLVM, _metadata

BUDGETS = [
    # four workgroups of four waves per compute unit: four waves per SIMD
    ("k_attn_forward.o", r"attn_forward_kernelIDF16bLi32ELi64ELb1E", 128),
    ("k_attn_forward.o", r"attn_forward_kernelIDF16bLi64ELi128ELb1E", 128),
    ("k_attn_forward.o", r"attn_forward_kernelIfLi32ELi64ELb1E", 128),
    # two workgroups
    ("k_attn_forward.o", r"attn_forward_kernelIDF16bLi128ELi256ELb1E", 256),
    ("k_attn_forward.o", r"attn_forward_kernelIfLi64ELi128ELb1E", 256),
    ("k_attn_backward.o", r"attn_(key|query)_side_kernelIDF16bLi32ELi64ELb1E", 256),
    ("k_attn_backward.o", r"attn_(key|query)_side_kernelIDF16bLi64ELi128ELb1E", 256),
    ("k_attn_backward.o", r"attn_(key|query)_side_kernelIfLi32ELi64ELb1E", 256),
    # one: all of a lane's registers, no scratch
    ("k_attn_forward.o", r"attn_forward_kernelIfLi128ELi256ELb1E", 512),
    ("k_attn_forward.o", r"attn_few_rows_kernelI(DF16b|f)Li\d+ELi\d+ELb1E", 512),
    ("k_attn_backward.o", r"attn_(key|query)_side_kernelI(DF16b|f)Li\d+ELi\d+ELb1E", 512),
]


@pytest.mark.skipif(not os.path.isdir(BUILD) or not shutil.which(f"{LLVM}/llvm-readelf"),
                    reason="library not built here, or no LLVM tools")
def test_attention_kernels_keep_their_occupancy():
    with tempfile.TemporaryDirectory() as tmp:
        cache = {}
        for obj, pattern, budget in BUDGETS:
            if obj not in cache:
                cache[obj] = _metadata(os.path.join(BUILD, obj), tmp)
            hits = {k: v for k, v in cache[obj].items() if re.search(pattern, k)}
            assert hits, f"{pattern} not found in {obj}"
            for name, res in hits.items():
                assert res.get("spill", 0) == 0, f"{name} spills {res['spill']} registers"
                assert res.get("vgpr", 0) <= budget, f"{name}: {res.get('vgpr')} registers > {budget}"
