"""Host-side checks of the head norms and of linear attention: refusals, plan
choices and struct layouts.  No kernel is launched."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2003_12621_amd as fs
from paper_2003_12621_amd import attention as at
from paper_2003_12621_amd import linear_attention as la

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARCH = "gfx950:sramecc+:xnack-"
FAKE = 1 << 30          # never dereferenced: the calls below are refused


def plan(**kw):
    base = dict(batch=2, tokens=500, heads_q=4, heads_k=2, dim=64, dim_v=128, dtype=torch.bfloat16)
    base.update(kw)
    return fs.LinearAttention(arch=ARCH, **base)


def status_of(**kw):
    try:
        plan(**kw)
    except fs.FftsplitError as e:
        return e.status
    return fs.SUCCESS


def test_plan_refusals():
    assert status_of() == fs.SUCCESS
    for name in ("batch", "tokens", "heads_q", "heads_k", "dim", "dim_v"):
        assert status_of(**{name: 0}) == fs.ERROR_INVALID_VALUE, name
        assert status_of(**{name: -1}) == fs.ERROR_INVALID_VALUE, name
    assert status_of(heads_k=3) == fs.ERROR_INVALID_VALUE
    assert status_of(dim=257) == fs.ERROR_NOT_SUPPORTED
    assert status_of(dim_v=257) == fs.ERROR_NOT_SUPPORTED
    assert status_of(dim=1, dim_v=256) == fs.SUCCESS
    assert status_of(scale=float("inf")) == fs.ERROR_INVALID_VALUE
    assert status_of(tokens=1 << 29) == fs.ERROR_NOT_SUPPORTED
    assert status_of(batch=1 << 22, tokens=1, heads_q=64, heads_k=64) == fs.ERROR_NOT_SUPPORTED
    assert status_of(batch=1 << 20, tokens=1, heads_q=1, heads_k=1, dim=256, dim_v=256) == fs.ERROR_NOT_SUPPORTED
    with pytest.raises(ValueError):
        plan(scale=-1.0)
    with pytest.raises(TypeError):
        plan(dtype=torch.float16)
    with pytest.raises(fs.FftsplitError) as e:
        fs.LinearAttention(2, 5, 1, 1, 8, 8, arch="gfx942")
    assert e.value.status == fs.ERROR_ARCH
    L, h = fs.lib(), ctypes.c_void_p()
    p = la.LinearAttentionProblem(1, 4, 1, 1, 8, 8, 2, 0.0)
    assert L.fftsplit_linear_attention_plan_for_arch(ctypes.byref(p), b"gfx950", ctypes.byref(h)) == fs.ERROR_NOT_SUPPORTED
    p = la.LinearAttentionProblem(1, 4, 1, 1, 8, 8, 0, -1.0)
    assert L.fftsplit_linear_attention_plan_for_arch(ctypes.byref(p), b"gfx950", ctypes.byref(h)) == fs.ERROR_INVALID_VALUE
    assert L.fftsplit_linear_attention_plan_for_arch(None, b"gfx950", ctypes.byref(h)) == fs.ERROR_INVALID_VALUE
    assert L.fftsplit_linear_attention_plan_info(None, ctypes.byref(la.LinearAttentionInfo())) == fs.ERROR_INVALID_VALUE
    L.fftsplit_linear_attention_plan_destroy(None)


def test_arch_only_plan_cannot_run():
    p = plan()
    x = la.LinearAttentionInputs(FAKE, FAKE, FAKE, FAKE)
    assert fs.lib().fftsplit_linear_attention_forward(p._h, ctypes.byref(x), FAKE, None, None, 0,
                                                      None) == fs.ERROR_INVALID_VALUE
    assert "architecture name only" in fs.last_error()
    assert fs.lib().fftsplit_linear_attention_backward(p._h, ctypes.byref(x), FAKE, None, None, FAKE, FAKE, FAKE, None,
                                                       None, 0, None) == fs.ERROR_INVALID_VALUE
    assert fs.lib().fftsplit_linear_attention_forward(None, ctypes.byref(x), FAKE, None, None, 0,
                                                      None) == fs.ERROR_INVALID_VALUE


def test_plan_choices():
    """Few tokens go one by one and need no workspace; longer sequences are cut
    into segments, whose states the workspace holds."""
    one = plan(tokens=1)
    assert one.info.recurrent == 1 and one.info.forward_workspace_bytes == 0
    assert one.info.state_bytes == 2 * 2 * 64 * 128 * 4
    long = plan(batch=1, tokens=8192)
    assert long.info.recurrent == 0 and long.info.segments > 8
    assert long.info.forward_workspace_bytes >= long.info.segments * long.info.state_bytes
    assert long.info.backward_workspace_bytes >= 2 * long.info.segments * long.info.state_bytes
    for tokens in (9, 33, 1000, 12345, 1 << 20, 1 << 28):
        for dtype in (torch.float32, torch.bfloat16):
            info = plan(batch=1, heads_q=1, heads_k=1, tokens=tokens, dtype=dtype).info
            assert info.segment_tokens % 128 == 0 and info.segments == -(-tokens // info.segment_tokens)


def rotary(**kw):
    f = dict(batch=1, tokens=4, dim=8, heads0=2, heads1=0, dtype=0, axes=1, sections=(4, 0, 0, 0), positions_per_batch=0,
             inverse=0, interleaved=0)
    f.update(kw)
    f["sections"] = (ctypes.c_int * 4)(*f["sections"])
    return at.Rotary(*f.values())


def forward_status(desc, t0=None, t1=None, positions=FAKE, freqs=FAKE + 4096):
    s = (ctypes.c_longlong * 3)(64, 16, 8)
    t0 = at.HeadNormTensor(FAKE + 8192, FAKE + 16384, s, s, FAKE + 24576) if t0 is None else t0
    return fs.lib().fftsplit_head_norm_rotary(ctypes.byref(desc), positions, freqs, ctypes.byref(t0),
                                              None if t1 is None else ctypes.byref(t1), None)


def test_head_norm_refusals():
    s = (ctypes.c_longlong * 3)(64, 16, 8)
    bad = fs.ERROR_INVALID_VALUE
    assert forward_status(at.HeadNorm(rotary(inverse=1), 1e-6)) == fs.ERROR_NOT_SUPPORTED
    assert forward_status(at.HeadNorm(rotary(dtype=3), 1e-6)) == fs.ERROR_NOT_SUPPORTED
    for eps in (-1.0, float("nan"), float("inf")):
        assert forward_status(at.HeadNorm(rotary(), eps)) == bad
    assert forward_status(at.HeadNorm(rotary(sections=(5, 0, 0, 0)), 1e-6)) == bad
    assert forward_status(at.HeadNorm(rotary(sections=(0, 0, 0, 0)), 1e-6)) == bad
    desc = at.HeadNorm(rotary(), 1e-6)
    assert forward_status(desc, positions=None) == bad
    assert forward_status(desc, freqs=None) == bad
    assert forward_status(desc, freqs=FAKE + 4098) == bad
    tensor = lambda x, y, xs=s, ys=s, w=None: at.HeadNormTensor(x, y, xs, ys, w)
    assert forward_status(desc, tensor(None, FAKE + 16384)) == bad
    assert forward_status(desc, tensor(FAKE + 8192, None)) == bad
    assert forward_status(desc, tensor(FAKE + 8194, FAKE + 16384)) == bad
    assert forward_status(desc, tensor(FAKE + 8192, FAKE + 16384, w=FAKE + 3)) == bad
    assert forward_status(desc, tensor(FAKE + 8192, FAKE + 8200)) == bad                       # overlap
    assert forward_status(desc, tensor(FAKE + 8192, FAKE + 8192, ys=(ctypes.c_longlong * 3)(64, 16, 16))) == bad
    assert forward_status(desc, tensor(FAKE + 8192, FAKE + 16384, ys=(ctypes.c_longlong * 3)(64, 4, 8))) == bad
    assert forward_status(desc, tensor(FAKE + 8192, FAKE + 16384, xs=(ctypes.c_longlong * 3)(64, -16, 8))) == bad
    assert forward_status(desc, tensor(FAKE + 8192, FAKE)) == bad                              # on the positions
    assert forward_status(desc, tensor(FAKE + 8192, FAKE + 16384, w=FAKE + 16384)) == bad      # weight in the output
    two = at.HeadNorm(rotary(heads1=2), 1e-6)
    assert forward_status(two) == bad                                                          # no second tensor
    assert forward_status(two, t1=tensor(FAKE + 32768, FAKE + 16384)) == bad                   # outputs overlap
    need = ctypes.c_size_t()
    L = fs.lib()
    assert L.fftsplit_head_norm_rotary_workspace(ctypes.byref(desc), None) == bad
    assert L.fftsplit_head_norm_rotary_workspace(None, ctypes.byref(need)) == bad
    assert L.fftsplit_head_norm_rotary_workspace(ctypes.byref(desc), ctypes.byref(need)) == fs.SUCCESS
    assert need.value == 4 * 2 * 8 * 4          # four tokens, each a workgroup's


def test_head_norm_gradient_refusals():
    s = (ctypes.c_longlong * 3)(64, 16, 8)
    desc, bad, L = at.HeadNorm(rotary(), 1e-6), fs.ERROR_INVALID_VALUE, fs.lib()

    def status(dy=FAKE + 8192, x=FAKE + 16384, dx=FAKE + 24576, w=None, dw=FAKE + 32768, dxs=s, ws=FAKE + 65536, n=1 << 16):
        t = at.HeadNormGradient(dy, x, dx, s, s, dxs, w, dw)
        return L.fftsplit_head_norm_rotary_backward(ctypes.byref(desc), FAKE, FAKE + 4096, ctypes.byref(t), None, ws, n, None)

    assert status(dy=None) == bad and status(x=None) == bad and status(dx=None) == bad
    assert status(dx=FAKE + 16384) == bad                    # on x
    assert status(dx=FAKE + 8200) == bad                     # across dy
    assert status(dw=FAKE + 16384) == bad                    # dweight in x
    assert status(dw=FAKE + 24576) == bad                    # in dx
    assert status(dw=FAKE + 2) == bad
    assert status(w=FAKE + 24576) == bad                     # weight in dx
    assert status(ws=None) == bad
    assert status(ws=FAKE + 24576) == bad
    assert status(n=16) == fs.ERROR_INSUFFICIENT_WORKSPACE
    assert status(dy=FAKE + 24576, dxs=(ctypes.c_longlong * 3)(64, 16, 16)) == bad   # in place, other strides


def test_binding_refuses_host_tensors():
    x = torch.zeros(1, 4, 2, 8)
    pos, freqs = torch.zeros(4, 1, dtype=torch.int32), torch.ones(4)
    with pytest.raises(TypeError):
        fs.head_norm_rotary(x, None, pos, freqs, (4,))
    with pytest.raises(TypeError):
        fs.head_norm_rotary_backward(x, x, None, pos, freqs, (4,))
    p = plan(batch=1, tokens=4, heads_q=2, heads_k=2, dim=8, dim_v=8, dtype=torch.float32)
    with pytest.raises(TypeError):
        p.forward(x, x, x, torch.zeros(2))


@pytest.mark.skipif(not shutil.which("g++") or not os.path.isdir("/opt/rocm/include"), reason="no compiler or headers")
def test_struct_layouts(tmp_path):
    structs = {"fftsplit_head_norm_t": at.HeadNorm, "fftsplit_head_norm_tensor_t": at.HeadNormTensor,
               "fftsplit_head_norm_gradient_t": at.HeadNormGradient,
               "fftsplit_linear_attention_problem_t": la.LinearAttentionProblem,
               "fftsplit_linear_attention_info_t": la.LinearAttentionInfo,
               "fftsplit_linear_attention_inputs_t": la.LinearAttentionInputs}
    lines = ["#include <stdio.h>", "#include <stddef.h>", "#define __HIP_PLATFORM_AMD__ 1", '#include "fftsplit.h"',
             "int main() {"]
    for name, cls in structs.items():
        lines.append(f'printf("{name} %zu", sizeof({name}));')
        lines += [f'printf(" %zu", offsetof({name}, {f}));' for f, _ in cls._fields_]
        lines.append('printf("\\n");')
    src = tmp_path / "layout.cpp"
    src.write_text("\n".join(lines + ["}"]))
    exe = tmp_path / "layout"
    subprocess.run(["g++", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", str(src), "-o", str(exe)],
                   check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()
    for line, (name, cls) in zip(out, structs.items()):
        want = [name, ctypes.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]
        assert line.split() == [str(w) for w in want]
