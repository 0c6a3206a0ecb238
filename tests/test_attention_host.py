"""Host-side checks of the attention block's entry points: refusals, plan
choices and struct layouts.  No kernel is launched."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2003_12621_amd as fs
from paper_2003_12621_amd import attention as at

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARCH = "gfx950:sramecc+:xnack-"


def plan(**kw):
    base = dict(batch=2, queries=50, keys=60, heads_q=4, heads_k=2, dim=64, dim_v=128, dtype=torch.bfloat16)
    base.update(kw)
    return fs.DiffAttention(arch=ARCH, **base)


def status_of(**kw):
    try:
        plan(**kw)
    except fs.FftsplitError as e:
        return e.status
    return fs.SUCCESS


def test_plan_refusals():
    assert status_of() == fs.SUCCESS
    for name in ("batch", "queries", "keys", "heads_q", "heads_k", "dim", "dim_v"):
        assert status_of(**{name: 0}) == fs.ERROR_INVALID_VALUE, name
        assert status_of(**{name: -1}) == fs.ERROR_INVALID_VALUE, name
    assert status_of(heads_k=3) == fs.ERROR_INVALID_VALUE
    assert status_of(dim=129) == fs.ERROR_NOT_SUPPORTED
    assert status_of(dim_v=257) == fs.ERROR_NOT_SUPPORTED
    assert status_of(dim=1, dim_v=256) == fs.SUCCESS
    assert status_of(scale=float("inf")) == fs.ERROR_INVALID_VALUE
    assert status_of(queries=1 << 29) == fs.ERROR_NOT_SUPPORTED
    assert status_of(batch=1 << 20, heads_q=64, heads_k=64) == fs.ERROR_NOT_SUPPORTED
    with pytest.raises(ValueError):
        plan(scale=-1.0)
    with pytest.raises(TypeError):
        plan(dtype=torch.float16)
    with pytest.raises(fs.FftsplitError) as e:
        fs.DiffAttention(2, 5, 5, 1, 1, 8, 8, arch="gfx942")
    assert e.value.status == fs.ERROR_ARCH


def test_problem_fields_are_checked():
    L = fs.lib()
    h = ctypes.c_void_p()
    for field, value, status in (("dtype", 2, fs.ERROR_NOT_SUPPORTED), ("causal", 2, fs.ERROR_INVALID_VALUE),
                                 ("scale", -1.0, fs.ERROR_INVALID_VALUE), ("scale", float("nan"), fs.ERROR_INVALID_VALUE)):
        p = at.AttentionProblem(1, 4, 4, 1, 1, 8, 8, 0, 0, 0.0)
        setattr(p, field, value)
        assert L.fftsplit_attention_plan_for_arch(ctypes.byref(p), b"gfx950", ctypes.byref(h)) == status, field
    p = at.AttentionProblem(1, 4, 4, 1, 1, 8, 8, 0, 0, 0.0)
    assert L.fftsplit_attention_plan_for_arch(None, b"gfx950", ctypes.byref(h)) == fs.ERROR_INVALID_VALUE
    assert L.fftsplit_attention_plan_for_arch(ctypes.byref(p), None, ctypes.byref(h)) == fs.ERROR_INVALID_VALUE
    assert L.fftsplit_attention_plan_info(None, ctypes.byref(at.AttentionInfo())) == fs.ERROR_INVALID_VALUE
    L.fftsplit_attention_plan_destroy(None)


def test_arch_only_plan_cannot_run():
    p = plan()
    fake = 1 << 20
    x = at.AttentionInputs(fake, fake, fake, fake)
    assert fs.lib().fftsplit_attention_forward(p._h, ctypes.byref(x), fake, None, None, None, None, 0,
                                               None) == fs.ERROR_INVALID_VALUE
    assert "architecture name only" in fs.last_error()


def test_kernel_choice():
    """Single tokens over a long cache share their keys among workgroups; many
    rows do not.  The workspace holds what is shared."""
    one = plan(batch=16, queries=1, keys=8192, heads_q=16, heads_k=4).info
    assert one.key_splits == 4 and one.forward_workspace_bytes >= 16 * 16 * 4 * (2 * 128 + 4) * 4
    many = plan(batch=8, queries=784, keys=784, heads_q=8, heads_k=8).info
    assert many.key_splits == 0 and many.forward_workspace_bytes == 0
    assert (many.tile_dim, many.tile_dim_v) == (64, 128)
    small = plan(dim=24, dim_v=40).info
    assert (small.tile_dim, small.tile_dim_v) == (32, 64)
    wide = plan(dim=24, dim_v=140).info
    assert (wide.tile_dim, wide.tile_dim_v) == (128, 256)
    assert many.lse_bytes == 8 * 8 * 2 * 784 * 4
    assert many.backward_workspace_bytes >= many.lse_bytes


def norm(**kw):
    base = dict(batch=2, positions=9, channels=16, x_dtype=0, y_dtype=0, x_layout=0, y_layout=0, eps=1e-5)
    base.update(kw)
    return at.LayerNorm(**base)


def norm_status(x=1 << 20, y=1 << 24, desc=None, **kw):
    d = norm(**kw) if desc is None else desc
    return fs.lib().fftsplit_layer_norm(ctypes.byref(d), x, None, None, y, None, None, None)


def test_layer_norm_refusals():
    for name in ("batch", "positions", "channels"):
        assert norm_status(**{name: 0}) == fs.ERROR_INVALID_VALUE
    assert norm_status(x_dtype=1, y_dtype=0) == fs.ERROR_NOT_SUPPORTED
    assert norm_status(x_dtype=2) == fs.ERROR_NOT_SUPPORTED
    assert norm_status(x_layout=0, y_layout=1) == fs.ERROR_NOT_SUPPORTED
    assert norm_status(x_layout=5) == fs.ERROR_INVALID_VALUE
    assert norm_status(channels=8193) == fs.ERROR_NOT_SUPPORTED
    assert norm_status(channels=2049, x_layout=1, y_layout=1) == fs.ERROR_NOT_SUPPORTED
    assert norm_status(positions=(1 << 22) + 1, x_layout=1, y_layout=1) == fs.ERROR_NOT_SUPPORTED
    assert norm_status(batch=1 << 16, positions=1 << 16) == fs.ERROR_NOT_SUPPORTED
    assert norm_status(eps=-1.0) == fs.ERROR_INVALID_VALUE
    assert norm_status(eps=float("nan")) == fs.ERROR_INVALID_VALUE
    assert norm_status(x=None) == fs.ERROR_INVALID_VALUE
    assert norm_status(x=(1 << 20) + 4) == fs.ERROR_INVALID_VALUE              # 16-byte alignment
    assert norm_status(y=1 << 20) == fs.ERROR_INVALID_VALUE                    # in place
    assert "overlaps" in fs.last_error()
    L, d = fs.lib(), norm()
    a = [1 << (20 + i) for i in range(10)]
    # mean without rstd
    assert L.fftsplit_layer_norm(ctypes.byref(d), a[0], None, None, a[1], a[2], None, None) == fs.ERROR_INVALID_VALUE
    need = ctypes.c_size_t()
    assert L.fftsplit_layer_norm_workspace(ctypes.byref(d), ctypes.byref(need)) == fs.SUCCESS and need.value > 0
    assert L.fftsplit_layer_norm_workspace(ctypes.byref(d), None) == fs.ERROR_INVALID_VALUE
    args = lambda ws, n: L.fftsplit_layer_norm_backward(ctypes.byref(d), a[0], a[1], a[2], a[3], None, a[4], a[5], a[6],
                                                        ws, n, None)
    assert args(a[7], need.value - 1) == fs.ERROR_INSUFFICIENT_WORKSPACE
    assert args(None, need.value) == fs.ERROR_INVALID_VALUE


def rotary_status(x=1 << 20, y=1 << 24, xs=(256, 64, 32), ys=(256, 64, 32), **kw):
    base = dict(batch=2, tokens=4, dim=32, heads0=2, heads1=0, dtype=0, axes=2, sections=(8, 8), positions_per_batch=0,
                inverse=0, interleaved=0)
    base.update(kw)
    sec = (ctypes.c_int * at.ROTARY_MAX_AXES)(*base.pop("sections"))
    d = at.Rotary(sections=sec, **base)
    arr = lambda v: (ctypes.c_longlong * 3)(*v)
    return fs.lib().fftsplit_rotary(ctypes.byref(d), 1 << 28, 1 << 29, x, arr(xs), y, arr(ys), None, None, None, None, None)


def test_rotary_refusals():
    for name in ("batch", "tokens", "dim", "heads0"):
        assert rotary_status(**{name: 0}) == fs.ERROR_INVALID_VALUE, name
    assert rotary_status(dtype=3) == fs.ERROR_NOT_SUPPORTED
    assert rotary_status(axes=0) == fs.ERROR_INVALID_VALUE
    assert rotary_status(axes=5) == fs.ERROR_INVALID_VALUE
    assert rotary_status(sections=(8, 9)) == fs.ERROR_INVALID_VALUE            # more than dim / 2
    assert rotary_status(sections=(0, 0)) == fs.ERROR_INVALID_VALUE
    assert rotary_status(sections=(-1, 8)) == fs.ERROR_INVALID_VALUE
    assert rotary_status(dim=1026) == fs.ERROR_NOT_SUPPORTED
    assert rotary_status(y=None) == fs.ERROR_INVALID_VALUE
    assert rotary_status(x=(1 << 20) + 2) == fs.ERROR_INVALID_VALUE            # not a float's alignment
    assert rotary_status(y=(1 << 20) + 64) == fs.ERROR_INVALID_VALUE           # overlaps x
    assert rotary_status(y=1 << 20, ys=(512, 128, 32)) == fs.ERROR_INVALID_VALUE   # in place, other strides
    assert rotary_status(ys=(256, 32, 32)) == fs.ERROR_INVALID_VALUE           # output overlaps itself
    assert rotary_status(ys=(256, 64, -32)) == fs.ERROR_INVALID_VALUE
    assert rotary_status(xs=(1 << 60, 64, 32)) == fs.ERROR_INVALID_VALUE
    assert rotary_status(heads1=1) == fs.ERROR_INVALID_VALUE                   # second tensor missing


@pytest.mark.skipif(not os.path.isdir("/opt/rocm/include"), reason="no HIP headers")
def test_struct_layouts_match_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = {"fftsplit_attention_problem_t": at.AttentionProblem, "fftsplit_attention_info_t": at.AttentionInfo,
               "fftsplit_attention_inputs_t": at.AttentionInputs, "fftsplit_layer_norm_t": at.LayerNorm,
               "fftsplit_rotary_t": at.Rotary}
    lines = []
    for cname, cls in structs.items():
        lines.append(f'printf("%zu\\n", sizeof({cname}));')
        lines += [f'printf("%zu\\n", offsetof({cname}, {f}));' for f, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"fftsplit.h\"\nint main(void) {\n"
                   + "\n".join(lines) + "\nreturn 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run([cc, "-x", "c", "-std=c11", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                    "-D__HIP_PLATFORM_AMD__", str(src), "-o", str(exe)], check=True, capture_output=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for cls in structs.values():
        want.append(ctypes.sizeof(cls))
        want += [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want


def test_reference_against_automatic_differentiation():
    """The tests' 64-bit reference: its gradients are those that torch derives
    from the formula."""
    from attention_reference import make_inputs, reference
    n, sq, sk, hq, hk, d, dv = 2, 5, 7, 4, 2, 6, 8
    arrays = make_inputs(0, n, sq, sk, hq, hk, d, dv)
    lengths = [7, 3]
    o, *grads = reference(*arrays[:4], lengths=lengths, causal=True, do=arrays[4])
    q, k, v, lam = (torch.from_numpy(a).double().requires_grad_() for a in arrays[:4])
    kk, vv = k.repeat_interleave(hq // hk, 2), v.repeat_interleave(hq // hk, 2)
    s = torch.einsum("bihmd,bjhmd->bhmij", q, kk) * d ** -0.5
    i, j = torch.arange(sq)[:, None], torch.arange(sk)[None]
    L = torch.tensor(lengths)[:, None, None]
    seen = (j < L) & (j <= i + L - sq)
    p = torch.where(seen[:, None, None], s, torch.tensor(-1e30, dtype=torch.float64)).softmax(-1)
    p = p * seen.any(-1)[:, None, None, :, None]
    want = torch.einsum("bhij,bjhe->bihe", p[:, :, 0] - lam[:, None, None] * p[:, :, 1], vv)
    assert torch.allclose(want, torch.from_numpy(o), atol=1e-12)
    for g, w in zip(grads, torch.autograd.grad(want, (q, k, v, lam), torch.from_numpy(arrays[4]).double())):
        assert torch.allclose(w, torch.from_numpy(g), atol=1e-12)
