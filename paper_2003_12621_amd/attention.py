"""Operators of the attention block over a convolution's feature map.

    import paper_2003_12621_amd as fs
    plan = fs.DiffAttention(n, tokens, tokens, heads, heads, dim, dim_v, dtype=torch.bfloat16)
    o = plan.forward(q, k, v, lam)

Argument marshalling only, as in the rest of the binding: the computation runs
in the HIP kernels behind fftsplit.h.
"""
from __future__ import annotations

import ctypes
import functools
from typing import Optional

import paper_2003_12621_amd as _fs

F32, BF16 = 0, 1
CHANNELS_LAST, CHANNELS_FIRST = 0, 1
ROTARY_MAX_AXES = 4


class AttentionProblem(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int) for f in ("batch", "queries", "keys", "heads_q", "heads_k", "dim", "dim_v", "dtype",
                                            "causal")] + [("scale", ctypes.c_float)]


class AttentionInfo(ctypes.Structure):
    _fields_ = [("forward_workspace_bytes", ctypes.c_size_t), ("backward_workspace_bytes", ctypes.c_size_t),
                ("lse_bytes", ctypes.c_size_t), ("tile_dim", ctypes.c_int), ("tile_dim_v", ctypes.c_int),
                ("key_splits", ctypes.c_int)]


class AttentionInputs(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("lam", ctypes.c_void_p),
                ("key_lengths", ctypes.c_void_p), ("q_stride", ctypes.c_longlong * 4),
                ("k_stride", ctypes.c_longlong * 4), ("v_stride", ctypes.c_longlong * 3), ("lam_dtype", ctypes.c_int),
                ("lam_count", ctypes.c_int)]


class LayerNorm(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int) for f in ("batch", "positions", "channels", "x_dtype", "y_dtype", "x_layout",
                                            "y_layout")] + [("eps", ctypes.c_float)]


class Rotary(ctypes.Structure):
    _fields_ = ([(f, ctypes.c_int) for f in ("batch", "tokens", "dim", "heads0", "heads1", "dtype", "axes")]
                + [("sections", ctypes.c_int * ROTARY_MAX_AXES)]
                + [(f, ctypes.c_int) for f in ("positions_per_batch", "inverse", "interleaved")])


class HeadNorm(ctypes.Structure):
    _fields_ = [("rotary", Rotary), ("eps", ctypes.c_float)]


class HeadNormTensor(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("x_stride", ctypes.c_longlong * 3),
                ("y_stride", ctypes.c_longlong * 3), ("weight", ctypes.c_void_p)]


class HeadNormGradient(ctypes.Structure):
    _fields_ = [("dy", ctypes.c_void_p), ("x", ctypes.c_void_p), ("dx", ctypes.c_void_p),
                ("dy_stride", ctypes.c_longlong * 3), ("x_stride", ctypes.c_longlong * 3),
                ("dx_stride", ctypes.c_longlong * 3), ("weight", ctypes.c_void_p), ("dweight", ctypes.c_void_p)]


_P, _SZ = ctypes.c_void_p, ctypes.c_size_t
_STRIDES = ctypes.POINTER(ctypes.c_longlong)
SIGNATURES = {
    "fftsplit_attention_plan": (ctypes.c_int, [ctypes.POINTER(AttentionProblem), ctypes.c_int, ctypes.POINTER(_P)]),
    "fftsplit_attention_plan_for_arch": (ctypes.c_int, [ctypes.POINTER(AttentionProblem), ctypes.c_char_p,
                                                        ctypes.POINTER(_P)]),
    "fftsplit_attention_plan_info": (ctypes.c_int, [_P, ctypes.POINTER(AttentionInfo)]),
    "fftsplit_attention_plan_destroy": (None, [_P]),
    "fftsplit_attention_forward": (ctypes.c_int, [_P, ctypes.POINTER(AttentionInputs), _P, _P, _P, _P, _P, _SZ, _P]),
    "fftsplit_attention_backward": (ctypes.c_int, [_P, ctypes.POINTER(AttentionInputs), _P,
                                                   ctypes.POINTER(ctypes.c_longlong), _P, _P, _P, _P, _P, _P, _P, _P,
                                                   _SZ, _P]),
    "fftsplit_layer_norm": (ctypes.c_int, [ctypes.POINTER(LayerNorm), _P, _P, _P, _P, _P, _P, _P]),
    "fftsplit_layer_norm_workspace": (ctypes.c_int, [ctypes.POINTER(LayerNorm), ctypes.POINTER(_SZ)]),
    "fftsplit_layer_norm_backward": (ctypes.c_int, [ctypes.POINTER(LayerNorm), _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                                    _SZ, _P]),
    "fftsplit_rotary": (ctypes.c_int, [ctypes.POINTER(Rotary), _P, _P, _P, _STRIDES, _P, _STRIDES, _P, _STRIDES, _P,
                                       _STRIDES, _P]),
    "fftsplit_head_norm_rotary": (ctypes.c_int, [ctypes.POINTER(HeadNorm), _P, _P, ctypes.POINTER(HeadNormTensor),
                                                 ctypes.POINTER(HeadNormTensor), _P]),
    "fftsplit_head_norm_rotary_workspace": (ctypes.c_int, [ctypes.POINTER(HeadNorm), ctypes.POINTER(_SZ)]),
    "fftsplit_head_norm_rotary_backward": (ctypes.c_int, [ctypes.POINTER(HeadNorm), _P, _P,
                                                          ctypes.POINTER(HeadNormGradient),
                                                          ctypes.POINTER(HeadNormGradient), _P, _SZ, _P]),
}


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        _torch_module = _fs._torch()
    return _torch_module


def _type_code(dtype) -> int:
    torch = _torch()
    if dtype == torch.float32:
        return F32
    if dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"dtype must be torch.float32 or torch.bfloat16, got {dtype}")


def _stream(device) -> int:
    """Handle of the device's current stream."""
    return _torch()._C._cuda_getCurrentRawStream(device.index)


def _tensor(t, name, dtype, device):
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) torch tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")


def _strided(t, name, dtype, shape, device):
    """Pointer of a tensor of the given shape whose last dimension is dense."""
    _tensor(t, name, dtype, device)
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
    if shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} must be dense in its last dimension")
    return t.data_ptr()


def _dense(t, name, dtype, numel, device):
    """Pointer of a dense tensor of `numel` elements (any shape)."""
    _tensor(t, name, dtype, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    return t.data_ptr()


class DiffAttention:
    """Differential attention of `batch` sequences: `queries` query rows over
    room for `keys` keys, `heads_q` query heads sharing `heads_k` key heads,
    widths `dim` (one map's queries and keys) and `dim_v` (values).  See
    fftsplit.h for the formula, masks and limits."""

    def __init__(self, batch, queries, keys, heads_q, heads_k, dim, dim_v, dtype=None, causal=False, scale=None,
                 device=None, arch: Optional[str] = None):
        torch = _torch()
        self.dtype = torch.float32 if dtype is None else dtype
        if scale is not None and not scale > 0:
            raise ValueError("scale must be positive")
        self.prob = AttentionProblem(batch, queries, keys, heads_q, heads_k, dim, dim_v, _type_code(self.dtype),
                                     int(bool(causal)), 0.0 if scale is None else float(scale))
        handle = ctypes.c_void_p()
        if arch is not None:
            _fs._check(_fs.lib().fftsplit_attention_plan_for_arch(ctypes.byref(self.prob), arch.encode(),
                                                                  ctypes.byref(handle)),
                       "fftsplit_attention_plan_for_arch")
            self.device = None
        else:
            dev = torch.device("cuda", torch.cuda.current_device() if device is None else int(device))
            _fs._check(_fs.lib().fftsplit_attention_plan(ctypes.byref(self.prob), dev.index, ctypes.byref(handle)),
                       "fftsplit_attention_plan")
            self.device = dev
        self._h = handle
        self.info = AttentionInfo()
        _fs._check(_fs.lib().fftsplit_attention_plan_info(self._h, ctypes.byref(self.info)),
                   "fftsplit_attention_plan_info")
        self.q_shape = (batch, queries, heads_q, 2, dim)
        self.k_shape = (batch, keys, heads_k, 2, dim)
        self.v_shape = (batch, keys, heads_k, dim_v)
        self.out_shape = (batch, queries, heads_q, dim_v)
        self._layouts = {}

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _fs._lib is not None:
            _fs._lib.fftsplit_attention_plan_destroy(h)
            self._h = None

    def new_workspace(self, backward=False):
        """Scratch for forward, or for forward and backward.  One workspace
        serves one call at a time."""
        need = self.info.forward_workspace_bytes
        if backward:
            need = max(need, self.info.backward_workspace_bytes)
        return _torch().empty(need, dtype=_torch().uint8, device=self.device)

    def _layout(self, q, k, v, lam):
        """AttentionInputs for these strides, without pointers: the same for
        all calls with tensors laid out alike."""
        key = (q.stride(), k.stride(), v.stride(), lam.dtype, lam.numel())
        x = self._layouts.get(key)
        if x is None:
            if lam.numel() not in (1, self.prob.heads_q):
                raise ValueError(f"lam must have 1 or {self.prob.heads_q} elements, has {lam.numel()}")
            x = AttentionInputs()
            x.q_stride[:] = q.stride()[:4]
            x.k_stride[:] = k.stride()[:4]
            x.v_stride[:] = v.stride()[:3]
            x.lam_dtype, x.lam_count = _type_code(lam.dtype), lam.numel()
            if len(self._layouts) >= 64:
                self._layouts.clear()
            self._layouts[key] = x
        return AttentionInputs.from_buffer_copy(x)

    def _inputs(self, q, k, v, lam, key_lengths):
        dev = self.device
        qp = _strided(q, "q", self.dtype, self.q_shape, dev)
        kp = _strided(k, "k", self.dtype, self.k_shape, dev)
        vp = _strided(v, "v", self.dtype, self.v_shape, dev)
        lp = _dense(lam, "lam", None, None, dev)
        x = self._layout(q, k, v, lam)
        x.q, x.k, x.v, x.lam = qp, kp, vp, lp
        if key_lengths is not None:
            x.key_lengths = _dense(key_lengths, "key_lengths", _torch().int32, self.prob.batch, dev)
        return x

    def _workspace(self, ws, need):
        torch = _torch()
        if ws is None:
            if need == 0:
                return None, 0
            ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return _dense(ws, "workspace", None, None, self.device), ws.numel() * ws.element_size()

    def forward(self, q, k, v, lam, key_lengths=None, out=None, workspace=None, save=False):
        """o [batch, queries, heads_q, dim_v]; with save=True (o, saved), where
        `saved` is what backward needs beside the inputs and o."""
        torch = _torch()
        x = self._inputs(q, k, v, lam, key_lengths)
        numel = _fs._prod(self.out_shape)
        o = torch.empty(self.out_shape, dtype=self.dtype, device=self.device) if out is None else out
        op = _dense(o, "out", self.dtype, numel, self.device)
        saved = None
        sp = (None, None, None)
        if save:
            saved = (torch.empty_like(o, dtype=torch.float32), torch.empty_like(o, dtype=torch.float32),
                     torch.empty(self.info.lse_bytes // 4, dtype=torch.float32, device=self.device))
            sp = tuple(t.data_ptr() for t in saved)
        ws, nbytes = self._workspace(workspace, self.info.forward_workspace_bytes)
        _fs._check(_fs.lib().fftsplit_attention_forward(self._h, ctypes.byref(x), op, *sp, ws, nbytes,
                                                        _stream(self.device)),
                   "fftsplit_attention_forward")
        return (o, saved) if save else o

    def backward(self, dout, q, k, v, lam, saved, key_lengths=None, workspace=None):
        """(dq, dk, dv, dlam) from the gradient of o; `saved` as
        forward(save=True) returned it."""
        torch, dev = _torch(), self.device
        x = self._inputs(q, k, v, lam, key_lengths)
        gp = _strided(dout, "dout", self.dtype, self.out_shape, dev)
        gs = (ctypes.c_longlong * 3)(*dout.stride()[:3])
        numel = _fs._prod(self.out_shape)
        o1 = _dense(saved[0], "saved[0]", torch.float32, numel, dev)
        o2 = _dense(saved[1], "saved[1]", torch.float32, numel, dev)
        lse = _dense(saved[2], "saved[2]", torch.float32, self.info.lse_bytes // 4, dev)
        dq = torch.empty(self.q_shape, dtype=self.dtype, device=dev)
        dk = torch.empty(self.k_shape, dtype=self.dtype, device=dev)
        dv = torch.empty(self.v_shape, dtype=self.dtype, device=dev)
        dlam = torch.empty_like(lam)
        ws, nbytes = self._workspace(workspace, self.info.backward_workspace_bytes)
        _fs._check(_fs.lib().fftsplit_attention_backward(self._h, ctypes.byref(x), gp, gs, o1, o2, lse, dq.data_ptr(),
                                                         dk.data_ptr(), dv.data_ptr(), dlam.data_ptr(), ws, nbytes,
                                                         _stream(dev)),
                   "fftsplit_attention_backward")
        return dq, dk, dv, dlam


_LAYOUTS = {"last": CHANNELS_LAST, "first": CHANNELS_FIRST}


def _device_of(t, name):
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) torch tensor")
    return t.device


def _launch(device, name, *args):
    """Calls an entry point that runs on the current device on `device`'s
    current stream."""
    torch = _torch()
    fn = getattr(_fs.lib(), name)
    if torch._C._cuda_getDevice() == device.index:
        status = fn(*args, _stream(device))
    else:
        with torch.cuda.device(device):
            status = fn(*args, _stream(device))
    if status != _fs.SUCCESS:
        _fs._check(status, name)


@functools.lru_cache(maxsize=256)
def _norm_desc(shape, dtype, layout, out_layout, out_dtype, eps):
    """The description of a call, the output's shape and the bytes of the
    backward pass's workspace, which depend on shapes and types alone."""
    out_layout = layout if out_layout is None else out_layout
    if layout not in _LAYOUTS or out_layout not in _LAYOUTS:
        raise ValueError("layout must be 'last' or 'first'")
    if len(shape) < 2:
        raise ValueError("layer_norm needs at least two dimensions")
    if layout == "first":
        n, c, s = shape[0], shape[1], _fs._prod(shape[2:])
        out_shape = tuple(shape) if out_layout == "first" else (n, s, c)
    else:
        n, s, c = 1, _fs._prod(shape[:-1]), shape[-1]
        out_shape = tuple(shape)
    desc = LayerNorm(n, s, c, _type_code(dtype), _type_code(out_dtype), _LAYOUTS[layout], _LAYOUTS[out_layout], eps)
    need = ctypes.c_size_t()
    _fs._check(_fs.lib().fftsplit_layer_norm_workspace(ctypes.byref(desc), ctypes.byref(need)),
               "fftsplit_layer_norm_workspace")
    return desc, out_shape, _fs._prod(out_shape), need.value


def _param(t, name, c, device):
    return None if t is None else _dense(t, name, _torch().float32, c, device)


def layer_norm(x, weight=None, bias=None, eps=1e-5, layout="last", out_layout=None, out_dtype=None, out=None,
               return_stats=False):
    """Layer norm over the channels: of tokens [..., channels] (layout "last")
    or of feature maps [n, channels, ...] ("first").  out_layout="last" turns
    a feature map into tokens [n, positions, channels], out_dtype an fp32 one
    into bf16.  return_stats=True also returns mean and rstd (fp32, one per
    position) for layer_norm_backward."""
    torch, dev = _torch(), _device_of(x, "x")
    out_dtype = x.dtype if out_dtype is None else out_dtype
    desc, shape, numel, _ = _norm_desc(x.shape, x.dtype, layout, out_layout, out_dtype, eps)
    xp = _dense(x, "x", None, None, dev)
    wp, bp = _param(weight, "weight", desc.channels, dev), _param(bias, "bias", desc.channels, dev)
    y = torch.empty(shape, dtype=out_dtype, device=dev) if out is None else out
    yp = _dense(y, "out", out_dtype, numel, dev)
    mean = rstd = None
    if return_stats:
        mean, rstd = torch.empty((2, desc.batch * desc.positions), dtype=torch.float32, device=dev)
    _launch(dev, "fftsplit_layer_norm", ctypes.byref(desc), xp, wp, bp, yp,
            mean.data_ptr() if return_stats else None, rstd.data_ptr() if return_stats else None)
    return (y, mean, rstd) if return_stats else y


def layer_norm_backward(dy, x, mean, rstd, weight=None, layout="last", out_layout=None, workspace=None):
    """(dx, dweight, dbias) from the gradient of layer_norm's output; the
    parameters' gradients are fp32."""
    torch, dev = _torch(), _device_of(x, "x")
    _device_of(dy, "dy")
    desc, _, numel, need = _norm_desc(x.shape, x.dtype, layout, out_layout, dy.dtype, 0.0)
    rows = desc.batch * desc.positions
    gp = _dense(dy, "dy", dy.dtype, numel, dev)
    xp = _dense(x, "x", None, None, dev)
    mp, rp = _dense(mean, "mean", torch.float32, rows, dev), _dense(rstd, "rstd", torch.float32, rows, dev)
    wp = _param(weight, "weight", desc.channels, dev)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if workspace is None else workspace
    dx = torch.empty_like(x)
    dweight, dbias = torch.empty((2, desc.channels), dtype=torch.float32, device=dev)
    _launch(dev, "fftsplit_layer_norm_backward", ctypes.byref(desc), gp, xp, mp, rp, wp, dx.data_ptr(),
            dweight.data_ptr(), dbias.data_ptr(), _dense(ws, "workspace", None, None, dev),
            ws.numel() * ws.element_size())
    return dx, dweight, dbias


def _heads_view(shape, strides, name):
    """[batch, tokens, heads, dim] strides of a [batch, tokens, ..., dim] tensor."""
    if shape[-1] > 1 and strides[-1] != 1:
        raise ValueError(f"{name} must be dense in its last dimension")
    heads, stride = 1, 0
    for size, st in zip(reversed(shape[2:-1]), reversed(strides[2:-1])):
        if size == 1:
            continue
        if heads == 1:
            stride = st
        elif st != stride * heads:
            raise ValueError(f"{name}: its head dimensions do not form one")
        heads *= size
    return heads, (ctypes.c_longlong * 3)(strides[0], strides[1], stride)


def _like(t, name, shaped, typed):
    if t.dtype != typed.dtype or t.device != typed.device or t.shape != shaped.shape:
        raise ValueError(f"{name} must be a {typed.dtype} tensor of shape {tuple(shaped.shape)} on {typed.device}")


@functools.lru_cache(maxsize=256)
def _rotary_desc(shape, other_shape, strides, dtype, pos_shape, sections, interleaved, inverse):
    """The description and strides of a call, which depend on shapes alone.
    `strides`: of x, its output, other, its output (None without other)."""
    if len(shape) < 4:
        raise ValueError("x must be [batch, tokens, heads, dim], heads possibly in several dimensions")
    n, s, d = shape[0], shape[1], shape[-1]
    axes = len(sections)
    if not 1 <= axes <= ROTARY_MAX_AXES:
        raise ValueError(f"sections must name 1 to {ROTARY_MAX_AXES} axes")
    if pos_shape not in ((s, axes), (n, s, axes)):
        raise ValueError(f"positions has shape {pos_shape}, expected [{s}, {axes}] or [{n}, {s}, {axes}]")
    if other_shape is not None and (len(other_shape) < 4 or other_shape[:2] != (n, s) or other_shape[-1] != d):
        raise ValueError(f"other has shape {tuple(other_shape)}, expected [{n}, {s}, heads, {d}]")
    heads, views = [0, 0], []
    for i, st in enumerate(strides):
        name = ("x", "output of x", "other", "output of other")[i]
        if st is None:
            views.append(None)
            continue
        heads[i // 2], view = _heads_view(other_shape if i >= 2 else shape, st, name)
        views.append(view)
    return Rotary(n, s, d, heads[0], heads[1], _type_code(dtype), axes, (ctypes.c_int * ROTARY_MAX_AXES)(*sections),
                  int(len(pos_shape) == 3), int(inverse), int(interleaved)), views


def rotary(x, positions, freqs, sections, other=None, interleaved=False, inverse=False, out=None, out_other=None):
    """Turns the pairs of every head of x [batch, tokens, heads, dim] (heads
    possibly in several dimensions) by its token's positions times freqs;
    `sections` counts the pairs of each axis of `positions` ([tokens, axes] or
    [batch, tokens, axes], int32).  `other` is turned in the same launch (the
    keys beside the queries); then both results are returned.  out=x works in
    place; inverse=True gives the gradient."""
    torch, dev = _torch(), _device_of(x, "x")
    if other is None and out_other is not None:
        raise ValueError("out_other given without other")
    sections = tuple(sections)
    out = torch.empty(x.shape, dtype=x.dtype, device=dev) if out is None else out
    _like(out, "output of x", x, x)
    strides = (x.stride(), out.stride(), None, None)
    if other is not None:
        _device_of(other, "other")
        out_other = torch.empty(other.shape, dtype=other.dtype, device=dev) if out_other is None else out_other
        _like(other, "other", other, x)
        _like(out_other, "output of other", other, x)
        strides = strides[:2] + (other.stride(), out_other.stride())
    desc, v = _rotary_desc(x.shape, None if other is None else other.shape, strides, x.dtype, positions.shape,
                           sections, bool(interleaved), bool(inverse))
    pp = _dense(positions, "positions", torch.int32, None, dev)
    fp = _dense(freqs, "freqs", torch.float32, sum(sections), dev)
    _launch(dev, "fftsplit_rotary", ctypes.byref(desc), pp, fp, x.data_ptr(), v[0], out.data_ptr(), v[1],
            None if other is None else other.data_ptr(), v[2], None if other is None else out_other.data_ptr(), v[3])
    return out if other is None else (out, out_other)


@functools.lru_cache(maxsize=256)
def _head_norm_desc(shape, other_shape, strides, dtype, pos_shape, sections, interleaved, eps):
    """The description and strides of a call, and the bytes of the backward
    pass's workspace.  `strides`: of x and its companions (output, or gradient
    and output), then of other and its."""
    per = len(strides) // 2
    views, rot = [], None
    # (the rotation's description takes tensors in pairs)
    for i in range(0, per, 2):
        pair = (strides[i], strides[min(i + 1, per - 1)])
        pair += (None, None) if other_shape is None else (strides[per + i], strides[per + min(i + 1, per - 1)])
        rot, v = _rotary_desc(shape, other_shape, pair, dtype, pos_shape, sections, interleaved, False)
        views.append(v)
    first = [views[i // 2][i % 2] for i in range(per)]
    second = [views[i // 2][2 + i % 2] for i in range(per)]
    desc = HeadNorm(rot, eps)
    need = ctypes.c_size_t()
    _fs._check(_fs.lib().fftsplit_head_norm_rotary_workspace(ctypes.byref(desc), ctypes.byref(need)),
               "fftsplit_head_norm_rotary_workspace")
    return desc, first, second, need.value


def head_norm_rotary(x, weight, positions, freqs, sections, other=None, other_weight=None, eps=1e-6,
                     interleaved=False, out=None, out_other=None):
    """rotary(x / sqrt(mean(x^2) + eps) * weight) in one pass, the mean over each
    head of x [batch, tokens, heads, dim]; weight fp32 [dim] or None.  The rest
    as for rotary: `other` (the keys) is done in the same launch, with a weight
    of its own; out=x works in place."""
    torch, dev = _torch(), _device_of(x, "x")
    if other is None and (out_other is not None or other_weight is not None):
        raise ValueError("out_other or other_weight given without other")
    sections = tuple(sections)
    out = torch.empty(x.shape, dtype=x.dtype, device=dev) if out is None else out
    _like(out, "output of x", x, x)
    strides = (x.stride(), out.stride(), None, None)
    if other is not None:
        _device_of(other, "other")
        out_other = torch.empty(other.shape, dtype=other.dtype, device=dev) if out_other is None else out_other
        _like(other, "other", other, x)
        _like(out_other, "output of other", other, x)
        strides = strides[:2] + (other.stride(), out_other.stride())
    desc, v, w, _ = _head_norm_desc(x.shape, None if other is None else other.shape, strides, x.dtype, positions.shape,
                                    sections, bool(interleaved), float(eps))
    pp = _dense(positions, "positions", torch.int32, None, dev)
    fp = _dense(freqs, "freqs", torch.float32, sum(sections), dev)
    t0 = HeadNormTensor(x.data_ptr(), out.data_ptr(), v[0], v[1], _param(weight, "weight", desc.rotary.dim, dev))
    t1 = None
    if other is not None:
        t1 = ctypes.byref(HeadNormTensor(other.data_ptr(), out_other.data_ptr(), w[0], w[1],
                                         _param(other_weight, "other_weight", desc.rotary.dim, dev)))
    _launch(dev, "fftsplit_head_norm_rotary", ctypes.byref(desc), pp, fp, ctypes.byref(t0), t1)
    return out if other is None else (out, out_other)


def head_norm_rotary_backward(dy, x, weight, positions, freqs, sections, dy_other=None, other=None, other_weight=None,
                              eps=1e-6, interleaved=False, out=None, out_other=None, workspace=None):
    """(dx, dweight) from the gradient of head_norm_rotary's output, with `other`
    (dx, dweight, dother, dother_weight); the weights' gradients are fp32.
    out=dy works in place."""
    torch, dev = _torch(), _device_of(x, "x")
    _device_of(dy, "dy")
    if (other is None) != (dy_other is None):
        raise ValueError("other and dy_other must both be given or both be None")
    if other is None and (out_other is not None or other_weight is not None):
        raise ValueError("out_other or other_weight given without other")
    sections = tuple(sections)
    out = torch.empty(x.shape, dtype=x.dtype, device=dev) if out is None else out
    _like(dy, "dy", x, x)
    _like(out, "gradient of x", x, x)
    strides = (dy.stride(), out.stride(), x.stride())
    if other is not None:
        _device_of(other, "other")
        _device_of(dy_other, "dy_other")
        out_other = torch.empty(other.shape, dtype=other.dtype, device=dev) if out_other is None else out_other
        _like(other, "other", other, x)
        _like(dy_other, "dy_other", other, x)
        _like(out_other, "gradient of other", other, x)
        strides += (dy_other.stride(), out_other.stride(), other.stride())
    else:
        strides += (None, None, None)
    desc, v, w, need = _head_norm_desc(x.shape, None if other is None else other.shape, strides, x.dtype,
                                       positions.shape, sections, bool(interleaved), float(eps))
    dim = desc.rotary.dim
    pp = _dense(positions, "positions", torch.int32, None, dev)
    fp = _dense(freqs, "freqs", torch.float32, sum(sections), dev)
    dweight = torch.empty((1 if other is None else 2, dim), dtype=torch.float32, device=dev)
    t0 = HeadNormGradient(dy.data_ptr(), x.data_ptr(), out.data_ptr(), v[0], v[2], v[1],
                          _param(weight, "weight", dim, dev), dweight.data_ptr())
    t1 = None
    if other is not None:
        t1 = ctypes.byref(HeadNormGradient(dy_other.data_ptr(), other.data_ptr(), out_other.data_ptr(), w[0], w[2], w[1],
                                           _param(other_weight, "other_weight", dim, dev),
                                           dweight.data_ptr() + 4 * dim))
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if workspace is None else workspace
    _launch(dev, "fftsplit_head_norm_rotary_backward", ctypes.byref(desc), pp, fp, ctypes.byref(t0), t1,
            _dense(ws, "workspace", None, None, dev), ws.numel() * ws.element_size())
    return (out, dweight[0]) if other is None else (out, dweight[0], out_other, dweight[1])
