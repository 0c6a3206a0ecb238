"""Linear attention with a decay for each head: causal attention whose cost
grows with the tokens, not with their square, and whose memory of a sequence is
a state of fixed size.

    import paper_2003_12621_amd as fs
    plan = fs.LinearAttention(n, tokens, heads, heads, dim, dim_v, dtype=torch.bfloat16)
    o, state = plan.forward(q, k, v, log_decay, return_state=True)
    step = fs.LinearAttention(n, 1, heads, heads, dim, dim_v, dtype=torch.bfloat16)
    o1, state = step.forward(q1, k1, v1, log_decay, state=state, out_state=state)

Argument marshalling only, as in the rest of the binding: the computation runs
in the HIP kernels behind fftsplit.h.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import paper_2003_12621_amd as _fs

from .attention import _P, _SZ, _STRIDES, _dense, _stream, _strided, _torch, _type_code


class LinearAttentionProblem(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int) for f in ("batch", "tokens", "heads_q", "heads_k", "dim", "dim_v",
                                            "dtype")] + [("scale", ctypes.c_float)]


class LinearAttentionInfo(ctypes.Structure):
    _fields_ = [("forward_workspace_bytes", ctypes.c_size_t), ("backward_workspace_bytes", ctypes.c_size_t),
                ("state_bytes", ctypes.c_size_t), ("recurrent", ctypes.c_int), ("segment_tokens", ctypes.c_int),
                ("segments", ctypes.c_int)]


class LinearAttentionInputs(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("log_decay", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("state", ctypes.c_void_p), ("q_stride", ctypes.c_longlong * 3),
                ("k_stride", ctypes.c_longlong * 3), ("v_stride", ctypes.c_longlong * 3)]


SIGNATURES = {
    "fftsplit_linear_attention_plan": (ctypes.c_int, [ctypes.POINTER(LinearAttentionProblem), ctypes.c_int,
                                                      ctypes.POINTER(_P)]),
    "fftsplit_linear_attention_plan_for_arch": (ctypes.c_int, [ctypes.POINTER(LinearAttentionProblem), ctypes.c_char_p,
                                                               ctypes.POINTER(_P)]),
    "fftsplit_linear_attention_plan_info": (ctypes.c_int, [_P, ctypes.POINTER(LinearAttentionInfo)]),
    "fftsplit_linear_attention_plan_destroy": (None, [_P]),
    "fftsplit_linear_attention_forward": (ctypes.c_int, [_P, ctypes.POINTER(LinearAttentionInputs), _P, _P, _P, _SZ,
                                                         _P]),
    "fftsplit_linear_attention_backward": (ctypes.c_int, [_P, ctypes.POINTER(LinearAttentionInputs), _P, _STRIDES, _P,
                                                          _P, _P, _P, _P, _P, _SZ, _P]),
}


class LinearAttention:
    """Linear attention of `batch` sequences of up to `tokens` tokens: `heads_q`
    query heads sharing the states of `heads_k` key heads, widths `dim` (queries
    and keys) and `dim_v` (values).  See fftsplit.h for the formula and limits."""

    def __init__(self, batch, tokens, heads_q, heads_k, dim, dim_v, dtype=None, scale=None, device=None,
                 arch: Optional[str] = None):
        torch = _torch()
        self.dtype = torch.float32 if dtype is None else dtype
        if scale is not None and not scale > 0:
            raise ValueError("scale must be positive")
        self.prob = LinearAttentionProblem(batch, tokens, heads_q, heads_k, dim, dim_v, _type_code(self.dtype),
                                           0.0 if scale is None else float(scale))
        handle = ctypes.c_void_p()
        if arch is not None:
            _fs._check(_fs.lib().fftsplit_linear_attention_plan_for_arch(ctypes.byref(self.prob), arch.encode(),
                                                                         ctypes.byref(handle)),
                       "fftsplit_linear_attention_plan_for_arch")
            self.device = None
        else:
            dev = torch.device("cuda", torch.cuda.current_device() if device is None else int(device))
            _fs._check(_fs.lib().fftsplit_linear_attention_plan(ctypes.byref(self.prob), dev.index,
                                                                ctypes.byref(handle)),
                       "fftsplit_linear_attention_plan")
            self.device = dev
        self._h = handle
        self.info = LinearAttentionInfo()
        _fs._check(_fs.lib().fftsplit_linear_attention_plan_info(self._h, ctypes.byref(self.info)),
                   "fftsplit_linear_attention_plan_info")
        self.q_shape = (batch, tokens, heads_q, dim)
        self.k_shape = (batch, tokens, heads_k, dim)
        self.v_shape = (batch, tokens, heads_k, dim_v)
        self.out_shape = (batch, tokens, heads_q, dim_v)
        self.state_shape = (batch, heads_k, dim, dim_v)
        self._layouts = {}

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _fs._lib is not None:
            _fs._lib.fftsplit_linear_attention_plan_destroy(h)
            self._h = None

    def new_workspace(self, backward=False):
        """Scratch for forward, or for forward and backward.  One workspace
        serves one call at a time."""
        need = self.info.forward_workspace_bytes
        if backward:
            need = max(need, self.info.backward_workspace_bytes)
        return _torch().empty(need, dtype=_torch().uint8, device=self.device)

    def _layout(self, q, k, v):
        """LinearAttentionInputs for these strides, without pointers."""
        key = (q.stride(), k.stride(), v.stride())
        x = self._layouts.get(key)
        if x is None:
            x = LinearAttentionInputs()
            x.q_stride[:] = q.stride()[:3]
            x.k_stride[:] = k.stride()[:3]
            x.v_stride[:] = v.stride()[:3]
            if len(self._layouts) >= 64:
                self._layouts.clear()
            self._layouts[key] = x
        return LinearAttentionInputs.from_buffer_copy(x)

    def _state(self, t, name):
        return _dense(t, name, _torch().float32, self.info.state_bytes // 4, self.device)

    def _inputs(self, q, k, v, log_decay, state, lengths):
        torch, dev = _torch(), self.device
        qp = _strided(q, "q", self.dtype, self.q_shape, dev)
        kp = _strided(k, "k", self.dtype, self.k_shape, dev)
        vp = _strided(v, "v", self.dtype, self.v_shape, dev)
        x = self._layout(q, k, v)
        x.q, x.k, x.v = qp, kp, vp
        x.log_decay = _dense(log_decay, "log_decay", torch.float32, self.prob.heads_k, dev)
        if lengths is not None:
            x.lengths = _dense(lengths, "lengths", torch.int32, self.prob.batch, dev)
        if state is not None:
            x.state = self._state(state, "state")
        return x

    def _workspace(self, ws, need):
        torch = _torch()
        if ws is None:
            if need == 0:
                return None, 0
            ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return _dense(ws, "workspace", None, None, self.device), ws.numel() * ws.element_size()

    def forward(self, q, k, v, log_decay, state=None, lengths=None, out=None, out_state=None, return_state=False,
                workspace=None):
        """o [batch, tokens, heads_q, dim_v]; with return_state=True, or
        out_state given, (o, state after the last token).  out_state may be
        `state`: then it is updated in place."""
        torch = _torch()
        x = self._inputs(q, k, v, log_decay, state, lengths)
        o = torch.empty(self.out_shape, dtype=self.dtype, device=self.device) if out is None else out
        op = _dense(o, "out", self.dtype, _fs._prod(self.out_shape), self.device)
        sp = None
        if return_state and out_state is None:
            out_state = torch.empty(self.state_shape, dtype=torch.float32, device=self.device)
        if out_state is not None:
            sp = self._state(out_state, "out_state")
        ws, nbytes = self._workspace(workspace, self.info.forward_workspace_bytes)
        _fs._check(_fs.lib().fftsplit_linear_attention_forward(self._h, ctypes.byref(x), op, sp, ws, nbytes,
                                                               _stream(self.device)),
                   "fftsplit_linear_attention_forward")
        return o if out_state is None else (o, out_state)

    def backward(self, dout, q, k, v, log_decay, state=None, dstate=None, lengths=None, workspace=None):
        """(dq, dk, dv, gradient of `state`) from the gradient of o and, where
        the state after the last token was used, `dstate`, that of it.  The last
        result is None where no state was given."""
        torch, dev = _torch(), self.device
        x = self._inputs(q, k, v, log_decay, state, lengths)
        gp = _strided(dout, "dout", self.dtype, self.out_shape, dev)
        gs = (ctypes.c_longlong * 3)(*dout.stride()[:3])
        dsp = None if dstate is None else self._state(dstate, "dstate")
        dq = torch.empty(self.q_shape, dtype=self.dtype, device=dev)
        dk = torch.empty(self.k_shape, dtype=self.dtype, device=dev)
        dv = torch.empty(self.v_shape, dtype=self.dtype, device=dev)
        first = None if state is None else torch.empty(self.state_shape, dtype=torch.float32, device=dev)
        ws, nbytes = self._workspace(workspace, self.info.backward_workspace_bytes)
        _fs._check(_fs.lib().fftsplit_linear_attention_backward(
            self._h, ctypes.byref(x), gp, gs, dsp, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
            None if first is None else first.data_ptr(), ws, nbytes, _stream(dev)),
            "fftsplit_linear_attention_backward")
        return dq, dk, dv, first
