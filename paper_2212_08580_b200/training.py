"""Training operators over libngc.so: the AdamW update of many tensors.

Arguments are torch tensors on the current CUDA device; only their checks and the marshalling happen here.  Like the
rest of the package the calls are asynchronous on `stream` (a cudaStream_t as an integer, 0 = legacy default stream).
"""
from __future__ import annotations

import ctypes as C

from .binding import ADAMW_BLOCK, NGC_BF16, NGC_E4M3, NGC_F32, AdamWConfig, AdamWTensor, NgcError, load_library

_INVALID = -1


def _refuse(what: str, why: str):
    raise NgcError(_INVALID, f"{what}: {why}")


def _check_rc(rc: int, what: str):
    if rc != 0:
        raise NgcError(rc, what + ": " + load_library().ngc_strerror(rc).decode())


def _on_device(what: str, name: str, t):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.get_device() != torch.cuda.current_device():
        _refuse(what, f"{name} is not a tensor on the current CUDA device")


class AdamW:
    """AdamW over a list of tensors (see ngc_adamw_update in include/ngc.h), updated in place.

    params, grads: lists of contiguous tensors, float32 or bfloat16 (one type for all params, one for all grads), of
    equal sizes; the gradients' buffers are read by every update (`set_grads` replaces them).
    weight_decay: a number for all tensors or a list with one for each.
    m, v: the states to go on from: float32, or float8_e4m3fn codes (of m and of sqrt(v)) with their scales in
    m_scale, v_scale (float32, one per 256 elements).  Without them the states start at zero in `state_dtype`
    ("f32" or "e4m3").  The lists stay readable as attributes.

    The object keeps the tensors alive and their addresses in a table for the library; an update costs one call.
    """

    def __init__(self, params, grads, lr: float, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.0,
                 state_dtype: str = "f32", m=None, v=None, m_scale=None, v_scale=None):
        import torch
        what = "AdamW"
        self.params = list(params)
        n = len(self.params)
        dtypes = {torch.float32: NGC_F32, torch.bfloat16: NGC_BF16}
        for t in self.params:
            _on_device(what, "params", t)
            if not t.is_contiguous() or t.dtype not in dtypes or t.dtype != self.params[0].dtype:
                _refuse(what, "params are contiguous and all float32 or all bfloat16")
        if (m is None) != (v is None):
            _refuse(what, "m and v are given together")
        if m is None:
            if state_dtype not in ("f32", "e4m3"):
                _refuse(what, "state_dtype is 'f32' or 'e4m3'")
            small = state_dtype == "e4m3"
            def zeros(dtype, sizes):
                return [torch.zeros(s, dtype=dtype, device="cuda") for s in sizes]
            sizes = [t.numel() for t in self.params]
            kind = torch.uint8 if small else torch.float32  # e4m3 zero is the zero byte
            m, v = (zeros(kind, sizes) for _ in range(2))
            if small:
                m, v = ([t.view(torch.float8_e4m3fn) for t in x] for x in (m, v))
                m_scale, v_scale = (zeros(torch.float32, [-(-s // ADAMW_BLOCK) for s in sizes]) for _ in range(2))
        self.m, self.v = list(m), list(v)
        small = n > 0 and bool(self.m) and self.m[0].dtype == torch.float8_e4m3fn
        if small and (m_scale is None or v_scale is None):
            _refuse(what, "8-bit states come with their scales")
        self.m_scale, self.v_scale = (list(m_scale), list(v_scale)) if small else (None, None)
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [float(weight_decay)] * n
        lists = [self.m, self.v, decay] + ([self.m_scale, self.v_scale] if small else [])
        if any(len(x) != n for x in lists):
            _refuse(what, "one state and one weight decay for every tensor")
        state = torch.float8_e4m3fn if small else torch.float32
        for i, p in enumerate(self.params):
            for name, t, dtype, size in (("m", self.m[i], state, p.numel()), ("v", self.v[i], state, p.numel())):
                self._state(what, name, t, dtype, size)
            if small:
                for name, t in (("m_scale", self.m_scale[i]), ("v_scale", self.v_scale[i])):
                    self._state(what, name, t, torch.float32, -(-p.numel() // ADAMW_BLOCK))
        self._table = (AdamWTensor * max(1, n))()
        for i, p in enumerate(self.params):
            e = self._table[i]
            e.theta, e.m, e.v, e.numel = p.data_ptr(), self.m[i].data_ptr(), self.v[i].data_ptr(), p.numel()
            if small:
                e.m_scale, e.v_scale = self.m_scale[i].data_ptr(), self.v_scale[i].data_ptr()
            e.weight_decay = decay[i]
        self._cfg = AdamWConfig(lr=lr, beta1=betas[0], beta2=betas[1], eps=eps, grad_scale=1.0, step=0, step_dev=None,
                                theta_dtype=dtypes[self.params[0].dtype] if n else NGC_F32, grad_dtype=NGC_F32,
                                state_dtype=NGC_E4M3 if small else NGC_F32)
        self._device = torch.cuda.current_device() if n else None
        self._lib = load_library()
        self.step = 0
        self.set_grads(grads)

    @staticmethod
    def _state(what, name, t, dtype, size):
        _on_device(what, name, t)
        if t.dtype != dtype or t.numel() != size or not t.is_contiguous():
            _refuse(what, f"{name} holds {size} contiguous values of {dtype} for this tensor")

    def set_grads(self, grads):
        """The buffers that the following updates read their gradients from."""
        import torch
        grads = list(grads)
        if len(grads) != len(self.params):
            _refuse("AdamW", "one gradient for every tensor")
        for g, p in zip(grads, self.params):
            _on_device("AdamW", "grads", g)
            if (g.numel() != p.numel() or not g.is_contiguous() or g.dtype not in (torch.float32, torch.bfloat16)
                    or g.dtype != grads[0].dtype):
                _refuse("AdamW", "gradients are contiguous, of their tensor's size, all float32 or all bfloat16")
        for e, g in zip(self._table, grads):
            e.grad = g.data_ptr()
        if grads:
            self._cfg.grad_dtype = NGC_F32 if grads[0].dtype == torch.float32 else NGC_BF16
        self.grads = grads

    def update(self, step: int | None = None, lr: float | None = None, grad_scale: float = 1.0, step_dev=None,
               stream: int = 0):
        """ngc_adamw_update: one step, number `step` (default: one more than the last; `self.step` holds it).
        With `step_dev` (an int64 tensor with one value on the device) the number is read there, for a captured call."""
        import torch
        if self._device is not None and torch.cuda.current_device() != self._device:
            _refuse("AdamW", "the tensors are not on the current CUDA device")
        c = self._cfg
        if step_dev is not None:
            _on_device("AdamW", "step_dev", step_dev)
            if step_dev.dtype != torch.int64 or step_dev.numel() != 1:
                _refuse("AdamW", "step_dev is one int64")
            c.step_dev = step_dev.data_ptr()
        else:
            c.step_dev = None
            c.step = self.step + 1 if step is None else int(step)
        if lr is not None:
            c.lr = lr
        c.grad_scale = grad_scale
        _check_rc(self._lib.ngc_adamw_update(C.byref(c), self._table, len(self.params), stream), "ngc_adamw_update")
        if step_dev is None:
            self.step = c.step
