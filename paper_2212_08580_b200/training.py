"""Training operators over libngc.so: the AdamW update of many tensors, two losses on logits with their gradients
(clipped policy loss with KL term, preference loss over pairs of packed sequences), softmax cross entropy over a large
vocabulary straight from features and weights, and dropout whose mask is a function of position.

Arguments are torch tensors on the current CUDA device; only their checks and the marshalling happen here.  Like the
rest of the package the calls are asynchronous on `stream` (a cudaStream_t as an integer, 0 = legacy default stream).
"""
from __future__ import annotations

import ctypes as C

from .binding import (ADAMW_BLOCK, NGC_BF16, NGC_E4M3, NGC_F32, AdamWConfig, AdamWTensor, DropoutConfig,
                      LinearCrossEntropyConfig, NgcError, PolicyLossConfig, PreferenceLossConfig, load_library)

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
    ("f32" or "e4m3"), which is refused during a graph capture (its replays would zero them again).  The lists stay readable
    as attributes.

    The object keeps the tensors alive and their addresses in a table for the library; an update costs one call.  It is
    kept until its updates have run.
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
            if n and torch.cuda.is_current_stream_capturing():
                _refuse(what, "states that start at zero are made outside a capture, whose replays would zero them again")
            small = state_dtype == "e4m3"

            def zeros(dtype, sizes):
                return [torch.zeros(s, dtype=dtype, device="cuda") for s in sizes]
            sizes = [t.numel() for t in self.params]
            kind = torch.uint8 if small else torch.float32  # e4m3 zero is the zero byte
            m, v = (zeros(kind, sizes) for _ in range(2))
            if small:
                m, v = ([t.view(torch.float8_e4m3fn) for t in x] for x in (m, v))
                m_scale, v_scale = (zeros(torch.float32, [-(-s // ADAMW_BLOCK) for s in sizes]) for _ in range(2))
            if n:
                torch.cuda.current_stream().synchronize()  # updates on any stream find the zeros
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
        `lr` stays for the steps after it.  With `step_dev` (an int64 tensor with one value on the device) the number is read there, for a captured call."""
        import torch
        if self._device is not None and torch.cuda.current_device() != self._device:
            _refuse("AdamW", "the tensors are not on the current CUDA device")
        c, old_lr = self._cfg, self._cfg.lr
        if step_dev is not None:
            _on_device("AdamW", "step_dev", step_dev)
            if step_dev.dtype != torch.int64 or step_dev.numel() != 1:
                _refuse("AdamW", "step_dev is one int64")
            c.step_dev = step_dev.data_ptr()
        else:
            c.step_dev = None
            number = self.step + 1 if step is None else int(step)
            if not 1 <= number < 1 << 63:
                _refuse("AdamW", "the step number is at least 1 and has 63 bits")
            c.step = number
        if lr is not None:
            c.lr = lr
        c.grad_scale = grad_scale
        rc = self._lib.ngc_adamw_update(C.byref(c), self._table, len(self.params), stream)
        if rc != 0:
            c.lr = old_lr
        _check_rc(rc, "ngc_adamw_update")
        if step_dev is None:
            self.step = c.step


def _logits(what: str, device: int, logits, dlogits):
    """Type, row stride and gradient's row stride of a matrix of logits, after checks of it and of its gradient's buffer."""
    import torch
    shape, dtype = logits.shape, logits.dtype
    if len(shape) == 2 and shape[1] >= 1 << 31:  # (ctypes would cut it to 32 bits)
        _refuse(what, "at most 2^31 - 1 classes")
    strides = []
    for name, t in (("logits", logits), ("dlogits", dlogits)):
        if t is None and name == "dlogits":
            strides.append(0)
            continue
        if t.get_device() != device:
            _refuse(what, f"{name} is not a tensor on the current CUDA device")
        if len(t.shape) != 2 or t.shape != shape or t.dtype != dtype or shape[1] < 1:
            _refuse(what, f"{name}: a matrix [rows, classes], both of one shape and type")
        rows, columns = t.stride()
        if (columns != 1 and shape[1] > 1) or (rows < shape[1] and shape[0] > 1):
            _refuse(what, f"{name}: the logits of a row are contiguous, rows do not overlap")
        strides.append(rows if shape[0] > 1 else max(shape[1], rows))
    if dtype == torch.float32:
        return NGC_F32, strides[0], strides[1]
    if dtype == torch.bfloat16:
        return NGC_BF16, strides[0], strides[1]
    _refuse(what, "logits are float32 or bfloat16")


def _vector(what: str, name: str, device: int, t, dtype, size: int):
    if t.get_device() != device:
        _refuse(what, f"{name} is not a tensor on the current CUDA device")
    if t.dtype != dtype or t.numel() != size or not t.is_contiguous():
        _refuse(what, f"{name} holds {size} contiguous values of {dtype}")
    return t.data_ptr()


def policy_loss(logits, actions, old_logp, advantage, dlogits, logp, row_loss, loss=None, *, ref_logp=None, weight=None,
                rows_per_partition: int | None = None, scale: float = 1.0, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, stream: int = 0):
    """ngc_policy_loss: clipped policy loss (with a KL term where ref_logp is given) of every row of logits
    [rows, classes], written to dlogits (may be `logits` itself; None: loss only), logp and row_loss [rows], and loss
    [ceil(rows / rows_per_partition)], the sums over partitions of consecutive rows (default: all rows are one).
    actions: int32; old_logp, ref_logp, advantage, weight: float32."""
    import torch
    what, f32 = "policy_loss", torch.float32
    dev = torch.cuda.current_device() if torch.cuda.is_initialized() else -2
    try:
        dtype, ld, ld_grad = _logits(what, dev, logits, dlogits)
        rows, classes = logits.shape
        each = max(rows, 1) if rows_per_partition is None else int(rows_per_partition)
        if each < 1:
            _refuse(what, "rows_per_partition is at least 1")
        each = min(each, max(rows, 1))  # (ctypes would cut it to 64 bits)
        cfg = PolicyLossConfig(rows, each, classes, dtype, scale, clip_low, clip_high, kl_coef)
        args = (C.byref(cfg), logits.data_ptr(), ld, _vector(what, "actions", dev, actions, torch.int32, rows),
                _vector(what, "old_logp", dev, old_logp, f32, rows),
                None if ref_logp is None else _vector(what, "ref_logp", dev, ref_logp, f32, rows),
                _vector(what, "advantage", dev, advantage, f32, rows),
                None if weight is None else _vector(what, "weight", dev, weight, f32, rows),
                None if dlogits is None else dlogits.data_ptr(), ld_grad,
                None if logp is None else _vector(what, "logp", dev, logp, f32, rows),
                _vector(what, "row_loss", dev, row_loss, f32, rows),
                None if loss is None else _vector(what, "loss", dev, loss, f32, -(-rows // each)), stream)
    except AttributeError as e:
        _refuse(what, f"not a tensor ({e})")
    _check_rc(load_library().ngc_policy_loss(*args), "ngc_policy_loss")


def preference_workspace_bytes(rows: int, pairs: int) -> int:
    """Bytes of workspace that preference_loss asks for."""
    return int(load_library().ngc_preference_workspace_bytes(rows, pairs))


def preference_loss(logits, labels, seq_begin, ref_logp, dlogits, seq_logp, pair_loss, workspace, *, pair_weight=None,
                    scale: float = 1.0, beta: float = 0.1, label_smoothing: float = 0.0, length_mean: bool = False,
                    stream: int = 0):
    """ngc_preference_loss: paired log-ratio loss over packed sequences.  logits [rows, classes]; labels int32 [rows];
    seq_begin int64 [2 pairs + 1] on the device; ref_logp, seq_logp float32 [2 pairs]; pair_loss, pair_weight float32
    [pairs]; dlogits like logits (may be `logits` itself; None: loss only); workspace: a uint8 tensor of
    preference_workspace_bytes(rows, pairs) that no overlapping call uses."""
    import torch
    what, f32 = "preference_loss", torch.float32
    dev = torch.cuda.current_device() if torch.cuda.is_initialized() else -2
    try:
        dtype, ld, ld_grad = _logits(what, dev, logits, dlogits)
        rows, classes = logits.shape
        pairs = pair_loss.numel()
        if pairs >= 1 << 31:
            _refuse(what, "fewer than 2^31 pairs")
        if workspace.get_device() != dev or not workspace.is_contiguous():
            _refuse(what, "workspace is contiguous memory of the current CUDA device")
        cfg = PreferenceLossConfig(rows, pairs, classes, dtype, 1 if length_mean else 0, scale, beta, label_smoothing)
        args = (C.byref(cfg), logits.data_ptr(), ld, _vector(what, "labels", dev, labels, torch.int32, rows),
                _vector(what, "seq_begin", dev, seq_begin, torch.int64, 2 * pairs + 1),
                _vector(what, "ref_logp", dev, ref_logp, f32, 2 * pairs),
                None if pair_weight is None else _vector(what, "pair_weight", dev, pair_weight, f32, pairs),
                None if dlogits is None else dlogits.data_ptr(), ld_grad,
                _vector(what, "seq_logp", dev, seq_logp, f32, 2 * pairs),
                _vector(what, "pair_loss", dev, pair_loss, f32, pairs),
                workspace.data_ptr(), workspace.numel() * workspace.element_size(), stream)
    except AttributeError as e:
        _refuse(what, f"not a tensor ({e})")
    _check_rc(load_library().ngc_preference_loss(*args), "ngc_preference_loss")


def _matrix(what: str, name: str, device: int, t, dtype, shape):
    """Row stride of a matrix of rows that are contiguous each and do not overlap."""
    if t.get_device() != device:
        _refuse(what, f"{name} is not a tensor on the current CUDA device")
    if t.dtype != dtype or t.shape != shape:
        _refuse(what, f"{name} is a matrix {tuple(shape)} of {dtype}")
    row, column = t.stride()
    columns = shape[1]
    if column == 1 and row >= columns:
        return row
    if (column != 1 and columns > 1) or (row < columns and shape[0] > 1):
        _refuse(what, f"{name}: the elements of a row are contiguous, rows do not overlap")
    return row if shape[0] > 1 else max(row, columns)


def _position(what: str, seed: int, step: int, first_row: int):
    if not (0 <= seed < 1 << 64 and 0 <= first_row < 1 << 63 and 0 <= step < 1 << 32):
        _refuse(what, "seed has 64 bits, first_row 63, step 32")


def dropout(x, out, p: float, *, seed: int, step: int = 0, first_row: int = 0, residual=None, stream: int = 0):
    """ngc_dropout: out = x / (1 - p) where the generator keeps an element and 0 where it does not, plus `residual`.
    x, out, residual: matrices [rows, columns], float32 or bfloat16, all of one type; out may be x or residual itself.  The
    mask depends on (seed, step, first_row + row, column) alone; the gradient is the same call on the gradient."""
    import torch
    what = "dropout"
    dev = torch.cuda.current_device() if torch.cuda.is_initialized() else -2
    try:
        dtype, shape = x.dtype, x.shape
        if len(shape) != 2 or shape[1] < 1 or shape[1] >= 1 << 31 or dtype not in (torch.float32, torch.bfloat16):
            _refuse(what, "x is a matrix [rows, columns] of float32 or bfloat16")
        _position(what, seed, step, first_row)
        ld_x, ld_out = _matrix(what, "x", dev, x, dtype, shape), _matrix(what, "out", dev, out, dtype, shape)
        at = None if residual is None else residual.data_ptr()
        ld = 0 if residual is None else _matrix(what, "residual", dev, residual, dtype, shape)
        cfg = DropoutConfig(shape[0], shape[1], NGC_F32 if dtype == torch.float32 else NGC_BF16, p, seed, first_row, step)
        args = (C.byref(cfg), x.data_ptr(), ld_x, at, ld, out.data_ptr(), ld_out, stream)
    except AttributeError as e:
        _refuse(what, f"not a tensor ({e})")
    _check_rc(load_library().ngc_dropout(*args), "ngc_dropout")


def _weights(what: str, name: str, device: int, t, classes: int, d: int, feature_major=None):
    """(feature_major, row stride) of a matrix [classes, d]; feature_major: the classes of a feature are contiguous."""
    import torch
    if t.get_device() != device:
        _refuse(what, f"{name} is not a tensor on the current CUDA device")
    if t.dtype != torch.bfloat16 or t.shape != (classes, d):
        _refuse(what, f"{name} is a matrix [classes, d] of bfloat16")
    a, b = t.stride()
    if b == 1 and a >= d and not feature_major:
        return False, a
    for major in ((False, True) if feature_major is None else (feature_major,)):
        rows, columns, row, column = (d, classes, b, a) if major else (classes, d, a, b)
        if (column == 1 or columns == 1) and (row >= columns or rows == 1):
            return major, row if rows > 1 else max(row, columns)
    _refuse(what, f"{name}: contiguous along d or along the classes" + ("" if feature_major is None else ", as the weights are"))


def _ce_config(what, x, weight, dx, dweight, rows_per_partition, keep_rows, piece_rows, scale=1.0, drop=0.0, seed=0, step=0,
               first_row=0):
    """(configuration, strides of x, weight, dx, dweight and of its partitions) after checks of them."""
    import torch
    dev = torch.cuda.current_device() if torch.cuda.is_initialized() else -2
    bf16 = torch.bfloat16
    if len(x.shape) != 2 or len(weight.shape) != 2 or x.shape[1] != weight.shape[1] or 0 in (*weight.shape, x.shape[1]):
        _refuse(what, "x is [rows, d], weight is [classes, d]")
    (rows, d), classes = x.shape, weight.shape[0]
    if d > 1 << 20 or classes > 1 << 24 or rows >= 1 << 31:
        _refuse(what, "at most 2^31 - 1 rows, 2^20 features and 2^24 classes")
    ld_x = _matrix(what, "x", dev, x, bf16, (rows, d))
    major, ld_w = _weights(what, "weight", dev, weight, classes, d)
    each = max(rows, 1) if rows_per_partition is None else int(rows_per_partition)
    if each < 1 or piece_rows < 0:
        _refuse(what, "rows_per_partition is at least 1, piece_rows is not negative")
    each = min(each, max(rows, 1))
    parts = max(1, -(-rows // each))
    ld_dx = _matrix(what, "dx", dev, dx, bf16, (rows, d)) if dx is not None else 0
    ld_dw = part = 0
    if dweight is not None:
        whole = len(dweight.shape) == 3
        if not whole and (len(dweight.shape) != 2 or parts != 1) or whole and dweight.shape[0] != parts:
            _refuse(what, f"dweight is [{parts}, classes, d]")
        one = dweight[0] if whole else dweight
        try:
            _, ld_dw = _weights(what, "dweight", dev, one, classes, d, major)
        except NgcError:
            if d > 1 and classes > 1:
                raise
            # one row or column of weights may be read either way: as the gradient is
            _, ld_dw = _weights(what, "dweight", dev, one, classes, d, not major)
            major, ld_w = _weights(what, "weight", dev, weight, classes, d, not major)
        part = dweight.stride(0) if whole else 0
    _position(what, seed, step, first_row)
    cfg = LinearCrossEntropyConfig(rows, each, min(int(piece_rows), 1 << 31), d, classes, 1 if major else 0, 1 if keep_rows else 0,
                                   scale, drop, seed, first_row, step)
    return cfg, ld_x, ld_w, ld_dx, ld_dw, part, dev


def linear_cross_entropy_workspace_bytes(x, weight, *, dx=None, dweight=None, rows_per_partition: int | None = None,
                                         keep_rows: bool = False, piece_rows: int = 0) -> int:
    """Bytes of workspace that linear_cross_entropy asks for with the same arguments."""
    what = "linear_cross_entropy_workspace_bytes"
    try:
        cfg, _, ld_w, *_ = _ce_config(what, x, weight, dx, dweight, rows_per_partition, keep_rows, piece_rows)
        address = weight.data_ptr()
    except AttributeError as e:
        _refuse(what, f"not a tensor ({e})")
    return int(load_library().ngc_linear_cross_entropy_workspace_bytes(C.byref(cfg), address, ld_w, int(dx is not None),
                                                                       int(dweight is not None)))


def linear_cross_entropy(x, weight, labels, logp, row_loss, loss, workspace, *, dx=None, dweight=None, row_weight=None,
                         rows_per_partition: int | None = None, scale: float = 1.0, dropout: float = 0.0, seed: int = 0,
                         step: int = 0, first_row: int = 0, keep_rows: bool = False, piece_rows: int = 0, stream: int = 0):
    """ngc_linear_cross_entropy: softmax cross entropy of `scale * x weight^T` with its gradients, the logits never stored.
    x [rows, d] and weight [classes, d] are bfloat16; weight is contiguous along d, or along the classes (theta.view(d, classes).t()
    of this library's softmax model).  labels int32 [rows] (outside the classes: the row is left out), row_weight float32.
    logp, row_loss: float32 [rows]; loss (or None): float32 [ceil(rows / rows_per_partition)].
    dx like x, dweight [partitions, classes, d] with the weight's layout (or [classes, d] for one partition); None: not wanted.
    dropout: on x, by the rule of `dropout` at (seed, step, first_row + row, feature).
    keep_rows: rows are read where they are instead of being packed (include/ngc.h has the conditions).
    piece_rows: at most so many rows at a time, but 64 at least (0: as many as 2 GiB of 16-bit powers holds).
    workspace: a tensor (of any type) of linear_cross_entropy_workspace_bytes(...) bytes that no overlapping call uses."""
    import torch
    what, f32 = "linear_cross_entropy", torch.float32
    try:
        cfg, ld_x, ld_w, ld_dx, ld_dw, part, dev = _ce_config(what, x, weight, dx, dweight, rows_per_partition, keep_rows, piece_rows,
                                                              scale, dropout, seed, step, first_row)
        rows = cfg.rows
        if workspace.get_device() != dev or not workspace.is_contiguous():
            _refuse(what, "workspace is contiguous memory of the current CUDA device")
        args = (C.byref(cfg), x.data_ptr(), ld_x, weight.data_ptr(), ld_w, _vector(what, "labels", dev, labels, torch.int32, rows),
                None if row_weight is None else _vector(what, "row_weight", dev, row_weight, f32, rows),
                None if dx is None else dx.data_ptr(), ld_dx, None if dweight is None else dweight.data_ptr(), ld_dw, part,
                _vector(what, "logp", dev, logp, f32, rows), _vector(what, "row_loss", dev, row_loss, f32, rows),
                None if loss is None else _vector(what, "loss", dev, loss, f32, -(-rows // cfg.rows_per_partition)),
                workspace.data_ptr(), workspace.numel() * workspace.element_size(), stream)
    except AttributeError as e:
        _refuse(what, f"not a tensor ({e})")
    _check_rc(load_library().ngc_linear_cross_entropy(*args), "ngc_linear_cross_entropy")


def linear_cross_entropy_gave_up(workspace) -> bool:
    """Whether a bounded device-side wait of the last call on this workspace gave up (waits for the device)."""
    import torch
    torch.cuda.synchronize(workspace.device)  # (the call may be on any stream)
    return bool(workspace.view(-1).view(torch.uint8)[:4].view(torch.int32).item())
