"""ctypes binding of the training operators (``include/egeria_ops.h``) -- argument marshalling only.

:class:`Ops` has the linear layers and the residual norms, :class:`AdamW` the optimizer step; their
methods have the names of the C entry points that they call.  Everything is computed by the CUDA
kernels of ``libegeria.so``; there is no fallback: a call that the library refuses raises
:class:`~paper_2201_06227_b200.binding.EgeriaError`, a tensor that it cannot take ``ValueError``.

Results are allocated on the stream that the call runs on.  Where a ``stream`` is given that is
not the current one, the caller orders it after the kernels that made the inputs, and the inputs
are recorded on it (their memory is not reused before the call has run).
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import binding
from .binding import ERR_INVALID_ARG, WORKSPACE_ALIGN, EgeriaError, _check

F32, BF16, F16 = 0, 1, 2
TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
KINDS = {"layer": 0, "rms": 1}
OPS_WORKSPACE_MIN = 65536
NORM_MAX_COLS = 8192
ADAMW_BLOCK = 256
ADAMW_8BIT = 1

EXPORTS = [
    "egeria_ops_create", "egeria_ops_destroy", "egeria_ops_device_status", "egeria_ops_launch_count",
    "egeria_linear_workspace_bytes", "egeria_linear_forward", "egeria_linear_backward",
    "egeria_norm_workspace_bytes", "egeria_norm_forward", "egeria_norm_backward",
    "egeria_adamw_workspace_bytes", "egeria_adamw_create", "egeria_adamw_destroy", "egeria_adamw_set_grads",
    "egeria_adamw_step", "egeria_adamw_device_status", "egeria_adamw_launch_count",
]

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


def _struct(name, *groups):
    """A ctypes mirror of a C struct: (type, "field field ...") groups in order."""
    return type(name, (ctypes.Structure,), {"_fields_": [(f, t) for t, names in groups for f in names.split()]})


_LinearForward = _struct("egeria_linear_forward_args", (_i32, "type act"), (_i64, "rows inp out"), (_vp, "x w bias residual"),
                         (_i64, "ldx ldw ldr"), (_vp, "y z"), (_i64, "ldy ldz"))
_LinearBackward = _struct("egeria_linear_backward_args", (_i32, "type act act_in"), (_i64, "rows inp out"),
                          (_vp, "dy x w z z_in"), (_i64, "lddy ldx ldw ldz ldz_in"), (_vp, "dx dw db"), (_i64, "lddx lddw"))
_NormForward = _struct("egeria_norm_forward_args", (_i32, "type param_type kind post pre"), (_f32, "alpha eps"),
                       (_i64, "rows cols gate_rows"), (_vp, "x f gate w_post b_post w_pre b_pre"), (_i64, "ldx ldf"),
                       (_vp, "y h"), (_i64, "ldy ldh"), (_vp, "stats"))
_NormBackward = _struct("egeria_norm_backward_args", (_i32, "type param_type kind post pre"), (_f32, "alpha"),
                        (_i64, "rows cols gate_rows"), (_vp, "dy dh y f gate w_post b_post w_pre b_pre"),
                        (_i64, "lddy lddh ldy ldf"), (_vp, "stats dx df"), (_i64, "lddx lddf"),
                        (_vp, "dgate dw_post db_post dw_pre db_pre"))
_AdamTensor = _struct("egeria_adamw_tensor", (_vp, "param master m v m_scale v_scale"), (_i64, "n"),
                      (_i32, "param_type grad_type"), (_f32, "weight_decay"), (_i32, "module"))

_ready = None


def lib() -> ctypes.CDLL:
    """The CUDA library with the signatures of the operators."""
    global _ready
    L = binding.lib()
    if _ready is L:
        return L
    for name, args in (("egeria_linear_workspace_bytes", [_i64] * 3), ("egeria_norm_workspace_bytes", [_i64] * 2),
                       ("egeria_adamw_workspace_bytes", [ctypes.c_int, ctypes.POINTER(_AdamTensor), ctypes.c_uint32])):
        getattr(L, name).argtypes, getattr(L, name).restype = args, ctypes.c_size_t
    L.egeria_ops_create.argtypes = [ctypes.POINTER(_vp), _vp, ctypes.c_size_t]
    L.egeria_adamw_create.argtypes = [ctypes.POINTER(_vp), ctypes.c_int, ctypes.POINTER(_AdamTensor), ctypes.POINTER(_vp), _vp, _vp,
                                      ctypes.c_size_t, ctypes.c_uint32]
    for name in ("egeria_ops_destroy", "egeria_ops_device_status", "egeria_ops_launch_count", "egeria_adamw_destroy",
                 "egeria_adamw_device_status", "egeria_adamw_launch_count"):
        getattr(L, name).argtypes = [_vp]
    L.egeria_ops_launch_count.restype = L.egeria_adamw_launch_count.restype = _i64
    L.egeria_linear_forward.argtypes = [_vp, _vp, ctypes.POINTER(_LinearForward)]
    L.egeria_linear_backward.argtypes = [_vp, _vp, ctypes.POINTER(_LinearBackward)]
    L.egeria_norm_forward.argtypes = [_vp, _vp, ctypes.POINTER(_NormForward)]
    L.egeria_norm_backward.argtypes = [_vp, _vp, ctypes.POINTER(_NormBackward)]
    L.egeria_adamw_set_grads.argtypes = [_vp, _vp, ctypes.POINTER(_vp)]
    L.egeria_adamw_step.argtypes = [_vp, _vp] + [ctypes.c_double] * 4 + [_vp, _vp]
    _ready = L
    return L


def egeria_linear_workspace_bytes(rows: int, inp: int, out: int) -> int:
    """Workspace of an :class:`Ops` whose linear calls have at most these sizes (take the largest over the layers)."""
    return int(lib().egeria_linear_workspace_bytes(int(rows), int(inp), int(out)))


def egeria_norm_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().egeria_norm_workspace_bytes(int(rows), int(cols)))


def _workspace(nbytes: int, device):
    raw = torch.empty(nbytes + WORKSPACE_ALIGN, dtype=torch.uint8, device=device)
    return raw, raw.data_ptr() + (-raw.data_ptr()) % WORKSPACE_ALIGN


class _On:
    """The stream of a call: allocations inside come from it, foreign inputs are recorded on it."""

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream], tensors):
        self.current = torch.cuda.current_stream(device)
        self.stream = self.current if stream is None else stream
        if self.stream.device != device:
            raise ValueError(f"the stream is of {self.stream.device}, the handle of {device}")
        self.tensors = tensors
        self.context = torch.cuda.stream(self.stream)

    def __enter__(self):
        self.context.__enter__()
        return int(self.stream.cuda_stream)

    def __exit__(self, *exc):
        if self.stream != self.current:
            for t in self.tensors:
                if t is not None:
                    t.record_stream(self.stream)
        return self.context.__exit__(*exc)


def _matrix(t: torch.Tensor, name: str, device, dtype, rows: int, cols: int):
    """(pointer, pitch) of a matrix whose rows are consecutive."""
    if t.device != device or t.dtype != dtype or t.dim() != 2 or tuple(t.shape) != (rows, cols):
        raise ValueError(f"{name}: expected {dtype} [{rows}, {cols}] on {device}, got {t.dtype} {list(t.shape)} on {t.device}")
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the values of a row have to be consecutive")
    if rows > 1 and t.stride(0) < cols:
        raise ValueError(f"{name}: rows overlap")
    return t.data_ptr(), (t.stride(0) if rows > 1 else cols)


def _optional(t: Optional[torch.Tensor], *args):
    return (None, 0) if t is None else _matrix(t, *args)


def _vector(t: Optional[torch.Tensor], name: str, device, dtype, n: int):
    if t is None:
        return None
    if t.device != device or t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: expected {n} consecutive {dtype} on {device}")
    return t.data_ptr()


class Ops:
    """Handle of the linear and norm calls; owns its workspace.  For one stream at a time."""

    def __init__(self, workspace_bytes: int = OPS_WORKSPACE_MIN, device="cuda"):
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.workspace_bytes = max(int(workspace_bytes), OPS_WORKSPACE_MIN)
        self._raw, ptr = _workspace(self.workspace_bytes, self.device)
        handle = _vp()
        with torch.cuda.device(self.device):
            _check(lib().egeria_ops_create(ctypes.byref(handle), ptr, self.workspace_bytes), "egeria_ops_create")
        self._h = handle

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().egeria_ops_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------------ linear layers
    def egeria_linear_forward(self, x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
                              residual: Optional[torch.Tensor] = None, save_z: bool = False, out: Optional[torch.Tensor] = None,
                              stream: Optional[torch.cuda.Stream] = None):
        """y = act(x w^T + bias) + residual for x [rows, inp] and w [out, inp] in bfloat16 or float16; (y, z) with
        save_z, z the argument of the activation.  `out` may be the residual."""
        if act not in ACTS:
            raise ValueError(f"unknown activation {act!r}")
        if x.dim() != 2 or w.dim() != 2:
            raise ValueError("x and w are matrices")
        (rows, inp), n = x.shape, w.shape[0]
        a = _LinearForward(type=TYPES.get(x.dtype, -1), act=ACTS[act], rows=rows, inp=inp, out=n)
        dev, t = self.device, x.dtype
        a.x, a.ldx = _matrix(x, "x", dev, t, rows, inp)
        a.w, a.ldw = _matrix(w, "w", dev, t, n, inp)
        a.bias = _vector(bias, "bias", dev, t, n)
        a.residual, a.ldr = _optional(residual, "residual", dev, t, rows, n)
        with _On(dev, stream, (self._raw, x, w, bias, residual, out)) as s:
            y = torch.empty((rows, n), dtype=t, device=dev) if out is None else out
            z = torch.empty((rows, n), dtype=t, device=dev) if save_z else None
            a.y, a.ldy = _matrix(y, "out", dev, t, rows, n)
            a.z, a.ldz = _optional(z, "z", dev, t, rows, n)
            _check(lib().egeria_linear_forward(self._h, s, ctypes.byref(a)), "egeria_linear_forward")
        return (y, z) if save_z else y

    def egeria_linear_backward(self, dy: torch.Tensor, x: Optional[torch.Tensor], w: Optional[torch.Tensor],
                               z: Optional[torch.Tensor] = None, act: str = "none", z_in: Optional[torch.Tensor] = None,
                               act_in: str = "none", need_dx: bool = True, need_dw: bool = True, need_db: bool = True,
                               stream: Optional[torch.cuda.Stream] = None):
        """(dx, dw, db) of a linear layer, None for what is not needed: a frozen layer takes need_dw = need_db = False and
        no x, the first layer that still trains need_dx = False and no w.  With act_in and z_in, dx is the gradient of
        z_in, x having come out of act_in(z_in)."""
        if act not in ACTS or act_in not in ACTS:
            raise ValueError(f"unknown activation {act!r} or {act_in!r}")
        if dy.dim() != 2 or (need_dx and w is None) or (need_dw and x is None) or (x is None and w is None):
            raise ValueError("dy is a matrix; dx needs w, dw needs x, and one of the two has to be there")
        rows, n = dy.shape
        inp = x.shape[1] if x is not None else w.shape[1]
        dev, t = self.device, dy.dtype
        a = _LinearBackward(type=TYPES.get(t, -1), act=ACTS[act], act_in=ACTS[act_in], rows=rows, inp=inp, out=n)
        a.dy, a.lddy = _matrix(dy, "dy", dev, t, rows, n)
        a.x, a.ldx = _optional(x, "x", dev, t, rows, inp)
        a.w, a.ldw = _optional(w, "w", dev, t, n, inp)
        a.z, a.ldz = _optional(z, "z", dev, t, rows, n)
        a.z_in, a.ldz_in = _optional(z_in, "z_in", dev, t, rows, inp)
        with _On(dev, stream, (self._raw, dy, x, w, z, z_in)) as s:
            dx = torch.empty((rows, inp), dtype=t, device=dev) if need_dx else None
            dw = torch.empty((n, inp), dtype=t, device=dev) if need_dw else None
            db = torch.empty(n, dtype=t, device=dev) if need_db else None
            a.dx, a.lddx = _optional(dx, "dx", dev, t, rows, inp)
            a.dw, a.lddw = _optional(dw, "dw", dev, t, n, inp)
            a.db = _vector(db, "db", dev, t, n)
            _check(lib().egeria_linear_backward(self._h, s, ctypes.byref(a)), "egeria_linear_backward")
        return dx, dw, db

    # ------------------------------------------------------------------ residual norms
    def _norm_common(self, a, like, gate, gate_rows, w_post, b_post, w_pre, b_pre, kind, post, pre):
        if kind not in KINDS:
            raise ValueError(f"unknown norm {kind!r}")
        given = [v for v in (gate, w_post, b_post, w_pre, b_pre) if v is not None]
        pt = given[0].dtype if given else like.dtype
        rows, cols = like.shape
        a.type, a.param_type, a.kind, a.post, a.pre = TYPES.get(like.dtype, -1), TYPES.get(pt, -1), KINDS[kind], int(post), int(pre)
        a.rows, a.cols, a.gate_rows = rows, cols, int(gate_rows)
        groups = 1 if gate_rows == 0 else -(-rows // gate_rows) if gate_rows > 0 else 0
        a.gate = _vector(gate, "gate", self.device, pt, groups * cols)
        for name, v in (("w_post", w_post), ("b_post", b_post), ("w_pre", w_pre), ("b_pre", b_pre)):
            setattr(a, name, _vector(v, name, self.device, pt, cols))
        return pt

    def egeria_norm_forward(self, x: torch.Tensor, f: torch.Tensor, gate: Optional[torch.Tensor] = None, gate_rows: int = 0,
                            w_post: Optional[torch.Tensor] = None, b_post: Optional[torch.Tensor] = None,
                            w_pre: Optional[torch.Tensor] = None, b_pre: Optional[torch.Tensor] = None, kind: str = "layer",
                            post: bool = True, pre: bool = True, alpha: float = 1.0, eps: float = 1e-5,
                            stream: Optional[torch.cuda.Stream] = None):
        """(y, h, stats): y = alpha x + gate * N_post(f), h = N_pre(y) (None without pre), stats for the backward call."""
        if x.dim() != 2:
            raise ValueError("x is a matrix")
        a, dev, t = _NormForward(alpha=alpha, eps=eps), self.device, x.dtype
        rows, cols = x.shape
        self._norm_common(a, x, gate, gate_rows, w_post, b_post, w_pre, b_pre, kind, post, pre)
        a.x, a.ldx = _matrix(x, "x", dev, t, rows, cols)
        a.f, a.ldf = _matrix(f, "f", dev, t, rows, cols)
        with _On(dev, stream, (self._raw, x, f, gate, w_post, b_post, w_pre, b_pre)) as s:
            y = torch.empty((rows, cols), dtype=t, device=dev)
            h = torch.empty((rows, cols), dtype=t, device=dev) if pre else None
            stats = torch.empty((rows, 4), dtype=torch.float32, device=dev)
            a.y, a.ldy = _matrix(y, "y", dev, t, rows, cols)
            a.h, a.ldh = _optional(h, "h", dev, t, rows, cols)
            a.stats = stats.data_ptr()
            _check(lib().egeria_norm_forward(self._h, s, ctypes.byref(a)), "egeria_norm_forward")
        return y, h, stats

    def egeria_norm_backward(self, dy: torch.Tensor, dh: Optional[torch.Tensor], y: torch.Tensor, f: torch.Tensor,
                             stats: torch.Tensor, gate: Optional[torch.Tensor] = None, gate_rows: int = 0,
                             w_post: Optional[torch.Tensor] = None, b_post: Optional[torch.Tensor] = None,
                             w_pre: Optional[torch.Tensor] = None, b_pre: Optional[torch.Tensor] = None, kind: str = "layer",
                             post: bool = True, pre: bool = True, alpha: float = 1.0, need_params: bool = True,
                             stream: Optional[torch.cuda.Stream] = None):
        """The gradients as a dict: dx, df, and for what is given (and with need_params) dgate, dw_post, db_post, dw_pre,
        db_pre, else None."""
        if dy.dim() != 2:
            raise ValueError("dy is a matrix")
        a, dev, t = _NormBackward(alpha=alpha), self.device, dy.dtype
        rows, cols = dy.shape
        pt = self._norm_common(a, dy, gate, gate_rows, w_post, b_post, w_pre, b_pre, kind, post, pre)
        a.dy, a.lddy = _matrix(dy, "dy", dev, t, rows, cols)
        a.dh, a.lddh = _optional(dh, "dh", dev, t, rows, cols)
        a.y, a.ldy = _matrix(y, "y", dev, t, rows, cols)
        a.f, a.ldf = _matrix(f, "f", dev, t, rows, cols)
        a.stats = _vector(stats, "stats", dev, torch.float32, 4 * rows)
        with _On(dev, stream, (self._raw, dy, dh, y, f, stats, gate, w_post, b_post, w_pre, b_pre)) as s:
            out = dict(dx=torch.empty((rows, cols), dtype=t, device=dev), df=torch.empty((rows, cols), dtype=t, device=dev))
            a.dx, a.lddx = _matrix(out["dx"], "dx", dev, t, rows, cols)
            a.df, a.lddf = _matrix(out["df"], "df", dev, t, rows, cols)
            for name, v, there in (("dgate", gate, True), ("dw_post", w_post, post), ("db_post", b_post, post),
                                   ("dw_pre", w_pre, pre), ("db_pre", b_pre, pre)):
                out[name] = torch.empty_like(v) if v is not None and there and need_params else None
                setattr(a, name, None if out[name] is None else out[name].data_ptr())
            _check(lib().egeria_norm_backward(self._h, s, ctypes.byref(a)), "egeria_norm_backward")
        return out

    def egeria_ops_device_status(self) -> int:
        return int(lib().egeria_ops_device_status(self._h))

    def check_device_status(self) -> None:
        _check(self.egeria_ops_device_status(), "egeria_ops_device_status")

    def egeria_ops_launch_count(self) -> int:
        return int(lib().egeria_ops_launch_count(self._h))


class AdamW:
    """The AdamW step of a model's tensors in one launch per combination of types; frozen modules are left out on the device.

    params, grads, exp_avg, exp_avg_sq: one contiguous CUDA tensor per tensor of the model; the moments are float32, or
    int8 and uint8 codes with their scales (float32, one per 256 values) in m_scales and v_scales.  masters: float32 copies
    that the step works on (entries may be None).  steps: int32 [count] on the device.  modules: each tensor's entry in
    the freeze mask, -1 for none.  The handle keeps all of them alive.
    """

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], exp_avg: Sequence[torch.Tensor],
                 exp_avg_sq: Sequence[torch.Tensor], steps: torch.Tensor, masters: Optional[Sequence] = None,
                 m_scales: Optional[Sequence[torch.Tensor]] = None, v_scales: Optional[Sequence[torch.Tensor]] = None,
                 weight_decay=0.0, modules: Optional[Sequence[int]] = None):
        n = len(params)
        if n < 1:
            raise ValueError("no tensors")
        self.device = params[0].device
        small = m_scales is not None or v_scales is not None
        none = [None] * n
        columns = dict(grads=grads, exp_avg=exp_avg, exp_avg_sq=exp_avg_sq, masters=masters or none, m_scales=m_scales or none,
                       v_scales=v_scales or none, modules=modules if modules is not None else [-1] * n,
                       weight_decay=[weight_decay] * n if isinstance(weight_decay, (int, float)) else weight_decay)
        for name, c in columns.items():
            if len(c) != n:
                raise ValueError(f"{name}: one entry per tensor is required")
        table = (_AdamTensor * n)()
        self.modules = [int(m) for m in columns["modules"]]
        for i, p in enumerate(params):
            k = p.numel()
            if p.dtype not in TYPES:
                raise ValueError(f"tensor {i}: {p.dtype} parameters are not supported")
            blocks = -(-k // ADAMW_BLOCK)
            row = table[i]
            row.n, row.param_type = k, TYPES[p.dtype]
            row.grad_type = TYPES.get(columns["grads"][i].dtype, -1)
            row.weight_decay, row.module = float(columns["weight_decay"][i]), self.modules[i]
            row.param = _vector(p, f"params[{i}]", self.device, p.dtype, k)
            row.master = _vector(columns["masters"][i], f"masters[{i}]", self.device, torch.float32, k)
            row.m = _vector(exp_avg[i], f"exp_avg[{i}]", self.device, torch.int8 if small else torch.float32, k)
            row.v = _vector(exp_avg_sq[i], f"exp_avg_sq[{i}]", self.device, torch.uint8 if small else torch.float32, k)
            row.m_scale = _vector(columns["m_scales"][i], f"m_scales[{i}]", self.device, torch.float32, blocks)
            row.v_scale = _vector(columns["v_scales"][i], f"v_scales[{i}]", self.device, torch.float32, blocks)
        self._sizes = [(p.numel(), g.dtype) for p, g in zip(params, grads)]
        self._steps = steps
        self._keep = (list(params), list(exp_avg), list(exp_avg_sq), columns["masters"], columns["m_scales"], columns["v_scales"])
        flags = ADAMW_8BIT if small else 0
        with torch.cuda.device(self.device):
            nbytes = int(lib().egeria_adamw_workspace_bytes(n, table, flags))
            if nbytes == 0:
                raise EgeriaError(ERR_INVALID_ARG, "egeria_adamw_workspace_bytes")
            self._raw, ptr = _workspace(nbytes, self.device)
            handle = _vp()
            _check(lib().egeria_adamw_create(ctypes.byref(handle), n, table, self._grad_pointers(grads),
                                             _vector(steps, "steps", self.device, torch.int32, n), ptr, nbytes, flags),
                   "egeria_adamw_create")
        self._h = handle

    def _grad_pointers(self, grads):
        if len(grads) != len(self._sizes):
            raise ValueError("grads: one entry per tensor is required")
        ptrs = (_vp * len(grads))(*[_vector(g, f"grads[{i}]", self.device, t, n)
                                    for i, (g, (n, t)) in enumerate(zip(grads, self._sizes))])
        self._grads = list(grads)
        return ptrs

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().egeria_adamw_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def egeria_adamw_set_grads(self, grads: Sequence[torch.Tensor], stream: Optional[torch.cuda.Stream] = None) -> None:
        """The gradients (same sizes and types) are in these tensors from the next step on."""
        ptrs = self._grad_pointers(grads)
        with _On(self.device, stream, (self._raw,)) as s:
            _check(lib().egeria_adamw_set_grads(self._h, s, ptrs), "egeria_adamw_set_grads")

    def egeria_adamw_step(self, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                          grad_scale: Optional[torch.Tensor] = None, frozen: Optional[torch.Tensor] = None,
                          stream: Optional[torch.cuda.Stream] = None) -> None:
        """One step of every tensor whose module is not marked in `frozen` (uint8, as egeria_plasticity_evaluate leaves it)."""
        gs = _vector(grad_scale, "grad_scale", self.device, torch.float32, 1)
        if frozen is not None and (frozen.dtype != torch.uint8 or frozen.device != self.device or not frozen.is_contiguous()
                                   or frozen.numel() <= max(self.modules)):
            raise ValueError("frozen: expected contiguous uint8, one per module, on the handle's device")
        with _On(self.device, stream, (self._raw, *self._grads, *[t for c in self._keep for t in c], self._steps, grad_scale, frozen)) as s:
            _check(lib().egeria_adamw_step(self._h, s, lr, beta1, beta2, eps, gs, None if frozen is None else frozen.data_ptr()),
                   "egeria_adamw_step")

    def egeria_adamw_device_status(self) -> int:
        return int(lib().egeria_adamw_device_status(self._h))

    def check_device_status(self) -> None:
        _check(self.egeria_adamw_device_status(), "egeria_adamw_device_status")

    def egeria_adamw_launch_count(self) -> int:
        return int(lib().egeria_adamw_launch_count(self._h))
