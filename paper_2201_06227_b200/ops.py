"""ctypes binding of the training operators (``include/egeria_ops.h``) -- argument marshalling only.

:class:`Ops` has the linear layers and the residual norms, :class:`AdamW` the optimizer step; their
methods have the names of the C entry points that they call.  Everything is computed by the CUDA
kernels of ``libegeria.so``; there is no fallback: a call that the library refuses raises
:class:`~paper_2201_06227_b200.binding.EgeriaError`, a tensor that it cannot take ``ValueError``.

Results are allocated on the stream that the call runs on.  Where a ``stream`` is given that is
not the current one, the caller orders it after the kernels that made the inputs, and the inputs
are recorded on it (their memory is not reused before the call has run).  What a handle itself holds
is recorded on every stream that it is called on; it may be dropped with calls in flight.

Autograd does not follow the calls: the gradients are the results of the ``*_backward`` methods.  Where it follows an
input of a forward call, going back through the result raises an error (under ``torch.no_grad()`` results are plain
tensors).  ``out`` and the parameters that require grad when an :class:`AdamW` is made get a new version when a call
writes to them (frozen ones too: the mask is not read on the host; a replayed graph raises none).
"""
from __future__ import annotations

import ctypes
import importlib.util
from pathlib import Path
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
    "egeria_ops_create", "egeria_ops_destroy", "egeria_ops_device_status", "egeria_ops_launch_count", "egeria_ops_debug_stall_next",
    "egeria_linear_workspace_bytes", "egeria_linear_forward", "egeria_linear_backward",
    "egeria_norm_workspace_bytes", "egeria_norm_forward", "egeria_norm_backward",
    "egeria_adamw_workspace_bytes", "egeria_adamw_create", "egeria_adamw_destroy", "egeria_adamw_set_grads",
    "egeria_adamw_step", "egeria_adamw_device_status", "egeria_adamw_launch_count",
]

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class _AdamTensor(ctypes.Structure):
    _fields_ = [(f, t) for t, names in ((_vp, "param master m v m_scale v_scale"), (_i64, "n"), (_i32, "param_type grad_type"),
                                        (_f32, "weight_decay"), (_i32, "module")) for f in names.split()]


_calls = None


def _native():
    """The extension module that marshals the calls (it needs torch's libraries, which `import torch` has loaded)."""
    global _calls
    if _calls is None:
        path = Path(__file__).resolve().parent / "_ops_python.so"
        if not path.exists():
            raise ImportError(f"{path} is missing: build it with `python -m paper_2201_06227_b200.build`")
        spec = importlib.util.spec_from_file_location("_ops_python", path)
        _calls = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(_calls)
    return _calls


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
    L.egeria_ops_debug_stall_next.argtypes = [_vp, ctypes.c_int]
    L.egeria_ops_create.argtypes = [ctypes.POINTER(_vp), _vp, ctypes.c_size_t]
    L.egeria_adamw_create.argtypes = [ctypes.POINTER(_vp), ctypes.c_int, ctypes.POINTER(_AdamTensor), ctypes.POINTER(_vp), _vp, _vp,
                                      ctypes.c_size_t, ctypes.c_uint32]
    for name in ("egeria_ops_destroy", "egeria_ops_device_status", "egeria_ops_launch_count", "egeria_adamw_destroy",
                 "egeria_adamw_device_status", "egeria_adamw_launch_count"):
        getattr(L, name).argtypes = [_vp]
    L.egeria_ops_launch_count.restype = L.egeria_adamw_launch_count.restype = _i64
    L.egeria_adamw_set_grads.argtypes = [_vp, _vp, ctypes.POINTER(_vp)]
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
    """The stream of a call that is not on the device's current stream: allocations inside come from it, and the
    tensors that the call touches are recorded on it."""

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream], tensors):
        self.stream = torch.cuda.current_stream(device) if stream is None else stream
        if self.stream.device != device:
            raise ValueError(f"the stream is of {self.stream.device}, the handle of {device}")
        self.tensors = () if stream is None else tensors
        self.context = torch.cuda.stream(self.stream)

    def __enter__(self):
        self.context.__enter__()
        return int(self.stream.cuda_stream)

    def __exit__(self, *exc):
        for t in self.tensors:
            if t is not None:
                t.record_stream(self.stream)
        return self.context.__exit__(*exc)


def _vector(t: Optional[torch.Tensor], name: str, device: int, dtype, n: int) -> int:
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != device or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: expected {n} consecutive {dtype} on cuda:{device}")
    return t.data_ptr()


class _Handle:
    """A library object on one device, with its workspace."""

    def _call(self, name, native, stream, args):
        """One call through the extension: its results, or EgeriaError."""
        entry = self._entry.get(name)
        if entry is None:
            entry = self._entry[name] = ctypes.cast(getattr(self._lib, name), _vp).value
        if stream is None and torch._C._cuda_getDevice() == self._index:
            raw = torch._C._cuda_getCurrentRawStream(self._index)
            if raw not in self._streams:
                self._join(raw)
            got = native(entry, self._h.value, self._index, raw, *args)
        else:
            with _On(self.device, stream, (self._raw, *self._touched(), *(a for a in args if isinstance(a, torch.Tensor)))) as s:
                got = native(entry, self._h.value, self._index, s, *args)
        if got.__class__ is int and got:
            _check(got, name)
        return got

    def _touched(self):
        return ()

    def _join(self, raw: int) -> None:
        """The first call on another stream than the one that the handle was made on: what the handle holds is recorded on
        it, so that its memory is not reused before that stream's calls have run, even if the handle is dropped."""
        if raw in self._streams:
            return
        stream = self._streams[raw] = torch.cuda.current_stream(self.device)
        for t in (self._raw, *self._touched()):
            if t is not None:
                t.record_stream(stream)

    def _place(self, device) -> None:
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("a CUDA device is required")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self._entry = {}
        self._streams = {torch._C._cuda_getCurrentRawStream(self._index): None}   # the ones that have the handle's memory on record

    def close(self) -> None:
        if getattr(self, "_h", None):
            self._destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Ops(_Handle):
    """Handle of the linear and norm calls; owns its workspace.  For one stream at a time."""

    def __init__(self, workspace_bytes: int = OPS_WORKSPACE_MIN, device="cuda"):
        self._place(device)
        self.workspace_bytes = max(int(workspace_bytes), OPS_WORKSPACE_MIN)
        self._raw, ptr = _workspace(self.workspace_bytes, self.device)
        handle = _vp()
        L = lib()
        with torch.cuda.device(self.device):
            _check(L.egeria_ops_create(ctypes.byref(handle), ptr, self.workspace_bytes), "egeria_ops_create")
        self._h, self._lib, self._destroy, self._native = handle, L, L.egeria_ops_destroy, _native()

    # ------------------------------------------------------------------ linear layers
    def egeria_linear_forward(self, x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
                              residual: Optional[torch.Tensor] = None, save_z: bool = False, out: Optional[torch.Tensor] = None,
                              stream: Optional[torch.cuda.Stream] = None):
        """y = act(x w^T + bias) + residual for x [rows, inp] and w [out, inp] in bfloat16 or float16; (y, z) with
        save_z, z the argument of the activation.  `out` may be the residual; it is refused where it overlaps anything else."""
        if act not in ACTS:
            raise ValueError(f"unknown activation {act!r}")
        return self._call("egeria_linear_forward", self._native.linear_forward, stream, (x, w, bias, ACTS[act], residual, save_z, out))

    def egeria_linear_backward(self, dy: torch.Tensor, x: Optional[torch.Tensor], w: Optional[torch.Tensor],
                               z: Optional[torch.Tensor] = None, act: str = "none", z_in: Optional[torch.Tensor] = None,
                               act_in: str = "none", need_dx: bool = True, need_dw: bool = True, need_db: bool = True,
                               stream: Optional[torch.cuda.Stream] = None):
        """(dx, dw, db) of a linear layer, None for what is not needed: a frozen layer takes need_dw = need_db = False and
        no x, the first layer that still trains need_dx = False and no w.  With act_in and z_in, dx is the gradient of
        z_in, x having come out of act_in(z_in)."""
        if act not in ACTS or act_in not in ACTS:
            raise ValueError(f"unknown activation {act!r} or {act_in!r}")
        return self._call("egeria_linear_backward", self._native.linear_backward, stream,
                          (dy, x, w, z, ACTS[act], z_in, ACTS[act_in], need_dx, need_dw, need_db))

    # ------------------------------------------------------------------ residual norms
    def egeria_norm_forward(self, x: torch.Tensor, f: torch.Tensor, gate: Optional[torch.Tensor] = None, gate_rows: int = 0,
                            w_post: Optional[torch.Tensor] = None, b_post: Optional[torch.Tensor] = None,
                            w_pre: Optional[torch.Tensor] = None, b_pre: Optional[torch.Tensor] = None, kind: str = "layer",
                            post: bool = True, pre: bool = True, alpha: float = 1.0, eps: float = 1e-5,
                            stream: Optional[torch.cuda.Stream] = None):
        """(y, h, stats): y = alpha x + gate * N_post(f), h = N_pre(y) (None without pre), stats for the backward call."""
        if kind not in KINDS:
            raise ValueError(f"unknown norm {kind!r}")
        return self._call("egeria_norm_forward", self._native.norm_forward, stream,
                          (x, f, gate, w_post, b_post, w_pre, b_pre, gate_rows, KINDS[kind], post, pre, alpha, eps))

    def egeria_norm_backward(self, dy: torch.Tensor, dh: Optional[torch.Tensor], y: torch.Tensor, f: torch.Tensor,
                             stats: torch.Tensor, gate: Optional[torch.Tensor] = None, gate_rows: int = 0,
                             w_post: Optional[torch.Tensor] = None, b_post: Optional[torch.Tensor] = None,
                             w_pre: Optional[torch.Tensor] = None, b_pre: Optional[torch.Tensor] = None, kind: str = "layer",
                             post: bool = True, pre: bool = True, alpha: float = 1.0, need_params: bool = True,
                             stream: Optional[torch.cuda.Stream] = None):
        """The gradients as a dict: dx, df, and for what is given (and with need_params) dgate, dw_post, db_post, dw_pre,
        db_pre, else None."""
        if kind not in KINDS:
            raise ValueError(f"unknown norm {kind!r}")
        got = self._call("egeria_norm_backward", self._native.norm_backward, stream,
                         (dy, dh, y, f, stats, gate, w_post, b_post, w_pre, b_pre, gate_rows, KINDS[kind], post, pre, alpha, need_params))
        return dict(zip(("dx", "df", "dgate", "dw_post", "db_post", "dw_pre", "db_pre"), got))

    def egeria_ops_device_status(self) -> int:
        with torch.cuda.device(self.device):
            return int(self._lib.egeria_ops_device_status(self._h))

    def check_device_status(self) -> None:
        _check(self.egeria_ops_device_status(), "egeria_ops_device_status")

    def egeria_ops_debug_stall_next(self, kind: int) -> None:
        """Test hook: the next product on the tensor cores gives up (see the header)."""
        _check(self._lib.egeria_ops_debug_stall_next(self._h, int(kind)), "egeria_ops_debug_stall_next")

    def egeria_ops_launch_count(self) -> int:
        return int(self._lib.egeria_ops_launch_count(self._h))


class AdamW(_Handle):
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
        self._place(params[0].device)
        dev = self._index
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
            row.param = _vector(p, f"params[{i}]", dev, p.dtype, k)
            row.master = _vector(columns["masters"][i], f"masters[{i}]", dev, torch.float32, k)
            row.m = _vector(exp_avg[i], f"exp_avg[{i}]", dev, torch.int8 if small else torch.float32, k)
            row.v = _vector(exp_avg_sq[i], f"exp_avg_sq[{i}]", dev, torch.uint8 if small else torch.float32, k)
            row.m_scale = _vector(columns["m_scales"][i], f"m_scales[{i}]", dev, torch.float32, blocks)
            row.v_scale = _vector(columns["v_scales"][i], f"v_scales[{i}]", dev, torch.float32, blocks)
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
                                             _vector(steps, "steps", dev, torch.int32, n), ptr, nbytes, flags),
                   "egeria_adamw_create")
        self._grads = list(grads)
        self._h, self._lib, self._destroy, self._native = handle, lib(), lib().egeria_adamw_destroy, _native()
        self._last_module = max(self.modules)
        self._followed = [p for p in params if p.requires_grad]

    def _grad_pointers(self, grads):
        if len(grads) != len(self._sizes):
            raise ValueError("grads: one entry per tensor is required")
        return (_vp * len(grads))(*[_vector(g, f"grads[{i}]", self._index, t, n) for i, (g, (n, t)) in enumerate(zip(grads, self._sizes))])

    def egeria_adamw_set_grads(self, grads: Sequence[torch.Tensor], stream: Optional[torch.cuda.Stream] = None) -> None:
        """The gradients (same sizes and types) are in these tensors from the next step on."""
        ptrs = self._grad_pointers(grads)
        if stream is None:
            self._join(torch._C._cuda_getCurrentRawStream(self._index))
        with _On(self.device, stream, (self._raw,)) as s:
            _check(self._lib.egeria_adamw_set_grads(self._h, s, ptrs), "egeria_adamw_set_grads")
        self._grads = list(grads)      # not before the library has taken them: until then the old ones are in force
        for known in self._streams.values():
            for g in grads if known is not None else ():
                g.record_stream(known)

    def egeria_adamw_step(self, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                          grad_scale: Optional[torch.Tensor] = None, frozen: Optional[torch.Tensor] = None,
                          stream: Optional[torch.cuda.Stream] = None) -> None:
        """One step of every tensor whose module is not marked in `frozen` (uint8, as egeria_plasticity_evaluate leaves it)."""
        self._call("egeria_adamw_step", self._native.adamw_step, stream, (lr, beta1, beta2, eps, grad_scale, frozen, self._last_module))
        if self._followed:
            torch.autograd.graph.increment_version(self._followed)

    def _touched(self):
        return [self._steps, *self._grads, *(t for column in self._keep for t in column)]

    def egeria_adamw_device_status(self) -> int:
        with torch.cuda.device(self.device):
            return int(self._lib.egeria_adamw_device_status(self._h))

    def check_device_status(self) -> None:
        _check(self.egeria_adamw_device_status(), "egeria_adamw_device_status")

    def egeria_adamw_launch_count(self) -> int:
        return int(self._lib.egeria_adamw_launch_count(self._h))
