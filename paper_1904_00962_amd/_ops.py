"""ctypes binding of the operators of ``liblamb_mi355x.so`` (include/lamb_ops.h).

Argument marshalling only, as in ``_lib``: the functions keep the C names, take
device pointers as integers and raise :class:`_lib.LambError` on failure.
"""

from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Tuple

from . import _lib
from ._lib import _check, _vp

LAMB_DTYPE_F32 = 0
LAMB_DTYPE_BF16 = 1
LAMB_DTYPE_I32 = 2
LAMB_DTYPE_I64 = 3

LAMB_NS_HALF = 0
LAMB_NS_SPLIT = 1
PRECISIONS = {"half": LAMB_NS_HALF, "split": LAMB_NS_SPLIT}

LAMB_MUON_RMS = 0
LAMB_MUON_SPECTRAL = 1
LAMB_MUON_UNIT = 2
SCALES = {"rms": LAMB_MUON_RMS, "spectral": LAMB_MUON_SPECTRAL, "unit": LAMB_MUON_UNIT}

# Every symbol include/lamb_ops.h declares (checked by the test suite).
EXPORTS = ("lamb_ns_params_init", "lamb_ortho_plan_create", "lamb_orthogonalize",
           "lamb_muon_plan_create", "lamb_muon_hparams_init", "lamb_muon_check", "lamb_muon_step",
           "lamb_ns_plan_destroy", "lamb_xent_workspace", "lamb_xent_forward",
           "lamb_xent_backward", "lamb_embed_forward", "lamb_embed_workspace",
           "lamb_embed_backward", "lamb_rms_forward", "lamb_rms_quantize", "lamb_rms_workspace",
           "lamb_rms_backward", "lamb_grad_plan_create", "lamb_grad_norm", "lamb_grad_clip",
           "lamb_grad_norm_clip", "lamb_grad_plan_destroy")


class lamb_ns_params(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int32), ("a", ctypes.c_float), ("b", ctypes.c_float),
                ("c", ctypes.c_float), ("eps", ctypes.c_float), ("reserved", ctypes.c_int32)]


class lamb_matrix(ctypes.Structure):
    _fields_ = [("input", ctypes.c_void_p), ("out", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("in_stride", ctypes.c_int64),
                ("out_stride", ctypes.c_int64)]


class lamb_muon_tensor(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("wd", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class lamb_muon_hparams(ctypes.Structure):
    _fields_ = [("ns", lamb_ns_params), ("lr", ctypes.c_float), ("momentum", ctypes.c_double),
                ("weight_decay", ctypes.c_float), ("grad_scale", ctypes.c_float),
                ("nesterov", ctypes.c_int32), ("scale", ctypes.c_int32),
                ("skip_nonfinite", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class lamb_xent(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("targets", ctypes.c_void_p), ("hidden_stride", ctypes.c_int64),
                ("table_stride", ctypes.c_int64), ("tokens", ctypes.c_int64),
                ("vocab", ctypes.c_int64), ("dim", ctypes.c_int64),
                ("ignore_index", ctypes.c_int64), ("target_dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class lamb_xent_grads(ctypes.Structure):
    _fields_ = [("grad_loss", ctypes.c_void_p), ("grad_hidden", ctypes.c_void_p),
                ("grad_table", ctypes.c_void_p), ("grad_hidden_stride", ctypes.c_int64),
                ("grad_table_stride", ctypes.c_int64), ("grad_table_dtype", ctypes.c_int32),
                ("add_table", ctypes.c_int32), ("mean", ctypes.c_int32),
                ("grad_scale", ctypes.c_float)]


class lamb_embed(ctypes.Structure):
    _fields_ = [("ids", ctypes.c_void_p), ("tokens", ctypes.c_int64), ("vocab", ctypes.c_int64),
                ("dim", ctypes.c_int64), ("id_dtype", ctypes.c_int32), ("scale", ctypes.c_float)]


class lamb_rms(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("residual", ctypes.c_void_p),
                ("weight", ctypes.c_void_p), ("x_stride", ctypes.c_int64),
                ("residual_stride", ctypes.c_int64), ("tokens", ctypes.c_int64),
                ("dim", ctypes.c_int64), ("x_dtype", ctypes.c_int32),
                ("residual_dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32),
                ("eps", ctypes.c_float)]


class lamb_rms_grads(ctypes.Structure):
    _fields_ = [("grad_out", ctypes.c_void_p), ("grad_sum", ctypes.c_void_p),
                ("grad_x", ctypes.c_void_p), ("grad_weight", ctypes.c_void_p),
                ("grad_out_stride", ctypes.c_int64), ("grad_sum_stride", ctypes.c_int64),
                ("grad_x_stride", ctypes.c_int64), ("grad_out_dtype", ctypes.c_int32),
                ("grad_x_dtype", ctypes.c_int32), ("grad_weight_dtype", ctypes.c_int32),
                ("add_weight", ctypes.c_int32), ("reserved", ctypes.c_int64)]


class lamb_grad_tensor(ctypes.Structure):
    _fields_ = [("input", ctypes.c_void_p), ("out", ctypes.c_void_p), ("numel", ctypes.c_int64),
                ("in_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32)]


_lib_ops: Optional[ctypes.CDLL] = None


def load() -> ctypes.CDLL:
    """The library with the operators' signatures set."""
    global _lib_ops
    if _lib_ops is not None:
        return _lib_ops
    lib = _lib.load()
    i32, vp, P = ctypes.c_int32, ctypes.c_void_p, ctypes.POINTER
    size = ctypes.c_size_t
    lib.lamb_ns_params_init.argtypes = [P(lamb_ns_params)]
    lib.lamb_ortho_plan_create.argtypes = [P(lamb_matrix), i32, i32, i32, i32, P(vp)]
    lib.lamb_orthogonalize.argtypes = [vp, P(lamb_ns_params), vp]
    lib.lamb_muon_plan_create.argtypes = [P(lamb_muon_tensor), i32, i32, i32, P(vp)]
    lib.lamb_muon_hparams_init.argtypes = [P(lamb_muon_hparams)]
    lib.lamb_muon_check.argtypes = [vp, P(lamb_muon_hparams)]
    lib.lamb_muon_step.argtypes = [vp, P(lamb_muon_hparams), vp, vp]
    lib.lamb_ns_plan_destroy.argtypes = [vp]
    lib.lamb_xent_workspace.argtypes = [P(lamb_xent), P(size), P(size)]
    lib.lamb_xent_forward.argtypes = [P(lamb_xent), vp, vp, vp, vp, size, vp]
    lib.lamb_xent_backward.argtypes = [P(lamb_xent), vp, P(lamb_xent_grads), vp, size, vp]
    i64 = ctypes.c_int64
    lib.lamb_embed_forward.argtypes = [P(lamb_embed), vp, i64, i32, vp, i64, i32, vp]
    lib.lamb_embed_workspace.argtypes = [P(lamb_embed), P(size)]
    lib.lamb_embed_backward.argtypes = [P(lamb_embed), vp, i64, i32, vp, i64, i32, i64, i32, vp,
                                        size, vp]
    lib.lamb_rms_forward.argtypes = [P(lamb_rms), vp, i64, vp, i64, i32, vp]
    lib.lamb_rms_quantize.argtypes = [P(lamb_rms), vp, i64, vp, i64, vp, i32, vp]
    lib.lamb_rms_workspace.argtypes = [P(lamb_rms), P(size)]
    lib.lamb_rms_backward.argtypes = [P(lamb_rms), P(lamb_rms_grads), vp, size, vp]
    f64 = ctypes.c_double
    lib.lamb_grad_plan_create.argtypes = [P(lamb_grad_tensor), i32, i32, P(vp)]
    lib.lamb_grad_norm.argtypes = [vp, vp, vp, vp]
    lib.lamb_grad_clip.argtypes = [vp, vp, f64, f64, vp, vp]
    lib.lamb_grad_norm_clip.argtypes = [vp, vp, vp, f64, f64, vp, vp]
    lib.lamb_grad_plan_destroy.argtypes = [vp]
    for name in EXPORTS:
        getattr(lib, name).restype = ctypes.c_int
    _lib_ops = lib
    return lib


class NsPlan(_lib.Plan):
    """Owning handle on a ``lamb_ns_plan``."""

    def close(self) -> None:
        if self.handle:
            h, self.handle = self.handle, 0
            _check(load().lamb_ns_plan_destroy(_vp(h)), "lamb_ns_plan_destroy")


def _set(struct, fields) -> None:
    for k, v in fields.items():
        if not hasattr(struct, k):
            raise AttributeError("%s has no field %r" % (type(struct).__name__, k))
        setattr(struct, k, v)


def lamb_ns_params_init(**fields) -> lamb_ns_params:
    """The defaults, then ``fields`` set by name."""
    p = lamb_ns_params()
    _check(load().lamb_ns_params_init(ctypes.byref(p)), "lamb_ns_params_init")
    _set(p, fields)
    return p


def lamb_muon_hparams_init(ns: Optional[lamb_ns_params] = None, **fields) -> lamb_muon_hparams:
    """The defaults, then ``ns`` and ``fields`` set by name (``scale`` may be "rms",
    "spectral" or "unit")."""
    hp = lamb_muon_hparams()
    _check(load().lamb_muon_hparams_init(ctypes.byref(hp)), "lamb_muon_hparams_init")
    if ns is not None:
        hp.ns = ns
    if isinstance(fields.get("scale"), str):
        fields["scale"] = SCALES[fields["scale"]]
    _set(hp, fields)
    return hp


def lamb_ortho_plan_create(matrices: Sequence[Tuple[int, int, int, int, int, int]], in_dtype: int,
                           out_dtype: int, precision: int) -> NsPlan:
    """matrices: (in_ptr, out_ptr, rows, cols, in_stride, out_stride) each."""
    n = len(matrices)
    arr = (lamb_matrix * max(n, 1))()
    for i, (a, b, rows, cols, sa, sb) in enumerate(matrices):
        arr[i] = lamb_matrix(int(a) or None, int(b) or None, int(rows), int(cols), int(sa), int(sb))
    out = ctypes.c_void_p()
    _check(load().lamb_ortho_plan_create(arr, n, int(in_dtype), int(out_dtype), int(precision),
                                         ctypes.byref(out)), "lamb_ortho_plan_create")
    return NsPlan(out.value)


def lamb_orthogonalize(plan: NsPlan, params: lamb_ns_params, stream: int = 0) -> None:
    _check(load().lamb_orthogonalize(_vp(plan.handle), ctypes.byref(params), _vp(stream)),
           "lamb_orthogonalize")


def lamb_muon_plan_create(tensors: Sequence[Tuple[int, int, int, int, int, int]], g_dtype: int,
                          precision: int) -> NsPlan:
    """tensors: (x_ptr, g_ptr, m_ptr, rows, cols, wd) each."""
    n = len(tensors)
    arr = (lamb_muon_tensor * max(n, 1))()
    for i, (x, g, m, rows, cols, wd) in enumerate(tensors):
        arr[i] = lamb_muon_tensor(int(x) or None, int(g) or None, int(m) or None, int(rows),
                                  int(cols), int(wd), 0)
    out = ctypes.c_void_p()
    _check(load().lamb_muon_plan_create(arr, n, int(g_dtype), int(precision), ctypes.byref(out)),
           "lamb_muon_plan_create")
    return NsPlan(out.value)


def lamb_muon_check(plan: NsPlan, hp: lamb_muon_hparams) -> None:
    """Raise what ``lamb_muon_step`` would of these before any HIP call (host only)."""
    _check(load().lamb_muon_check(_vp(plan.handle), ctypes.byref(hp)), "lamb_muon_check")


def lamb_muon_step(plan: NsPlan, hp: lamb_muon_hparams, stream: int = 0,
                   nonfinite_out: int = 0) -> None:
    _check(load().lamb_muon_step(_vp(plan.handle), ctypes.byref(hp), _vp(stream),
                                 _vp(nonfinite_out)), "lamb_muon_step")


def lamb_xent_workspace(xent: lamb_xent, backward: bool) -> int:
    """Bytes that a forward or a backward call needs."""
    n = ctypes.c_size_t()
    to = (None, ctypes.byref(n)) if backward else (ctypes.byref(n), None)
    _check(load().lamb_xent_workspace(ctypes.byref(xent), *to), "lamb_xent_workspace")
    return n.value


def lamb_xent_forward(xent: lamb_xent, loss: int, lse: int, mean: int, workspace: int,
                      workspace_bytes: int, stream: int = 0) -> None:
    _check(load().lamb_xent_forward(ctypes.byref(xent), loss, lse, mean, workspace,
                                    workspace_bytes, stream), "lamb_xent_forward")


def lamb_xent_backward(xent: lamb_xent, lse: int, grads: lamb_xent_grads, workspace: int,
                       workspace_bytes: int, stream: int = 0) -> None:
    _check(load().lamb_xent_backward(ctypes.byref(xent), lse, ctypes.byref(grads), workspace,
                                     workspace_bytes, stream), "lamb_xent_backward")


def lamb_embed_forward(embed: lamb_embed, table: int, table_stride: int, table_dtype: int, out: int,
                       out_stride: int, out_dtype: int, stream: int = 0) -> None:
    _check(load().lamb_embed_forward(ctypes.byref(embed), table, table_stride, table_dtype, out,
                                     out_stride, out_dtype, stream), "lamb_embed_forward")


def lamb_embed_workspace(embed: lamb_embed) -> int:
    n = ctypes.c_size_t()
    _check(load().lamb_embed_workspace(ctypes.byref(embed), ctypes.byref(n)),
           "lamb_embed_workspace")
    return n.value


def lamb_embed_backward(embed: lamb_embed, grad_out: int, grad_out_stride: int,
                        grad_out_dtype: int, grad_table: int, grad_table_stride: int,
                        grad_table_dtype: int, padding_id: int, add: int, workspace: int,
                        workspace_bytes: int, stream: int = 0) -> None:
    _check(load().lamb_embed_backward(ctypes.byref(embed), grad_out, grad_out_stride,
                                      grad_out_dtype, grad_table, grad_table_stride,
                                      grad_table_dtype, padding_id, add, workspace,
                                      workspace_bytes, stream), "lamb_embed_backward")


def lamb_rms_forward(rms: lamb_rms, summed: int, summed_stride: int, out: int, out_stride: int,
                     out_dtype: int, stream: int = 0) -> None:
    _check(load().lamb_rms_forward(ctypes.byref(rms), summed, summed_stride, out, out_stride,
                                   out_dtype, stream), "lamb_rms_forward")


def lamb_rms_quantize(rms: lamb_rms, summed: int, summed_stride: int, out: int, out_stride: int,
                      scales: int, group: int, stream: int = 0) -> None:
    _check(load().lamb_rms_quantize(ctypes.byref(rms), summed, summed_stride, out, out_stride,
                                    scales, group, stream), "lamb_rms_quantize")


def lamb_rms_workspace(rms: lamb_rms) -> int:
    n = ctypes.c_size_t()
    _check(load().lamb_rms_workspace(ctypes.byref(rms), ctypes.byref(n)), "lamb_rms_workspace")
    return n.value


def lamb_rms_backward(rms: lamb_rms, grads: lamb_rms_grads, workspace: int, workspace_bytes: int,
                      stream: int = 0) -> None:
    _check(load().lamb_rms_backward(ctypes.byref(rms), ctypes.byref(grads), workspace,
                                    workspace_bytes, stream), "lamb_rms_backward")


class GradPlan(_lib.Plan):
    """Owning handle on a ``lamb_grad_plan``."""

    def close(self) -> None:
        if self.handle:
            h, self.handle = self.handle, 0
            _check(load().lamb_grad_plan_destroy(_vp(h)), "lamb_grad_plan_destroy")


def lamb_grad_plan_create(tensors: Sequence[Tuple[int, int, int, int, int]],
                          norm: int) -> GradPlan:
    """tensors: (in_ptr, out_ptr, numel, in_dtype, out_dtype) each."""
    n = len(tensors)
    arr = (lamb_grad_tensor * max(n, 1))()
    for t, (a, b, numel, in_dtype, out_dtype) in zip(arr, tensors):
        t.input, t.out, t.numel = a or None, b or None, numel
        t.in_dtype, t.out_dtype = in_dtype, out_dtype
    out = ctypes.c_void_p()
    _check(load().lamb_grad_plan_create(arr, n, int(norm), ctypes.byref(out)),
           "lamb_grad_plan_create")
    return GradPlan(out.value)


def lamb_grad_norm(plan: GradPlan, norms: int, total: int, stream: int = 0) -> None:
    _check(load().lamb_grad_norm(plan.handle, norms, total, stream), "lamb_grad_norm")


def lamb_grad_clip(plan: GradPlan, total: int, max_norm: float, scale: float = 1.0,
                   nonfinite_out: int = 0, stream: int = 0) -> None:
    _check(load().lamb_grad_clip(plan.handle, total, max_norm, scale, nonfinite_out, stream),
           "lamb_grad_clip")


def lamb_grad_norm_clip(plan: GradPlan, norms: int, total: int, max_norm: float,
                        scale: float = 1.0, nonfinite_out: int = 0, stream: int = 0) -> None:
    _check(load().lamb_grad_norm_clip(plan.handle, norms, total, max_norm, scale, nonfinite_out,
                                      stream), "lamb_grad_norm_clip")
