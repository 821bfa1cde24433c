"""Operators around the optimizer step, over torch tensors on an MI355X.

  Orthogonalizer   lists of matrices made orthogonal by Newton-Schulz products

PyTorch supplies device memory and the current stream only; the work is the HIP
library's (``_ops``). Argument errors raise ``ValueError`` or ``TypeError`` here,
or ``LambError`` from the library.
"""

from __future__ import annotations

from typing import Optional, Sequence, Tuple

from . import _lib, _ops

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _torch():
    import torch
    return torch


def _stream(device) -> int:
    return _torch().cuda.current_stream(device).cuda_stream


def _float_code(dtype) -> int:
    torch = _torch()
    if dtype == torch.float32:
        return _ops.LAMB_DTYPE_F32
    if dtype == torch.bfloat16:
        return _ops.LAMB_DTYPE_BF16
    raise TypeError("need float32 or bfloat16, got %s" % dtype)


def _on_gpu(name, t, device=None):
    if t.device.type != "cuda":
        raise ValueError("%s must live on a GPU" % name)
    if device is not None and t.device != device:
        raise ValueError("%s is on another device" % name)


class Orthogonalizer:
    """X of each input G after ``steps`` times X <- (a I + b A + c A A) X, A = X X^T,
    from X = G / (||G||_F + eps): G with its singular values moved towards 1.

    ``inputs`` and ``outputs`` are persistent 2-D tensors (float32 or bfloat16, one
    type each, rows contiguous); ``run()`` reads the inputs as they are then. An
    output may be its own input. ``precision``: "half" rounds the products' operands
    to 16-bit floats with 11 significant bits (the result is 1e-3 to 7e-3 off),
    "split" to pairs of them (as fp32, three times the work); by default "half" for
    bfloat16 outputs, whose own rounding is 1.7e-3, and "split" for float32 ones.
    The plan keeps a workspace of about 4 bytes per element (8 for "split").
    """

    def __init__(self, inputs: Sequence, outputs: Optional[Sequence] = None, steps: int = 5,
                 coefficients: Tuple[float, float, float] = COEFFICIENTS, eps: float = 1e-7,
                 precision: Optional[str] = None):
        torch = _torch()
        self.inputs = list(inputs)
        if not self.inputs:
            raise ValueError("need at least one matrix")
        self.outputs = ([torch.empty_like(t, memory_format=torch.contiguous_format)
                         for t in self.inputs] if outputs is None else list(outputs))
        if len(self.outputs) != len(self.inputs):
            raise ValueError("need one output per input (got %d and %d)"
                             % (len(self.outputs), len(self.inputs)))
        self.device = self.inputs[0].device
        rows = []
        for i, (a, b) in enumerate(zip(self.inputs, self.outputs)):
            for name, t, first in (("input", a, self.inputs[0]), ("output", b, self.outputs[0])):
                _on_gpu("%s %d" % (name, i), t, self.device)
                if t.dtype != first.dtype:
                    raise TypeError("all %ss must share one dtype" % name)
                if t.dim() != 2 or t.numel() == 0:
                    raise ValueError("%s %d is not a matrix, or is empty" % (name, i))
                if t.shape[1] > 1 and t.stride(1) != 1:
                    raise ValueError("%s %d: the elements of a row must be adjacent" % (name, i))
            if a.shape != b.shape:
                raise ValueError("matrix %d: input and output shapes differ" % i)
            r, c = a.shape
            rows.append((a.data_ptr(), b.data_ptr(), r, c, *(t.stride(0) if r > 1 else c
                                                            for t in (a, b))))
        if precision is None:
            precision = "half" if self.outputs[0].dtype == torch.bfloat16 else "split"
        if precision not in _ops.PRECISIONS:
            raise ValueError("precision must be one of %s" % (tuple(_ops.PRECISIONS),))
        self.precision = precision
        self.params = _ops.lamb_ns_params_init(steps=int(steps), a=coefficients[0],
                                               b=coefficients[1], c=coefficients[2], eps=eps)
        with torch.cuda.device(self.device):
            self.plan = _ops.lamb_ortho_plan_create(
                rows, _float_code(self.inputs[0].dtype), _float_code(self.outputs[0].dtype),
                _ops.PRECISIONS[precision])

    def run(self) -> list:
        """Enqueue the products on the current stream; returns the outputs."""
        _ops.lamb_orthogonalize(self.plan, self.params, _stream(self.device))
        return self.outputs

    def close(self) -> None:
        self.plan.close()
