"""Operators around the optimizer step, over torch tensors on an MI355X.

  Orthogonalizer            lists of matrices made orthogonal by Newton-Schulz products
  linear_cross_entropy      softmax cross entropy against a vocabulary table, and
  linear_cross_entropy_grad its gradients, without keeping the logits
  embedding                 rows of a token table, scaled
  embedding_grad            the table's gradient, summed in the tokens' order
  rms_norm                  root-mean-square norm, after the residual's addition,
  rms_norm_fp8              its result in 8 bits with scales, and
  rms_norm_grad             its gradients
  GradNorm                  the norm of all gradients of a model, and clipping by it

PyTorch supplies device memory and the current stream only; the work is the HIP
library's (``_ops``). Argument errors raise ``ValueError`` or ``TypeError`` here,
or ``LambError`` from the library.
"""

from __future__ import annotations

from typing import Optional, Sequence, Tuple

from . import _lib, _ops

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


_torch_module = None
_FLOAT_CODES = {}
_ID_CODES = {}
# what a call asks torch for each time: the current device's index, and a stream's raw handle
_current_device = _raw_stream = None


def _torch():
    global _torch_module, _current_device, _raw_stream
    if _torch_module is None:
        import torch
        # without torch's look whether CUDA is there (a tensor lies on a device), and without a
        # Stream object, which costs 4 us a call; where torch has them
        _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda index: torch.cuda.current_stream(index).cuda_stream)
        _FLOAT_CODES.update({torch.float32: _ops.LAMB_DTYPE_F32,
                             torch.bfloat16: _ops.LAMB_DTYPE_BF16})
        _ID_CODES.update({torch.int32: _ops.LAMB_DTYPE_I32, torch.int64: _ops.LAMB_DTYPE_I64})
        _torch_module = torch
    return _torch_module


def _stream(device) -> int:
    _torch()
    return _raw_stream(device.index)


class _NoSwitch:
    def __enter__(self):
        return self

    def __exit__(self, *exc):
        return False


_NO_SWITCH = _NoSwitch()


def _on(device):
    """A context on ``device``; nothing where it is current already."""
    torch = _torch()
    return _NO_SWITCH if _current_device() == device.index else torch.cuda.device(device)


def _float_code(dtype) -> int:
    code = _FLOAT_CODES.get(dtype)
    if code is None:
        raise TypeError("need float32 or bfloat16, got %s" % dtype)
    return code


def _on_gpu(name, t, device=None):
    if not t.is_cuda:
        raise ValueError("%s must live on a GPU" % name)
    if device is not None and t.device != device:
        raise ValueError("%s is on another device" % name)


def _no_graph(name, *tensors):
    """The operators record nothing for autograd: a result whose gradient would be lost
    without a word is refused."""
    if not _torch().is_grad_enabled():
        return
    for t in tensors:
        if t is None or not t.requires_grad:
            continue
        raise ValueError("%s records no gradient for a tensor that requires one: pass "
                         "tensor.detach(), or call it under torch.no_grad(), and take the "
                         "gradient from %s_grad" % (name, name.removesuffix("_fp8")))


class Orthogonalizer:
    """X of each input G after ``steps`` times X <- (a I + b A + c A A) X, A = X X^T,
    from X = G / (||G||_F + eps): G with its singular values moved towards 1.

    ``inputs`` and ``outputs`` are persistent 2-D tensors (float32 or bfloat16, one
    type each, rows contiguous); ``run()`` reads the inputs as they are then. An
    output may be its own input.

    ``precision``: "split" (the default) rounds the products' operands to pairs of 16-bit
    floats (22 bits, an error as of fp32), "half" to one (11 bits, a third of the work).
    "half" has to be asked for: its error depends on the singular values. The steps
    multiply the small ones by up to 485 (by default), and the rounding of the large ones
    with them: 1.3e-3 off (2-norm, relative) for independent entries, 1e-2 where the
    singular values span decades, 1e-1 where a few outweigh the rest, as a network's
    gradients and momenta often have it.

    The plan keeps a workspace of about 4 bytes per element, and 4 to 12 per entry of the
    short sides' squares; twice that for "split". Calls share it, so one on another stream
    than the last waits for that one; replays of a captured call are the caller's to
    order, and so is what else uses the inputs and outputs.
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
        precision = "split" if precision is None else precision
        if precision not in _ops.PRECISIONS:
            raise ValueError("precision must be one of %s" % (tuple(_ops.PRECISIONS),))
        self.precision = precision
        self.params = _ops.lamb_ns_params_init(steps=int(steps), a=coefficients[0],
                                               b=coefficients[1], c=coefficients[2], eps=eps)
        with _on(self.device):
            self.plan = _ops.lamb_ortho_plan_create(
                rows, _float_code(self.inputs[0].dtype), _float_code(self.outputs[0].dtype),
                _ops.PRECISIONS[precision])

    def run(self) -> list:
        """Enqueue the products on the current stream; returns the outputs."""
        _ops.lamb_orthogonalize(self.plan, self.params, _stream(self.device))
        return self.outputs

    def close(self) -> None:
        self.plan.close()


def _rows(name, t, dtype, device=None):
    """A 2-D tensor whose rows are contiguous: its row stride."""
    if not t.is_cuda or (device is not None and t.device != device):
        _on_gpu(name, t, device)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.dim() != 2:
        raise ValueError("%s must have two dimensions" % name)
    rows, cols = t.shape
    stride, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("%s: the elements of a row must be adjacent" % name)
    return stride if rows > 1 else cols  # the stride of a single row means nothing


def _ids(name, t, device):
    _on_gpu(name, t, device)
    code = _ID_CODES.get(t.dtype)
    if code is None:
        raise TypeError("%s must be int32 or int64, got %s" % (name, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return code


def _xent(hidden, table, targets, ignore_index):
    torch = _torch()
    stride = _rows("hidden", hidden, torch.bfloat16)
    table_stride = _rows("table", table, torch.bfloat16, hidden.device)
    code = _ids("targets", targets, hidden.device)
    if hidden.shape[1] != table.shape[1]:
        raise ValueError("hidden has %d columns, the table %d" % (hidden.shape[1], table.shape[1]))
    if targets.dim() != 1 or targets.shape[0] != hidden.shape[0]:
        raise ValueError("need one target per row of hidden")
    return _ops.lamb_xent(hidden.data_ptr() or None, table.data_ptr() or None,
                          targets.data_ptr() or None, stride, table_stride, hidden.shape[0],
                          table.shape[0], hidden.shape[1], int(ignore_index), code, 0)


def _workspace(bytes_, device):
    return _torch().empty(bytes_, dtype=_torch().uint8, device=device)


def linear_cross_entropy(hidden, table, targets, *, ignore_index: int = -100):
    """(mean, loss, lse) of softmax cross entropy with logits hidden table^T, fp32.

    ``hidden`` [tokens, dim] and ``table`` [vocab, dim] are bfloat16 with contiguous
    rows, ``targets`` int32 or int64. Tokens whose target is ``ignore_index`` do not
    count: loss 0, and the mean is over the others (0 without any). A target outside
    the vocabulary gives NaN. ``lse`` is what :func:`linear_cross_entropy_grad` needs.

    Autograd does not see the call: tensors that require gradients are refused where
    grad mode is on (pass them detached).
    """
    torch = _torch()
    _no_graph("linear_cross_entropy", hidden, table)
    x = _xent(hidden, table, targets, ignore_index)
    need = _ops.lamb_xent_workspace(x, False)
    out = torch.empty(2, hidden.shape[0], dtype=torch.float32, device=hidden.device)
    mean = torch.empty((), dtype=torch.float32, device=hidden.device)
    work = _workspace(need, hidden.device)
    with _on(hidden.device):
        _ops.lamb_xent_forward(x, out[0].data_ptr(), out[1].data_ptr(), mean.data_ptr(),
                               work.data_ptr(), need, _stream(hidden.device))
    return mean, out[0], out[1]


def linear_cross_entropy_grad(hidden, table, targets, lse, grad_hidden=None, grad_table=None, *,
                              ignore_index: int = -100, reduction: str = "mean",
                              grad_loss=None, grad_scale: float = 1.0,
                              accumulate: bool = False) -> None:
    """Gradients of ``grad_scale`` x ``grad_loss`` x the mean or the sum (``reduction``)
    of the losses: into ``grad_hidden`` (bfloat16, like hidden) and ``grad_table``
    (bfloat16 or float32, like the table), either of them optional; ``accumulate`` adds
    to what ``grad_table`` holds. ``grad_loss``: a float32 tensor of one element on the
    device (default 1). ``lse`` is the forward's.

    The softmax is rounded to bfloat16 for bfloat16 gradients, which so are up to 2.5e-3
    off (1.7e-3 by their own rounding), and held in 16 bits for a float32 ``grad_table``,
    whose product takes twice as long."""
    torch = _torch()
    x = _xent(hidden, table, targets, ignore_index)
    device = hidden.device
    if lse.dtype != torch.float32 or lse.shape != targets.shape or not lse.is_contiguous():
        raise ValueError("lse must be the forward's")
    _on_gpu("lse", lse, device)
    if reduction not in ("mean", "sum"):
        raise ValueError("reduction must be 'mean' or 'sum'")
    g = _ops.lamb_xent_grads(mean=int(reduction == "mean"), grad_scale=float(grad_scale),
                             add_table=int(bool(accumulate)))
    if grad_loss is not None:
        _on_gpu("grad_loss", grad_loss, device)
        if grad_loss.dtype != torch.float32 or grad_loss.numel() != 1:
            raise TypeError("grad_loss must be one float32 element")
        g.grad_loss = grad_loss.data_ptr()
    if grad_hidden is not None:
        g.grad_hidden_stride = _rows("grad_hidden", grad_hidden, torch.bfloat16, device)
        if grad_hidden.shape != hidden.shape:
            raise ValueError("grad_hidden must have hidden's shape")
        g.grad_hidden = grad_hidden.data_ptr() or None
    if grad_table is not None:
        g.grad_table_dtype = _float_code(grad_table.dtype)
        g.grad_table_stride = _rows("grad_table", grad_table, grad_table.dtype, device)
        if grad_table.shape != table.shape:
            raise ValueError("grad_table must have the table's shape")
        g.grad_table = grad_table.data_ptr()
    need = _ops.lamb_xent_workspace(x, True)
    work = _workspace(need, device)
    with _on(device):
        _ops.lamb_xent_backward(x, lse.data_ptr(), g, work.data_ptr(), need, _stream(device))


def _embed(ids, table, scale, device):
    code = _ids("ids", ids, device)
    vocab, dim = table.shape
    return _ops.lamb_embed(ids.data_ptr() or None, ids.numel(), vocab, dim, code, scale)


def embedding(ids, table, *, scale: float = 1.0, out_dtype=None, out=None):
    """``scale`` x the rows of ``table`` [vocab, dim] (float32 or bfloat16) that ``ids``
    (int32 or int64, any shape) name: a tensor [*ids.shape, dim] of ``out_dtype`` (the
    table's by default), or ``out`` [ids.numel(), dim]. An id outside the table gives a
    row of NaN. Autograd does not see the call: a table that requires a gradient is refused
    where grad mode is on (pass it detached)."""
    torch = _torch()
    _no_graph("embedding", table, *(() if out is None else (out,)))
    device, dtype = table.device, table.dtype
    stride = _rows("table", table, dtype)
    e = _embed(ids, table, scale, device)
    if out is None:
        out_dtype = out_dtype or dtype
        out_code = _float_code(out_dtype)
        out_stride = e.dim
        result = torch.empty((*ids.shape, out_stride), dtype=out_dtype, device=device)
    else:
        result = out
        out_code = _float_code(out.dtype)
        out_stride = _rows("out", out, out_dtype or out.dtype, device)
        if out.shape != (e.tokens, e.dim):
            raise ValueError("out must be [%d, %d]" % (e.tokens, e.dim))
    with _on(device):
        _ops.lamb_embed_forward(e, table.data_ptr(), stride, _float_code(dtype),
                                result.data_ptr(), out_stride, out_code, _stream(device))
    return result


def embedding_grad(ids, grad_out, grad_table, *, scale: float = 1.0,
                   padding_id: Optional[int] = None, accumulate: bool = False) -> None:
    """The gradient of :func:`embedding` for its table into ``grad_table`` [vocab, dim]:
    row v becomes, or with ``accumulate`` grows by, ``scale`` x the sum of the rows of
    ``grad_out`` [ids.numel(), dim] whose id is v, in their order and in fp32. Either is
    float32 or bfloat16. Tokens with id ``padding_id``, or outside the table, add
    nothing."""
    _torch()
    device = grad_table.device
    stride = _rows("grad_table", grad_table, grad_table.dtype)
    out_stride = _rows("grad_out", grad_out, grad_out.dtype, device)
    e = _embed(ids, grad_table, scale, device)
    if grad_out.shape != (e.tokens, e.dim):
        raise ValueError("grad_out must be [%d, %d]" % (e.tokens, e.dim))
    out_code, code = _float_code(grad_out.dtype), _float_code(grad_table.dtype)
    need = _ops.lamb_embed_workspace(e)
    work = _workspace(need, device)
    with _on(device):
        _ops.lamb_embed_backward(e, grad_out.data_ptr(), out_stride, out_code,
                                 grad_table.data_ptr(), stride, code,
                                 -1 if padding_id is None else padding_id, bool(accumulate),
                                 work.data_ptr(), need, _stream(device))


def _rms(x, weight, residual, eps):
    """The C struct."""
    device, shape, dtype = x.device, x.shape, x.dtype
    stride = _like("x", x, shape, device)
    code = _float_code(dtype)
    at = w_at = None
    r_stride = r_code = w_code = 0
    if residual is not None:
        r_stride = _like("residual", residual, shape, device)
        r_code = _float_code(residual.dtype)
        at = residual.data_ptr() or None
    if weight is not None:
        w_at, w_code = _row("weight", weight, shape[1], device), _float_code(weight.dtype)
    return _ops.lamb_rms(x.data_ptr() or None, at, w_at, stride, r_stride, *shape, code, r_code,
                         w_code, eps)


def _like(name, t, shape, device):
    """The row stride of a 2-D tensor of x's shape."""
    if t.shape != shape:
        raise ValueError("%s must have x's shape" % name)
    # most are contiguous: nothing else to look at
    if len(shape) == 2 and t.is_contiguous() and t.is_cuda and t.device == device:
        return shape[1]
    return _rows(name, t, t.dtype, device)


def _row(name, t, dim, device):
    if not t.is_cuda or t.device != device:
        _on_gpu(name, t, device)
    if t.shape != (dim,):
        raise ValueError("%s must be [%d]" % (name, dim))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr()


def _result(name, t, like, dtype):
    """A result's tensor (``t``, or a new one like ``like``) and its row stride."""
    if t is None:
        torch = _torch_module
        return (torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format),
                like.shape[1])
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    return t, _like(name, t, like.shape, like.device)


def rms_norm(x, weight=None, *, residual=None, eps: float = 1e-6, out_dtype=None, out=None,
             summed=None):
    """``h weight / sqrt(mean(h^2) + eps)`` of every row h of ``x`` [tokens, dim], or of
    ``x + residual``: then (the norm, the sum) is returned, the sum rounded to the
    residual's type, and the norm is that of the rounded sum.

    ``x``, ``residual`` and ``weight`` [dim] are float32 or bfloat16 each, rows contiguous;
    the residual of a float32 x is float32. The norm has ``out_dtype`` (x's by default).
    ``out`` and ``summed`` are written where given; each may be x or the residual itself.
    Autograd does not see the call: tensors that require gradients are refused where grad
    mode is on (pass them detached)."""
    _torch()
    _no_graph("rms_norm", x, weight, residual, out, summed)
    r, device = _rms(x, weight, residual, eps), x.device
    if out is not None:
        out_dtype = out_dtype or out.dtype
    out, out_stride = _result("out", out, x, out_dtype or x.dtype)
    code = _float_code(out.dtype)
    summed, to, stride = _summed(r, x, residual, summed)
    with _on(device):
        _ops.lamb_rms_forward(r, to, stride, out.data_ptr(), out_stride, code, _stream(device))
    return out if residual is None else (out, summed)


def _summed(r, x, residual, summed):
    """The sum's tensor, its address and its row stride."""
    if residual is None:
        if summed is not None:
            raise ValueError("summed needs a residual")
        return None, None, 0
    summed, stride = _result("summed", summed, x, residual.dtype)
    return summed, summed.data_ptr(), stride


def rms_norm_fp8(x, weight=None, *, residual=None, eps: float = 1e-6, group: int = 0, out=None,
                 scales=None, summed=None):
    """:func:`rms_norm` with its result in 8 bits: (out, scales), with a residual (out,
    scales, sum). ``out`` (float8_e4m3fn, like x) times its scale is the norm; ``scales``
    (float32 [tokens, groups]) has one for a row (``group`` 0), or one for every 32, 64, 128
    or 256 columns, the last for what is left of a row: the largest magnitude / 448, at
    least 2^-126."""
    torch = _torch()
    _no_graph("rms_norm_fp8", x, weight, residual, out, scales, summed)
    r, device = _rms(x, weight, residual, eps), x.device
    out, out_stride = _result("out", out, x, torch.float8_e4m3fn)
    groups = -(-r.dim // group) if group > 0 else 1
    if scales is None:
        scales = torch.empty(r.tokens, groups, dtype=torch.float32, device=device)
    else:
        _on_gpu("scales", scales, device)
        if scales.dtype != torch.float32:
            raise TypeError("scales must be float32")
        if scales.shape != (r.tokens, groups) or not scales.is_contiguous():
            raise ValueError("scales must be [%d, %d] and contiguous" % (r.tokens, groups))
    summed, to, stride = _summed(r, x, residual, summed)
    with _on(device):
        _ops.lamb_rms_quantize(r, to, stride, out.data_ptr(), out_stride, scales.data_ptr(),
                               group, _stream(device))
    return (out, scales) if residual is None else (out, scales, summed)


def rms_norm_grad(x, weight, grad_out, grad_x=None, grad_weight=None, *, eps: float = 1e-6,
                  grad_sum=None, accumulate: bool = False) -> None:
    """Gradients of :func:`rms_norm`, given that of its result: into ``grad_x`` [tokens, dim]
    and ``grad_weight`` [dim], float32 or bfloat16 each and either optional; ``accumulate``
    adds to what ``grad_weight`` holds.

    ``x`` is what was normed: the sum, where there was a residual, and ``grad_x`` is the
    gradient of both its terms. ``grad_sum`` (of grad_x's type) is added to it: the gradient
    that the sum has from elsewhere, as the residual stream. ``grad_x`` may be ``x``,
    ``grad_out`` or ``grad_sum`` itself."""
    _torch()
    r, device = _rms(x, weight, None, eps), x.device
    g = _ops.lamb_rms_grads(add_weight=int(bool(accumulate)))
    g.grad_out_stride = _like("grad_out", grad_out, x.shape, device)
    g.grad_out_dtype = _float_code(grad_out.dtype)
    g.grad_out = grad_out.data_ptr() or None
    if grad_x is not None:
        g.grad_x_dtype = _float_code(grad_x.dtype)
        _, g.grad_x_stride = _result("grad_x", grad_x, x, grad_x.dtype)
        g.grad_x = grad_x.data_ptr() or None
    if grad_sum is not None:
        if grad_x is None:
            raise ValueError("grad_sum needs grad_x")
        _, g.grad_sum_stride = _result("grad_sum", grad_sum, x, grad_x.dtype)
        g.grad_sum = grad_sum.data_ptr() or None
    if grad_weight is not None:
        g.grad_weight = _row("grad_weight", grad_weight, r.dim, device)
        g.grad_weight_dtype = _float_code(grad_weight.dtype)
    need = _ops.lamb_rms_workspace(r)
    work = _workspace(need, device)
    with _on(device):
        _ops.lamb_rms_backward(r, g, work.data_ptr() or None, need, _stream(device))


class GradNorm:
    """The norm of a list of gradients, tensor by tensor and over all of them, and the
    gradients scaled so that it keeps a limit.

    ``grads`` are persistent contiguous tensors, float32 or bfloat16 each, of any size, none
    of them twice; ``run()`` and ``clip()`` read them as they are then. ``outputs``: where
    ``clip()`` writes, one tensor of as many elements for each, float32 or bfloat16 (default:
    the gradients themselves). ``norm``: "l2", "l1" or "linf".

    The results are on the device: ``norms`` (float64, one per tensor) and ``total`` (float64),
    which ``run()`` and ``clip()`` without a ``total`` write, and ``found_nonfinite`` (int32: 1
    where the last ``clip()`` met a total that is no finite number), which every ``clip()``
    writes. Streams and captures as for :class:`Orthogonalizer`.

    To be made once for tensors that stay: that takes an allocation, a copy and a wait for the
    stream, 0.3 ms for 391 tensors.
    """

    def __init__(self, grads: Sequence, outputs: Optional[Sequence] = None, norm: str = "l2"):
        torch = _torch()
        self.grads = list(grads)
        if not self.grads:
            raise ValueError("need at least one gradient")
        self.outputs = self.grads if outputs is None else list(outputs)
        if len(self.outputs) != len(self.grads):
            raise ValueError("need one output per gradient (got %d and %d)"
                             % (len(self.outputs), len(self.grads)))
        if norm not in _lib.NORMS:
            raise ValueError("norm must be one of %s" % (tuple(_lib.NORMS),))
        self.norm = norm
        self.device = self.grads[0].device
        same = self.outputs is self.grads
        rows = []
        for i, (a, b) in enumerate(zip(self.grads, self.outputs)):
            row = self._tensor("gradient", i, a)
            to = row if same else self._tensor("output", i, b)
            if row[1] != to[1]:
                raise ValueError("gradient %d has %d elements, its output %d" % (i, row[1], to[1]))
            rows.append((row[0], to[0], row[1], row[2], to[2]))
        results = torch.zeros(len(rows) + 2, dtype=torch.float64, device=self.device)
        self.norms, self.total = results[:-2], results[-2]
        self.found_nonfinite = results[-1:].view(torch.int32)[:1]
        with _on(self.device):
            self.plan = _ops.lamb_grad_plan_create(rows, _lib.NORMS[norm])
            # the zeros come before any call's results, whatever its stream
            torch.cuda.current_stream(self.device).synchronize()

    def _tensor(self, name, i, t):
        """(address, elements, type) of a tensor of the list."""
        if not t.is_cuda or t.device != self.device:
            _on_gpu("%s %d" % (name, i), t, self.device)
        if not t.is_contiguous():
            raise ValueError("%s %d is not contiguous" % (name, i))
        return t.data_ptr(), t.numel(), _float_code(t.dtype)

    def run(self):
        """Enqueue the norms on the current stream; returns ``total``."""
        _ops.lamb_grad_norm(self.plan, self.norms.data_ptr(), self.total.data_ptr(),
                            _stream(self.device))
        return self.total

    def clip(self, max_norm: float, *, scale: float = 1.0, total=None):
        """Write ``scale`` x the gradients, and less where their norm would pass
        ``max_norm``, into the outputs; returns the gradients' norm before that (without
        ``scale``). ``total``: that norm, where it is known already or is that of more
        gradients than these (one float64 element on the device); else it is computed.
        Gradients in place that need no change are only read. Where the norm is no finite
        number nothing is limited and ``found_nonfinite`` is set: the step that follows can
        see what the gradients hold (``skip_nonfinite``)."""
        if total is None:
            _ops.lamb_grad_norm_clip(self.plan, self.norms.data_ptr(), self.total.data_ptr(),
                                     max_norm, scale, self.found_nonfinite.data_ptr(),
                                     _stream(self.device))
            return self.total
        _on_gpu("total", total, self.device)
        if total.dtype != _torch().float64 or total.numel() != 1:
            raise TypeError("total must be one float64 element")
        _ops.lamb_grad_clip(self.plan, total.data_ptr(), max_norm, scale,
                            self.found_nonfinite.data_ptr(), _stream(self.device))
        return total

    def close(self) -> None:
        self.plan.close()
