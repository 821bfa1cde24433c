"""The C interface of the root-mean-square norm and of the gradients' norm on the CPU: bad
arguments are refused before any HIP call."""

import ctypes
import math

import pytest

from paper_1904_00962_amd import _lib, _ops, build

A = 1 << 40  # fake device addresses: refused calls dereference nothing
F32, BF16 = _ops.LAMB_DTYPE_F32, _ops.LAMB_DTYPE_BF16
FAR = A + (1 << 30)


@pytest.fixture(scope="module")
def lib():
    if build.is_stale():
        build.build()
    return _ops.load()


def _refused(status, call, *words):
    with pytest.raises(_lib.LambError) as e:
        call()
    assert e.value.status == status, str(e.value)
    for w in words:
        assert w in str(e.value)


def _rms(**fields):
    r = _ops.lamb_rms(A, A + (1 << 24), A + (1 << 25), 64, 64, 10, 64, BF16, BF16, F32, 1e-6)
    for k, v in fields.items():
        setattr(r, k, v)
    return r


@pytest.mark.parametrize("fields,status", [
    (dict(tokens=-1), _lib.LAMB_EINVAL), (dict(tokens=(1 << 24) + 1), _lib.LAMB_EINVAL),
    (dict(dim=0), _lib.LAMB_EINVAL), (dict(dim=(1 << 16) + 1), _lib.LAMB_EINVAL),
    (dict(eps=-1e-9), _lib.LAMB_EINVAL), (dict(eps=math.inf), _lib.LAMB_EINVAL),
    (dict(eps=math.nan), _lib.LAMB_EINVAL), (dict(x_stride=63), _lib.LAMB_EINVAL),
    (dict(x_stride=(1 << 36) + 1), _lib.LAMB_EINVAL), (dict(x_dtype=2), _lib.LAMB_EINVAL),
    (dict(residual_dtype=3), _lib.LAMB_EINVAL), (dict(weight_dtype=-1), _lib.LAMB_EINVAL),
    (dict(residual_stride=1), _lib.LAMB_EINVAL), (dict(x=None), _lib.LAMB_ENULL),
    (dict(x_dtype=F32, residual_dtype=BF16), _lib.LAMB_EINVAL),
    (dict(x=A + 1), _lib.LAMB_EALIGN), (dict(residual=A + (1 << 24) + 1), _lib.LAMB_EALIGN),
    (dict(weight=A + (1 << 25) + 2), _lib.LAMB_EALIGN),
])
def test_norm_refusals(lib, fields, status):
    r = _rms(**fields)
    g = _ops.lamb_rms_grads()
    for call in (lambda: _ops.lamb_rms_forward(r, FAR, 64, FAR + 8192, 64, BF16),
                 lambda: _ops.lamb_rms_quantize(r, FAR, 64, FAR + 8192, 64, FAR + 65536, 0),
                 lambda: _ops.lamb_rms_workspace(r),
                 lambda: _ops.lamb_rms_backward(r, g, FAR, 1 << 40)):
        _refused(status, call)


def test_norm_results(lib):
    r = _rms()
    for args, status in (((FAR, 64, 0, 64, BF16), _lib.LAMB_ENULL),
                         ((FAR, 64, FAR + 8192, 63, BF16), _lib.LAMB_EINVAL),
                         ((FAR, 63, FAR + 8192, 64, BF16), _lib.LAMB_EINVAL),
                         ((FAR, 64, FAR + 8192, 64, 2), _lib.LAMB_EINVAL),
                         ((FAR, 64, FAR + 8194, 64, F32), _lib.LAMB_EALIGN),
                         ((FAR + 1, 64, FAR + 8192, 64, BF16), _lib.LAMB_EALIGN),
                         ((FAR, 64, FAR + 64, 64, BF16), _lib.LAMB_EOVERLAP),
                         ((FAR, 64, FAR, 64, BF16), _lib.LAMB_EOVERLAP),
                         ((FAR, 64, A + 128, 64, BF16), _lib.LAMB_EOVERLAP),   # x, a row on
                         ((FAR, 64, A, 64, F32), _lib.LAMB_EOVERLAP),          # x, another type
                         ((FAR, 64, A, 128, BF16), _lib.LAMB_EOVERLAP),        # x, another stride
                         ((A + (1 << 25), 64, FAR, 64, BF16), _lib.LAMB_EOVERLAP)):  # the weight
        _refused(status, lambda: _ops.lamb_rms_forward(r, *args))
    _refused(_lib.LAMB_EINVAL, lambda: _ops.lamb_rms_forward(
        _rms(residual=None), FAR, 64, FAR + 8192, 64, BF16), "residual")
    for scales, group, out, status in ((0, 0, FAR, _lib.LAMB_ENULL),
                                       (FAR + 8192, 16, FAR, _lib.LAMB_EINVAL),
                                       (FAR + 8192, 512, FAR, _lib.LAMB_EINVAL),
                                       (FAR + 8192, -1, FAR, _lib.LAMB_EINVAL),
                                       (FAR + 8194, 0, FAR, _lib.LAMB_EALIGN),
                                       (FAR + 128, 0, FAR, _lib.LAMB_EOVERLAP),
                                       (FAR + 8192, 0, A, _lib.LAMB_EOVERLAP)):
        _refused(status, lambda: _ops.lamb_rms_quantize(r, 0, 0, out, 64, scales, group))


def test_norm_gradients(lib):
    r = _rms(residual=None)
    need = _ops.lamb_rms_workspace(r)
    assert need > 0 and need % 256 == 0
    good = dict(grad_out=FAR, grad_out_stride=64, grad_out_dtype=BF16, grad_x=FAR + 8192,
                grad_x_stride=64, grad_x_dtype=BF16, grad_weight=FAR + 16384)
    work = FAR + (1 << 20)
    for fields, status in ((dict(grad_out=None), _lib.LAMB_ENULL),
                           (dict(grad_out_stride=63), _lib.LAMB_EINVAL),
                           (dict(grad_out_dtype=4), _lib.LAMB_EINVAL),
                           (dict(grad_x_dtype=2), _lib.LAMB_EINVAL),
                           (dict(grad_x_stride=0), _lib.LAMB_EINVAL),
                           (dict(grad_sum=FAR + 32768), _lib.LAMB_EINVAL),  # no stride
                           (dict(grad_weight_dtype=2), _lib.LAMB_EINVAL),
                           (dict(add_weight=2), _lib.LAMB_EINVAL),
                           (dict(reserved=1), _lib.LAMB_EINVAL),
                           (dict(grad_out=FAR + 1), _lib.LAMB_EALIGN),
                           (dict(grad_weight=FAR + 16386), _lib.LAMB_EALIGN),
                           (dict(grad_weight=FAR + 8192), _lib.LAMB_EOVERLAP),
                           (dict(grad_x=FAR + 128), _lib.LAMB_EOVERLAP),
                           (dict(grad_x=work), _lib.LAMB_EOVERLAP),
                           (dict(grad_x=FAR, grad_x_dtype=F32), _lib.LAMB_EOVERLAP)):
        _refused(status, lambda: _ops.lamb_rms_backward(
            r, _ops.lamb_rms_grads(**{**good, **fields}), work, need))
    g = _ops.lamb_rms_grads(**good)
    _refused(_lib.LAMB_EINVAL, lambda: _ops.lamb_rms_backward(_rms(), g, work, need), "residual")
    _refused(_lib.LAMB_ENULL, lambda: _ops.lamb_rms_backward(r, g, 0, need), "workspace")
    _refused(_lib.LAMB_EALIGN, lambda: _ops.lamb_rms_backward(r, g, work + 128, need))
    _refused(_lib.LAMB_EINVAL, lambda: _ops.lamb_rms_backward(r, g, work, need - 1), "workspace")
    wide = _rms(residual=None, dim=9000, x_stride=9000)
    g = _ops.lamb_rms_grads(grad_out=FAR, grad_out_stride=9000, grad_x=FAR + (1 << 20),
                            grad_x_stride=9000)
    _refused(_lib.LAMB_ENULL, lambda: _ops.lamb_rms_backward(wide, g, 0, 0), "workspace")


@pytest.mark.parametrize("dim", [1, 100, 1600, 8192, 8193, 65536])
def test_norm_workspace_is_within_the_stated_bytes(lib, dim):
    columns = (dim + 7) // 8 * 8
    for tokens in (0, 1, 7, 4096, 4097, 100000, 1 << 24):
        r = _rms(residual=None, tokens=tokens, dim=dim, x_stride=dim)
        if dim <= 8192:
            most = 4 * columns * min(1024, tokens + 3) + 256
        else:
            most = 4 * columns * (tokens // 16 + 1) + 16 * tokens + 512
        assert _ops.lamb_rms_workspace(r) <= most, tokens


def _tensor(base=A, out=None, numel=100, types=(F32, F32)):
    return (base, base if out is None else out, numel, *types)


@pytest.mark.parametrize("rows,norm,status", [
    ([], 0, _lib.LAMB_EINVAL), ([_tensor()], 3, _lib.LAMB_EINVAL),
    ([_tensor()], -1, _lib.LAMB_EINVAL),
    ([_tensor(numel=-1)], 0, _lib.LAMB_EINVAL),
    ([_tensor(numel=(1 << 40) + 1)], 0, _lib.LAMB_EINVAL),
    ([_tensor(types=(2, 0))], 0, _lib.LAMB_EINVAL), ([_tensor(types=(0, 3))], 0, _lib.LAMB_EINVAL),
    ([_tensor(base=0, out=A)], 0, _lib.LAMB_ENULL), ([_tensor(base=A + 2)], 0, _lib.LAMB_EALIGN),
    ([_tensor(out=A + 401, types=(0, 1))], 0, _lib.LAMB_EALIGN),
    ([_tensor(out=A + 396)], 0, _lib.LAMB_EOVERLAP),
    ([_tensor(types=(0, 1))], 0, _lib.LAMB_EOVERLAP),  # in place, another type
    ([_tensor(), _tensor()], 0, _lib.LAMB_EOVERLAP),
    ([_tensor(), _tensor(base=A + 200)], 0, _lib.LAMB_EOVERLAP),
    ([_tensor(out=FAR), _tensor(base=FAR + 4, out=FAR + 4096)], 0, _lib.LAMB_EOVERLAP),
    ([_tensor(numel=1 << 40)] + [_tensor(base=A + (k << 42), numel=1 << 40) for k in range(1, 200)],
     0, _lib.LAMB_EINVAL),  # more chunks than a launch counts
])
def test_gradient_plan_refusals(lib, rows, norm, status):
    _refused(status, lambda: _ops.lamb_grad_plan_create(rows, norm))


def test_null_arguments(lib):
    none = ctypes.c_void_p(0)
    assert lib.lamb_rms_forward(None, none, 0, none, 0, 0, none) == _lib.LAMB_ENULL
    assert lib.lamb_rms_quantize(None, none, 0, none, 0, none, 0, none) == _lib.LAMB_ENULL
    assert lib.lamb_rms_workspace(ctypes.byref(_rms()), None) == _lib.LAMB_ENULL
    assert lib.lamb_rms_backward(ctypes.byref(_rms(residual=None)), None, none, 0,
                                 none) == _lib.LAMB_ENULL
    assert lib.lamb_grad_plan_create(None, 1, 0, None) == _lib.LAMB_ENULL
    assert lib.lamb_grad_norm(none, none, none, none) == _lib.LAMB_ENULL
    assert lib.lamb_grad_clip(none, none, 1.0, 1.0, none, none) == _lib.LAMB_ENULL
    assert lib.lamb_grad_plan_destroy(none) == _lib.LAMB_OK
