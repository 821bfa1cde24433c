"""The operators' C interface on the CPU: every declared symbol is exported and bound,
the header compiles as C99 and C++11, and bad arguments are refused before any HIP
call."""

import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest

from paper_1904_00962_amd import _lib, _ops, build

HEADER = os.path.join(build.INCLUDE, "lamb_ops.h")
A = 1 << 40  # fake device addresses: refused calls dereference nothing


@pytest.fixture(scope="module")
def lib():
    if build.is_stale():
        build.build()
    return _ops.load()


def test_header_declares_the_bound_functions(lib):
    names = re.findall(r"LAMB_API\s+[\w\s\*]+?\b(\w+)\s*\(", open(HEADER).read())
    assert sorted(names) == sorted(_ops.EXPORTS)
    for name in names:
        assert hasattr(lib, name), name


@pytest.mark.parametrize("compiler,std", [("gcc", "-std=c99"), ("g++", "-std=c++11")])
def test_header_compiles_and_structs_match(tmp_path, compiler, std):
    cc = shutil.which(compiler)
    if cc is None:
        pytest.skip("%s is not installed" % compiler)
    structs = [s for s in vars(_ops).values()
               if isinstance(s, type) and issubclass(s, ctypes.Structure)
               and s.__module__ == _ops.__name__]
    src = tmp_path / ("h.c" if compiler == "gcc" else "h.cpp")
    src.write_text('#include <stdio.h>\n#include "lamb_ops.h"\nint main(void) {\n' + "".join(
        'printf("%%s %%d\\n", "%s", (int)sizeof(%s));\n' % (s.__name__, s.__name__)
        for s in structs) + "return 0; }\n")
    exe = tmp_path / "h"
    r = subprocess.run([cc, std, "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", build.INCLUDE,
                        str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    sizes = dict(line.split() for line in
                 subprocess.run([str(exe)], capture_output=True, text=True).stdout.splitlines())
    assert sizes == {s.__name__: str(ctypes.sizeof(s)) for s in structs}


def _refused(status, call, *words):
    with pytest.raises(_lib.LambError) as e:
        call()
    assert e.value.status == status, str(e.value)
    for w in words:
        assert w in str(e.value)


def _matrix(base=A, rows=4, cols=8, stride=None, out=None):
    s = cols if stride is None else stride
    return (base, base + (1 << 24) if out is None else out, rows, cols, s, s)


@pytest.mark.parametrize("rows,types,status", [
    ([], (0, 0, 0), _lib.LAMB_EINVAL),
    ([_matrix()], (2, 0, 0), _lib.LAMB_EINVAL),
    ([_matrix()], (0, 3, 0), _lib.LAMB_EINVAL),
    ([_matrix()], (0, 0, 2), _lib.LAMB_EINVAL),
    ([_matrix(base=0, out=A)], (0, 0, 0), _lib.LAMB_ENULL),
    ([(A, 0, 4, 8, 8, 8)], (0, 0, 0), _lib.LAMB_ENULL),
    ([_matrix(rows=0)], (0, 0, 0), _lib.LAMB_EINVAL),
    ([_matrix(cols=(1 << 20) + 1)], (0, 0, 0), _lib.LAMB_EINVAL),
    ([_matrix(stride=7)], (0, 0, 0), _lib.LAMB_EINVAL),
    ([_matrix(base=A + 2)], (0, 0, 0), _lib.LAMB_EALIGN),
    ([_matrix(base=A + 1)], (1, 1, 0), _lib.LAMB_EALIGN),
    ([_matrix(out=A + 64)], (0, 0, 0), _lib.LAMB_EOVERLAP),
    ([_matrix(out=A)], (0, 1, 0), _lib.LAMB_EOVERLAP),               # in place, other type
    ([_matrix(), _matrix(base=A + (1 << 26), out=A + (1 << 24))], (0, 0, 0), _lib.LAMB_EOVERLAP),
    ([_matrix(out=A), _matrix(base=A, out=A + (1 << 24))], (0, 0, 0), _lib.LAMB_EOVERLAP),
])
def test_ortho_plan_refusals(lib, rows, types, status):
    _refused(status, lambda: _ops.lamb_ortho_plan_create(rows, *types))


@pytest.mark.parametrize("row,g,precision,status", [
    ((A, A + 4096, A + 8192, 4, 8, 1), 2, 0, _lib.LAMB_EINVAL),
    ((A, A + 4096, A + 8192, 4, 8, 1), 0, 5, _lib.LAMB_EINVAL),
    ((0, A + 4096, A + 8192, 4, 8, 1), 0, 0, _lib.LAMB_ENULL),
    ((A, A + 4096, 0, 4, 8, 1), 0, 0, _lib.LAMB_ENULL),
    ((A, A + 4096, A + 8192, 4, 0, 1), 0, 0, _lib.LAMB_EINVAL),
    ((A, A + 4096, A + 8192, 4, 8, 2), 0, 0, _lib.LAMB_EINVAL),
    ((A, A + 4096, A + 8200, 4, 8, 1), 0, 0, _lib.LAMB_EALIGN),
    ((A, A + 64, A + 8192, 4, 8, 1), 0, 0, _lib.LAMB_EOVERLAP),
])
def test_muon_plan_refusals(lib, row, g, precision, status):
    _refused(status, lambda: _ops.lamb_muon_plan_create([row], g, precision))


def test_null_arguments(lib):
    none = ctypes.c_void_p(0)
    assert lib.lamb_ns_params_init(None) == _lib.LAMB_ENULL
    assert lib.lamb_muon_hparams_init(None) == _lib.LAMB_ENULL
    assert lib.lamb_ortho_plan_create(None, 1, 0, 0, 0, None) == _lib.LAMB_ENULL
    assert lib.lamb_orthogonalize(none, None, none) == _lib.LAMB_ENULL
    assert lib.lamb_muon_step(none, None, none, none) == _lib.LAMB_ENULL
    assert lib.lamb_ns_plan_destroy(none) == _lib.LAMB_OK


def test_defaults(lib):
    p = _ops.lamb_ns_params_init()
    assert (p.steps, round(p.a, 4), round(p.b, 4), round(p.c, 4)) == (5, 3.4445, -4.775, 2.0315)
    hp = _ops.lamb_muon_hparams_init(scale="spectral")
    assert hp.scale == _ops.LAMB_MUON_SPECTRAL and hp.nesterov == 1 and hp.ns.steps == 5
    with pytest.raises(AttributeError):
        _ops.lamb_muon_hparams_init(beta=1)
    assert math.isclose(hp.momentum, 0.95, rel_tol=1e-6)


def _xent(**fields):
    x = _ops.lamb_xent(A, A + (1 << 24), A + (1 << 25), 64, 64, 10, 20, 64, -100,
                       _ops.LAMB_DTYPE_I64, 0)
    for k, v in fields.items():
        setattr(x, k, v)
    return x


@pytest.mark.parametrize("fields,status", [
    (dict(tokens=-1), _lib.LAMB_EINVAL), (dict(tokens=(1 << 24) + 1), _lib.LAMB_EINVAL),
    (dict(vocab=0), _lib.LAMB_EINVAL), (dict(dim=0), _lib.LAMB_EINVAL),
    (dict(dim=(1 << 16) + 1), _lib.LAMB_EINVAL), (dict(hidden_stride=63), _lib.LAMB_EINVAL),
    (dict(table_stride=63), _lib.LAMB_EINVAL), (dict(target_dtype=0), _lib.LAMB_EINVAL),
    (dict(hidden_stride=1 << 40, tokens=1 << 24), _lib.LAMB_EINVAL),
    (dict(reserved=1), _lib.LAMB_EINVAL), (dict(table=None), _lib.LAMB_ENULL),
    (dict(hidden=None), _lib.LAMB_ENULL), (dict(targets=None), _lib.LAMB_ENULL),
    (dict(hidden=A + 1), _lib.LAMB_EALIGN), (dict(targets=A + 4), _lib.LAMB_EALIGN),
])
def test_cross_entropy_refusals(lib, fields, status):
    x = _xent(**fields)
    for call in (lambda: _ops.lamb_xent_workspace(x, False),
                 lambda: _ops.lamb_xent_forward(x, A, A, A, A, 1 << 40),
                 lambda: _ops.lamb_xent_backward(x, A, _ops.lamb_xent_grads(), A, 1 << 40)):
        _refused(status, call)


def test_cross_entropy_buffers(lib):
    x, far = _xent(), A + (1 << 30)
    need = _ops.lamb_xent_workspace(x, False)
    back = _ops.lamb_xent_workspace(x, True)
    assert need > 0 and back > 0 and need % 256 == 0
    fwd = lambda loss, lse, mean, work, size: _ops.lamb_xent_forward(  # noqa: E731
        x, loss, lse, mean, work, size)
    _refused(_lib.LAMB_ENULL, lambda: fwd(0, far, 0, far, need))
    _refused(_lib.LAMB_ENULL, lambda: fwd(far, far + 64, 0, 0, need))
    _refused(_lib.LAMB_EALIGN, lambda: fwd(far, far + 64, 0, far + 128, need))
    _refused(_lib.LAMB_EALIGN, lambda: fwd(far + 2, far + 64, 0, far + 256, need))
    _refused(_lib.LAMB_EINVAL, lambda: fwd(far, far + 64, 0, far + 256, need - 1), "workspace")
    _refused(_lib.LAMB_EOVERLAP, lambda: fwd(far, far + 36, 0, far + 256, need))
    _refused(_lib.LAMB_EOVERLAP, lambda: fwd(far, far + 64, A, far + 256, need))
    for fields, status in ((dict(add_table=2), _lib.LAMB_EINVAL), (dict(mean=-1), _lib.LAMB_EINVAL),
                           (dict(grad_scale=math.inf), _lib.LAMB_EINVAL),
                           (dict(grad_table=far, grad_table_stride=64, grad_table_dtype=2),
                            _lib.LAMB_EINVAL),
                           (dict(grad_table=far, grad_table_stride=63), _lib.LAMB_EINVAL),
                           (dict(grad_hidden=A, grad_hidden_stride=64), _lib.LAMB_EOVERLAP),
                           (dict(grad_hidden=far + 1, grad_hidden_stride=64), _lib.LAMB_EALIGN)):
        _refused(status, lambda: _ops.lamb_xent_backward(
            x, A, _ops.lamb_xent_grads(**fields), far + (1 << 20), back))
    _refused(_lib.LAMB_ENULL, lambda: _ops.lamb_xent_backward(
        x, 0, _ops.lamb_xent_grads(), far, back))


def test_cross_entropy_workspace_is_a_piece(lib):
    """Far below the logits, which 16384 tokens against 200,000 words would take 6.5 GB for."""
    x = _xent(tokens=16384, vocab=200000, dim=1024, hidden_stride=1024, table_stride=1024)
    assert _ops.lamb_xent_workspace(x, True) < 16384 * 1024 * (2 + 8 * 4) + (200 << 20)


def _embed(**fields):
    e = _ops.lamb_embed(A, 10, 20, 64, _ops.LAMB_DTYPE_I64, 1.0)
    for k, v in fields.items():
        setattr(e, k, v)
    return e


@pytest.mark.parametrize("fields,status", [
    (dict(tokens=-1), _lib.LAMB_EINVAL), (dict(vocab=0), _lib.LAMB_EINVAL),
    (dict(dim=1 << 20), _lib.LAMB_EINVAL), (dict(id_dtype=1), _lib.LAMB_EINVAL),
    (dict(scale=math.nan), _lib.LAMB_EINVAL), (dict(ids=None), _lib.LAMB_ENULL),
    (dict(ids=A + 4), _lib.LAMB_EALIGN),
])
def test_table_refusals(lib, fields, status):
    e, t, o = _embed(**fields), A + (1 << 24), A + (1 << 25)
    for call in (lambda: _ops.lamb_embed_forward(e, t, 64, 0, o, 64, 0),
                 lambda: _ops.lamb_embed_workspace(e),
                 lambda: _ops.lamb_embed_backward(e, o, 64, 0, t, 64, 0, -1, 0, A, 1 << 40)):
        _refused(status, call)


def test_table_buffers(lib):
    e, t, o, w = _embed(), A + (1 << 24), A + (1 << 25), A + (1 << 26)
    need = _ops.lamb_embed_workspace(e)
    for args, status in (((0, 64, 0, o, 64, 0), _lib.LAMB_ENULL),
                         ((t, 63, 0, o, 64, 0), _lib.LAMB_EINVAL),
                         ((t, 64, 2, o, 64, 0), _lib.LAMB_EINVAL),
                         ((t, 64, 0, o + 2, 64, 0), _lib.LAMB_EALIGN),
                         ((t, 64, 0, t + 256, 64, 0), _lib.LAMB_EOVERLAP)):
        _refused(status, lambda: _ops.lamb_embed_forward(e, *args))
    for args, status in (((0, 64, 0, t, 64, 0, -1, 0, w, need), _lib.LAMB_ENULL),
                         ((o, 64, 0, t, 64, 0, -1, 2, w, need), _lib.LAMB_EINVAL),
                         ((o, 64, 0, t, 64, 0, -1, 0, 0, need), _lib.LAMB_ENULL),
                         ((o, 64, 0, t, 64, 0, -1, 0, w, need - 1), _lib.LAMB_EINVAL),
                         ((o, 64, 0, o, 64, 0, -1, 0, w, need), _lib.LAMB_EOVERLAP)):
        _refused(status, lambda: _ops.lamb_embed_backward(e, *args))
