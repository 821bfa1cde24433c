"""The checks of a step's arguments by themselves, on the CPU: their bindings, and that they
refuse what no plan is needed to refuse."""

import ctypes

import pytest

from paper_1904_00962_amd import _lib, _ops, build


@pytest.fixture(scope="module", autouse=True)
def lib():
    if build.is_stale():
        build.build()
    return _ops.load()


def test_null_plans(lib):
    hp = _lib.lamb_hparams_init("lamb")
    muon = _ops.lamb_muon_hparams_init(_ops.lamb_ns_params_init())
    none = ctypes.c_void_p(0)
    assert lib.lamb_step_check(none, ctypes.byref(hp)) == _lib.LAMB_ENULL
    assert lib.lamb_muon_check(none, ctypes.byref(muon)) == _lib.LAMB_ENULL
    for check, fields in ((_lib.lamb_step_check, hp), (_ops.lamb_muon_check, muon)):
        with pytest.raises(_lib.LambError) as e:
            check(_lib.Plan(0), fields)
        assert e.value.status == _lib.LAMB_ENULL


def test_hyperparameters_without_a_plan_are_not_read():
    """NULL hyperparameters beside a NULL plan."""
    assert _lib.load().lamb_step_check(None, None) == _lib.LAMB_ENULL
    assert _ops.load().lamb_muon_check(None, None) == _lib.LAMB_ENULL
