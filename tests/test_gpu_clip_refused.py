"""A step that is refused leaves the gradients as they are, also where it would have clipped
them."""

import math

import pytest

from gpu_harness import torch_cuda

pytestmark = pytest.mark.gpu

NAN, INF = math.nan, math.inf
# fields of the optimizer, then the step's learning rate
LAYERWISE = [({}, NAN), ({}, INF), (dict(grad_scale=INF), None), (dict(grad_scale=NAN), None),
             (dict(weight_decay=NAN), None), (dict(gamma_l=3.0, gamma_u=1.0), None)]
LAMB_ONLY = [(dict(beta1=1.0), None), (dict(beta2=-1.0), None), (dict(eps=NAN), None)]
LARS_ONLY = [(dict(momentum=1.0), None), (dict(trust_coef=INF), None)]
MUON = [({}, NAN), ({}, -1.0), (dict(grad_scale=0.0), None), (dict(grad_scale=INF), None),
        (dict(momentum=1.0), None), (dict(weight_decay=-1.0), None)]


@pytest.mark.parametrize("optimizer,cases", [("LAMB", LAYERWISE + LAMB_ONLY),
                                             ("LARS", LAYERWISE + LARS_ONLY), ("Muon", MUON)])
def test_refused_steps(optimizer, cases):
    torch = torch_cuda()
    from paper_1904_00962_amd import LAMB, LARS, Muon, _lib
    kind = {"LAMB": LAMB, "LARS": LARS, "Muon": Muon}[optimizer]
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda: [torch.randn(s, generator=gen, device="cuda")  # noqa: E731
                   for s in ((64, 48), (33, 128))]
    xs, gs = new(), new()
    kept = [t.clone() for t in xs + gs]

    def same():
        torch.cuda.synchronize()
        return all(torch.equal(a, b) for a, b in zip(xs + gs, kept))

    for fields, lr in cases:
        opt = kind(xs, gs, lr=0.01, max_grad_norm=0.5)
        for name, value in fields.items():
            setattr(opt.hparams if optimizer == "Muon" else opt, name, value)
        with pytest.raises(_lib.LambError) as e:
            opt.step(lr)
        assert e.value.status == _lib.LAMB_EINVAL
        assert same() and float(opt.grad_norm) == 0.0, (fields, lr)
        opt.close()
    opt = kind(xs, gs, lr=0.01, max_grad_norm=0.5)
    opt.plan.close()
    with pytest.raises(_lib.LambError) as e:
        opt.step()
    assert e.value.status == _lib.LAMB_ENULL and same()
    # and one that is not refused clips and steps
    opt = kind(xs, gs, lr=0.01, max_grad_norm=0.5)
    opt.step()
    torch.cuda.synchronize()
    assert float(opt.grad_norm) > 0.5
    assert not any(torch.equal(a, b) for a, b in zip(xs + gs, kept))
