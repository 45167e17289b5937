"""The example that trains several tenants' adapters beside one compressed
projection (examples/train_adapters.py): its loss falls, the tenants' alone are
changed, and the gradients of a step are those of fp64 autograd through the
decoded weights."""
import importlib.util
import os

import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_adapters.py")


def _example():
    spec = importlib.util.spec_from_file_location("train_adapters", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_loss_falls_and_decode_runs(gpu):
    ex = _example()
    model = ex.Tenants(device=gpu)
    X, ids, target = ex.batch(model)
    codes = [c.clone() for c in model.layer.codes]
    losses = [float(model.step(X, ids, target)[0]) for _ in range(25)]
    say(f"  loss {losses[0]:.3f} -> {losses[-1]:.3f}")
    assert losses[-1] < 0.8 * losses[0]
    assert all(torch.equal(a, b) for a, b in zip(codes, model.layer.codes))
    words, lse = model.decode(X[:8].contiguous(), ids[:8].contiguous())
    assert words.shape == (8,) and torch.isfinite(lse).all()


def test_a_step_is_the_gradient_of_the_loss(gpu):
    """Every bf16 rounding on the way (W_hat, y, d, dy: 2^-8 each) moves a
    gradient by that part of its norm at most: four of them, added."""
    ex = _example()
    model = ex.Tenants(device=gpu)
    model.B += 0.02 * torch.randn(model.B.shape, generator=torch.Generator().manual_seed(3)).to(gpu)
    model.refresh()
    X, ids, target = ex.batch(model)
    A = model.pool.A.double().requires_grad_()
    B = model.pool.B.double().requires_grad_()
    W = bsq.bsq_decode(model.cfg, model.codec, model.layer).double()
    y = X.double() @ W.T
    for a in range(model.tenants):
        mine = (ids == a).double()[:, None]
        y = y + mine * 2.0 * ((X.double() @ A[a].T) @ B[a].T)
    z = y @ model.head.double().T
    live = target >= 0
    loss = (torch.logsumexp(z, 1) - z.gather(1, target.clamp_min(0)[:, None])[:, 0])[live].mean()
    loss.backward()
    got, norm = model.step(X, ids, target, lr=0.0, max_norm=1e9)
    for name, mine, want in (("dA", model.dA, A.grad), ("dB", model.dB, B.grad)):
        rel = float((mine.double() - want).norm() / want.norm())
        say(f"  {name}: off by {rel:.2e} of its norm")
        assert rel <= 4 * 2.0 ** -8
    assert abs(float(got) - float(loss)) <= 2.0 ** -8 * float(loss)
    want = float(torch.cat([A.grad.flatten(), B.grad.flatten()]).norm())
    assert abs(float(norm) - want) <= 4 * 2.0 ** -8 * want
