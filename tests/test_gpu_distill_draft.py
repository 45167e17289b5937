"""The example that distils a compressed projection from its teacher and has it draft
for it (examples/distill_draft.py): the operators together, as a program uses them. A step's
gradients are those of fp64 autograd through the decoded weights; what stands of the
drafts is what the definition says."""
import importlib.util
import os

import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say
from test_gpu_draft import _check, _reference

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "distill_draft.py")


def _pair(gpu):
    spec = importlib.util.spec_from_file_location("distill_draft", PATH)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    return ex, ex.Pair(device=gpu)


def test_a_step_is_the_gradient_of_the_divergence(gpu):
    """Every bf16 rounding on the way (W_hat, y, d, dy: 2^-8 each) moves a gradient by that
    part of its norm at most, and what is kept of the probabilities by 2^-11: four of the
    first and one of the second, added."""
    ex, pair = _pair(gpu)
    pair.B += 0.02 * torch.randn(pair.B.shape, generator=torch.Generator().manual_seed(3)).to(gpu)
    pair.refresh()
    tokens, ignore = ex.batch(pair)
    X = pair.embed[tokens]
    ids, top, norm = bsq.bsq_top_logits(pair.teacher(X), pair.K, scale=pair.scale)
    A = pair.pool.A.double().requires_grad_()
    B = pair.pool.B.double().requires_grad_()
    W = bsq.bsq_decode(pair.cfg, pair.codec, pair.layer).double()
    y = X.double() @ W.T + (X.double() @ A[0].T) @ B[0].T
    logq = torch.log_softmax(pair.scale * (y @ pair.head.double().T), 1).gather(1, ids.long())
    logp = pair.scale * top.double() - norm.double()[:, None]
    loss = (logp.exp() * (logp - logq)).sum(1)[~ignore].mean()
    loss.backward()
    got, size = pair.step(tokens, ignore, lr=0.0, max_norm=1e9)
    bar = 4 * 2.0 ** -8 + 2.0 ** -11
    for name, mine, want in (("dA", pair.dA, A.grad), ("dB", pair.dB, B.grad)):
        rel = float((mine.double() - want).norm() / want.norm())
        say(f"  {name}: off by {rel:.2e} of its norm")
        assert rel <= bar
    # y in bf16 moves a logit by 2^-8 of its terms' norm (a sum of independent roundings), the
    # divergence by no more than that of its largest
    z = pair.scale * 2.0 ** -8 * float(y.detach().norm(dim=1).max()) * float(pair.head.double().norm(dim=1).max())
    say(f"  divergence {float(got):.5f}, in 64 bits {float(loss.detach()):.5f}")
    assert abs(float(got) - float(loss.detach())) <= z
    want = float(torch.cat([A.grad.flatten(), B.grad.flatten()]).norm())
    assert abs(float(size) - want) <= bar * want


def test_training_leaves_the_codes_and_decoding_keeps_the_rules(gpu):
    ex, pair = _pair(gpu)
    tokens, ignore = ex.batch(pair)
    codes = [c.clone() for c in pair.layer.codes]
    for _ in range(3):
        loss, size = pair.step(tokens, ignore)
        assert torch.isfinite(loss) and torch.isfinite(size)
    assert all(torch.equal(a, b) for a, b in zip(codes, pair.layer.codes))
    gen = torch.Generator().manual_seed(5)
    last = torch.arange(20, device=gpu)
    for L in (1, 4, 0):
        if L == 0:
            none = torch.empty((20, 0), device=gpu)
            given = (pair.teacher(pair.embed[last])[:, None], none.int(), none, torch.rand(20, generator=gen).to(gpu), None)
            got = bsq.bsq_draft_verify(*given[:4])
        else:
            given, got = pair.decode(last, L, gen)
        say(f"  L={L}: {int(got[0].sum())} of {20 * L} stand")
        target, tokens, u, r, draft = given
        _check(_reference(target, tokens, u.cpu(), r.cpu(), draft), got)
