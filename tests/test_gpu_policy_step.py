"""The example's training step: it runs, its loss falls, and its whole gradient (head, embedding added to it, layer)
agrees with torch's automatic differentiation of the same formulas in 64 bits."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def ex():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as pkg
    pkg.build()
    import policy_step
    return policy_step


def test_the_loss_falls(ex):
    losses = ex.train(steps=4, groups=2)
    assert all(b < a for a, b in zip(losses, losses[1:])), losses


def test_tied_gradient_against_automatic_differentiation(ex):
    import torch
    import paper_2606_18954_gb300 as P
    gp = P.GraphPO()
    V, d, T = 700, 64, 400
    torch.manual_seed(2)
    policy = ex.Policy(V, d, seed=3)
    ids = torch.randint(0, V, (T,), device="cuda")
    target = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    target[::7] = -1
    g, e = torch.randn(T, device="cuda") / T, torch.randn(T, device="cuda") * 0.1 / T
    x, t, hidden = policy.forward(gp, ids)
    head = gp.vocab_logp(hidden, policy.table, target, entropy=True)
    grads = gp.vocab_grad(hidden, policy.table, target, head["lse"], g, entropy=head["entropy"], grad_entropy=e)
    d_layer = policy.backward(gp, ids, x, t, grads["d_hidden"], grads["d_weight"])
    gp.check()
    table = policy.table.double().requires_grad_()
    layer = policy.layer.double().requires_grad_()
    xx = table[ids] * policy.scale
    hh = xx + torch.tanh(xx @ layer)
    q = torch.log_softmax(hh @ table.t(), 1)
    keep = target >= 0
    lp = q.gather(1, target.clamp(min=0).long()[:, None])[:, 0]
    ent = -(q.exp() * q).sum(1)
    (torch.where(keep, g.double() * lp + e.double() * ent, 0.0)).sum().backward()
    # bf16 all the way: activations, their derivatives and each gradient carry 2^-8 relative errors, a dozen of them
    # in a row at most; norms of the whole against 12 * 2^-8
    for got, want in ((grads["d_weight"], table.grad), (d_layer, layer.grad)):
        assert float((got.double() - want).norm() / want.norm()) < 12 * 2.0 ** -8
