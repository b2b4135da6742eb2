"""The example's training step with a teacher runs, and its gradients are the formulas' (test_gpu_distill.py tests the operators)."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_step_with_a_teacher_runs():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as P
    P.build()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import policy_step
    plain = policy_step.train(steps=2, vocab=700, d=64)
    taught = policy_step.train(steps=2, vocab=700, d=64, teacher_weight=0.1)
    assert len(taught) == 2 and all(math.isfinite(x) for x in taught)
    # the first step's loss is the same policy's, and a divergence of about log(700) is added to it
    assert 0.0 < taught[0] - plain[0] < 0.1 * 20


def test_gradients_of_both_losses_add_up():
    """d (surrogate + weight * divergence) / d matrix and d hidden, against differences in 64 bits along a direction."""
    import torch
    import paper_2606_18954_gb300 as P
    from distill_ref import exact, inputs
    from vocab_ref import head_exact
    P.build()
    gp = P.GraphPO()
    T, V, d, k = 24, 300, 64, 7
    h, w, ids, t = inputs(T, V, d, k, torch.float16, seed=8, tail=True, sure=4.0)
    y = torch.randint(0, V, (T,), device="cuda")
    g, share = torch.randn(T, device="cuda"), torch.full((T,), 0.3, device="cuda")
    head = gp.vocab_logp(h, w, y)
    grads = gp.vocab_grad(h, w, y, head["lse"], g, logp=head["logp"])
    far = gp.vocab_distill(h, w, ids, t, tail=True)
    more = gp.vocab_distill_grad(h, w, ids, far["delta"], far["rest"], far["rest_lse"], share, accumulate=True,
                                 out={"d_hidden": torch.empty_like(h), "d_weight": grads["d_weight"]})
    gp.check()
    dh = grads["d_hidden"].double() + more["d_hidden"].double()
    a, b = head_exact(h, w, y, 1.0, g), exact(h, w, ids, t, tail=True, g=share)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    uh, uw = (torch.randn(x.shape, generator=gen, device="cuda", dtype=torch.float64) for x in (h, w))
    step = 1e-5

    def loss(hh, ww):
        z = hh @ ww.t()
        logq = torch.log_softmax(z, 1)
        p = logq.exp().gather(1, ids.long())
        q = t.double().exp()
        qr, pr = (1 - q.sum(1)).clamp(min=0), 1 - p.sum(1)
        kl = (q * (t.double() - logq.gather(1, ids.long()))).sum(1) + qr * (qr / pr).log()
        return float((g.double() * logq.gather(1, y[:, None])[:, 0]).sum() + (share.double() * kl).sum())
    slope = (loss(h.double() + step * uh, w.double() + step * uw) - loss(h.double() - step * uh, w.double() - step * uw)) / (2 * step)
    got = float((dh * uh).sum() + (grads["d_weight"].double() * uw).sum())
    # the roundings of both gradients (the matrix's once more, as it is added to), and of the differences
    tol = float(((a["t_d_hidden"] + b["t_d_hidden"]) * uh.abs()).sum() + ((a["t_d_weight"] + b["t_d_weight"] + 2.0 ** -10 * (
        a["d_weight"].abs() + b["d_weight"].abs())) * uw.abs()).sum()) + 1e3 * 20 ** 3 * step ** 2 + 1e-6
    assert abs(got - slope) <= tol, (got, slope, tol)
