"""Tokens whose teacher gives no entry a probability, among others that have one."""
import math

import pytest

from test_gpu_distill import P, _types, gp  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T, V, d, dtype", [(40, 500, 64, "bf16"), (300, 700, 264, "f16"), (5000, 700, 64, "bf16")])
def test_teachers_of_nothing_have_no_gradient(gp, T, V, d, dtype):  # noqa: F811
    """Their ids are given, their logits are -inf, their gradient of the loss is not 0: their results are 0, and their hidden rows,
    which hold NaN, infinities, or states whose logits are above 100, reach no other result."""
    import torch
    from distill_ref import exact, inputs, near
    dt = _types()[dtype]
    h, w, ids, t = inputs(T, V, d, 8, dt, seed=T)
    to = 1024.0 if dtype == "f16" else 1.0
    g = (torch.rand(T, device="cuda") + 0.5) * to / T
    none = torch.zeros(T, dtype=torch.bool, device="cuda")
    none[::3] = True
    at = torch.nonzero(none)[:, 0]
    t[at] = -math.inf
    big = w[torch.randint(0, V, (len(at),), device="cuda")].double()
    rows = big * (150.0 / big.square().sum(1, keepdim=True))
    assert float((rows @ w.double().t()).amax()) > 100.0
    bad = torch.tensor([math.nan, math.inf, -math.inf], dtype=torch.float64, device="cuda")[torch.arange(len(at), device="cuda") % 3]
    rows = torch.where((torch.arange(len(at), device="cuda") % 2 == 0)[:, None], bad[:, None], rows)
    h[at] = rows.to(dt)
    ref = exact(h, w, ids, t, g=g)
    f = gp.vocab_distill(h, w, ids, t, lse=True)
    gp.check()
    for name in ("lse", "rest_lse", "rest", "delta", "loss"):
        near(f[name], ref[name], ref["t_" + name], name)
        assert not f[name][at].any()
    r = gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g)
    gp.check()
    assert not r["d_hidden"][at].any()
    for name in ("d_hidden", "d_weight"):
        near(r[name], ref[name], ref["t_" + name], name)


def test_nan_is_no_zero(gp):  # noqa: F811
    """A token whose delta or rest is NaN has a gradient, which is NaN."""
    import torch
    from distill_ref import inputs
    h, w, ids, t = inputs(12, 300, 64, 4, torch.bfloat16, seed=1)
    g = torch.ones(12, device="cuda")
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    for j in range(4):
        delta = z(12, 4)
        delta[3, j] = math.nan
        r = gp.vocab_distill_grad(h, w, ids, delta, z(12), z(12), g)
        gp.check()
        assert bool(torch.isnan(r["d_hidden"][3]).all()) and not r["d_hidden"][4:].any()
    rest = z(12)
    rest[3] = math.nan
    r = gp.vocab_distill_grad(h, w, ids, z(12, 4), rest, z(12), g)
    gp.check()
    assert bool(torch.isnan(r["d_hidden"][3]).all()) and not r["d_hidden"][4:].any()
