"""Distillation with numbers that are none: a student's logits, a teacher's."""
import math

import pytest

from test_gpu_distill import P, gp  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T", [5, 300])
def test_a_logit_outside_the_entries(gp, T, tail):  # noqa: F811
    """A row of the matrix that no entry names: NaN in it makes every token's results NaN, as its log-probabilities; an infinite
    element those of the tokens whose logit is not -inf by it."""
    import torch
    from distill_ref import inputs
    V, d, k = 600, 64, 6
    h, w, ids, t = inputs(T, V, d, k, torch.bfloat16, seed=T, tail=tail)
    unused = torch.ones(V, dtype=torch.bool, device="cuda")
    unused[ids.flatten().long()] = False
    v = int(torch.nonzero(unused)[-1])
    ids[1] = -1  # (a token without a teacher)
    live = torch.ones(T, dtype=torch.bool, device="cuda")
    live[1] = False
    c = int(torch.nonzero((h[live] < 0).any(0) & (h[live] > 0).any(0))[0])  # a column of both signs
    y = torch.zeros(T, dtype=torch.int32, device="cuda")
    g = torch.ones(T, device="cuda")
    bad = w.clone()
    bad[v, c] = math.nan
    assert bool(torch.isnan(gp.vocab_logp(h, bad, y)["lse"]).all())
    f = gp.vocab_distill(h, bad, ids, t, tail=tail, lse=True)
    gp.check()
    for name in f:
        assert bool(torch.isnan(f[name][live]).all()), name
        assert not f[name][1].any(), name
    r = gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g)
    gp.check()
    assert bool(torch.isnan(r["d_hidden"][live]).all()) and not r["d_hidden"][1].any()
    bad = w.clone()
    bad[v, c] = math.inf
    f = gp.vocab_distill(h, bad, ids, t, tail=tail, lse=True)
    gp.check()
    low = live & (h[:, c] < 0)
    z = h.double() @ w.double().t()
    z[:, v] = -math.inf
    want = torch.logsumexp(z, 1)
    assert bool(low.any()) and bool((live & ~low).any())
    for name in f:
        assert bool(torch.isnan(f[name][live & ~low]).all()), name
        assert bool(torch.isfinite(f[name][low]).all()), name
    # (products of 64 terms: 2 d / 16 + 32 roundings of at most 64 in all; sums of exponentials)
    assert bool(((f["lse"].double() - want)[low].abs() <= 1e-4).all())


def test_entries_beside_logits_of_minus_infinity(gp):  # noqa: F811
    """All other tokens' logits are -inf: they have no probability, but the teacher's remainder is not theirs to lose."""
    import torch
    h = torch.ones(3, 64, device="cuda").bfloat16()
    w = torch.full((40, 64), -math.inf, device="cuda").bfloat16()
    w[:4] = 0.0
    ids = torch.arange(4, device="cuda").repeat(3, 1)
    t = torch.full((3, 4), math.log(0.2), device="cuda")
    f = gp.vocab_distill(h, w, ids, t, tail=True)
    gp.check()
    assert bool((f["loss"] == math.inf).all()) and bool((f["rest_lse"] == -math.inf).all())
    assert bool(((f["rest"] + 0.2).abs() < 1e-6).all()) and bool(((f["delta"] - 0.05).abs() < 1e-6).all())
    f = gp.vocab_distill(h, w, ids, t)
    gp.check()
    assert bool((f["loss"].abs() < 1e-6).all()) and bool((f["rest"] == 0).all())


def test_a_teachers_logit_past_the_largest_number(P, gp):  # noqa: F811
    """That is infinite with the scale, though not without."""
    import torch
    from distill_ref import inputs
    h, w, ids, t = inputs(9, 300, 64, 4, torch.bfloat16, seed=1)
    for value, scale in ((3e38, 2.0), (1e38, 10.0)):
        t[4, 2] = value
        gp.vocab_distill(h, w, ids, t, teacher_scale=scale)
        with pytest.raises(P.GraphPOError) as e:
            gp.check()
        assert e.value.code == 4
    t[4, 2] = -3e38  # (a token of probability 0)
    f = gp.vocab_distill(h, w, ids, t, teacher_scale=2.0)
    gp.check()
    assert all(bool(torch.isfinite(f[k]).all()) for k in f)
