"""Distillation: digits of a teacher's remainder, of nearly certain and of flat distributions, against 64 bits.

The students' logits are exact: each hidden row is one 1 among zeros, a logit an element of the matrix (bf16).  A logit's error is
then that of its scaling, below 4 roundings of itself, a probability's that of two logits (8), of an approximate exponential (4),
and of its sums (64), each of itself."""
import math

import pytest

from test_gpu_distill import P, gp  # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _student(T, V, d, size, lift):
    """hidden, weight, the logits: token t's are column t % d of the matrix, of a normal law, with one that is `lift` above."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(T + V)
    w = (torch.randn(V, d, generator=g, device="cuda") * size).bfloat16()
    top = torch.randint(0, V, (d,), generator=g, device="cuda")
    if lift:
        w[top, torch.arange(d, device="cuda")] = (lift + 4 * torch.rand(d, generator=g, device="cuda")).bfloat16()
    h = torch.zeros(T, d, device="cuda")
    h[torch.arange(T, device="cuda"), torch.arange(T, device="cuda") % d] = 1.0
    z = w.double().t()[torch.arange(T, device="cuda") % d]
    return h.bfloat16(), w, z, top[torch.arange(T, device="cuda") % d], g


def _exact(z, ids, t):
    """Results with a tail in 64 bits from logits and log-probabilities: loss, delta, rest, and p, q of the entries and the others."""
    import torch
    t = t.double()
    mass = torch.logsumexp(t, 1).clamp(min=0)[:, None]
    lq = t - mass
    q = lq.exp()
    inside = torch.zeros_like(z, dtype=torch.bool).scatter(1, ids, True)
    p_all = torch.softmax(z, 1)
    p, pr = p_all.gather(1, ids), torch.where(inside, 0.0, p_all).sum(1)
    first = q.argmax(1, keepdim=True)
    others = q.scatter(1, first, 0.0).sum(1)
    # 1 - sum q: of the largest by expm1
    qr = torch.where(mass[:, 0] > 0, 0.0, (-torch.expm1(lq.gather(1, first)[:, 0]) - others).clamp(min=0))
    # log p of a nearly certain token: by the others' sum
    big = p.argmax(1, keepdim=True)
    rest = p.scatter(1, big, 0.0).sum(1) + pr
    lp = torch.log_softmax(z, 1).gather(1, ids)
    lp = lp.scatter(1, big, torch.where(rest < 0.5, torch.log1p(-rest), lp.gather(1, big)[:, 0])[:, None])
    loss = torch.where(q > 0, q * (lq - lp), 0.0).sum(1) + torch.where(qr > 0, qr * (qr.log() - pr.log()), 0.0)
    delta = torch.where((p > 0.5) & (q > 0.5), (1 - q.double()) - (1 - p), p - q)
    return dict(loss=loss, delta=delta, rest=pr - qr, p=p, q=q, pr=pr, qr=qr, lq=lq, lp=lp, others=others, unsure=rest)


@pytest.mark.parametrize("teacher", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("left", [1e-2, 1e-4, 1e-5, 1e-6, 1e-7])
def test_nearly_certain_teachers(gp, left, teacher):  # noqa: F811
    """One entry of probability 1 - left, 30 that share nine tenths of it, the remainder a tenth.  The largest entry's 1 - q is within a
    rounding and a half by expm1, exponentials are good to 2^-22: q_r is off by 6 roundings of 1 - q.  (In 16 bits log q of the
    largest is what it is rounded to, and the sum may pass 1.)"""
    import torch
    T, V, d, k = 64, 500, 64, 31
    h, w, z, top, g = _student(T, V, d, 1.0, 12.0)
    share = torch.rand(T, k - 1, generator=g, device="cuda", dtype=torch.float64) + 0.1
    share = share / share.sum(1, keepdim=True) * 0.9 * left
    order = torch.rand(T, V, generator=g, device="cuda").scatter(1, top[:, None], 2.0)
    ids = order.topk(k, dim=1).indices
    t = torch.cat([torch.full((T, 1), math.log1p(-left), dtype=torch.float64, device="cuda"), share.log()], 1)
    by = torch.rand(T, k, generator=g, device="cuda").argsort(1)
    ids, t = ids.gather(1, by), t.gather(1, by).to({"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[teacher])
    ref = _exact(z, ids, t)
    f = gp.vocab_distill(h, w, ids, t, tail=True)
    gp.check()
    size = float(z.abs().amax())
    p_err = (8 * size + 4 + 64) * U                     # of a probability below 1/2, of itself
    q_err = 6 * U * (ref["others"] + ref["qr"])         # of q_r, and of 1 - q
    over = torch.where(ref["qr"] == 0, 8 * U * ref["others"] + 2 * U * torch.expm1(torch.logsumexp(t.double(), 1)).clamp(min=0), 0.0)
    tol = p_err * ref["pr"] + q_err + 2 * over + 2 * U * (ref["pr"] + ref["qr"])
    assert bool(((f["rest"].double() - ref["rest"]).abs() <= tol).all()), float(((f["rest"].double() - ref["rest"]).abs() / tol).max())
    both = (ref["p"] > 0.5) & (ref["q"] > 0.5)
    tol = torch.where(both, (p_err * ref["unsure"] + q_err + 2 * over)[:, None], p_err * ref["p"] + (8 * U + over[:, None]) * ref["q"])
    err = (f["delta"].double() - ref["delta"]).abs()
    assert bool((err <= tol + 2 * U * ref["delta"].abs()).all()), float((err / tol).max())
    # the loss: log q is given (but for what a sum above 1 takes), log p of the largest is good as 1 - p is, others absolutely
    lp_err = torch.where(ref["p"] > 0.5, (p_err * ref["unsure"])[:, None], p_err + 4 * U * ref["lp"].abs())
    terms = ref["q"] * (ref["lq"] - ref["lp"]).abs()
    tol = (ref["q"] * (lp_err + 2 * over[:, None] + 4 * U * ref["lq"].abs()) + 8 * U * terms).sum(1)
    gap = torch.where(ref["qr"] > 0, (ref["qr"].clamp(min=1e-300) / ref["pr"]).log(), 0.0)
    tol = tol + q_err * (gap.abs() + 40) + ref["qr"] * (p_err + 8 * U * (gap.abs() + 40)) + over + 40 * U * (terms.sum(1) + ref["qr"] * gap.abs())
    err = (f["loss"].double() - ref["loss"]).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T, V, d", [(5, 40, 72), (300, 200, 64)])
def test_the_whole_vocabulary_with_a_tail(gp, T, V, d, dtype):  # noqa: F811
    """Every token is an entry, log-probabilities rounded to few bits: q_r is 0 whatever their sum leaves, and delta p - q."""
    import torch
    from distill_ref import exact, inputs, near
    teacher = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    h, w, ids, t = inputs(T, V, d, V, torch.bfloat16, seed=T, tail=True, teacher=teacher)
    ref = exact(h, w, ids, t, tail=True)
    f = gp.vocab_distill(h, w, ids, t, tail=True, lse=True)
    gp.check()
    for name in ("lse", "rest_lse", "rest", "delta", "loss"):
        near(f[name], ref[name], ref["t_" + name], name)
    assert not f["rest"].any()


@pytest.mark.parametrize("T, V", [(64, 20000), (300, 131072)])
def test_flat_distributions(gp, T, V):  # noqa: F811
    """No token of either has much: p - q of the largest entry and of the others together are differences of small numbers, not
    of what they leave of 1."""
    import torch
    d, k = 64, 8
    h, w, z, _, g = _student(T, V, d, 0.25, 0.0)
    other = z + 0.25 * torch.randn(T, V, generator=g, device="cuda", dtype=torch.float64)
    t, ids = torch.log_softmax(other, 1).topk(k, dim=1)
    t = t.float()
    ref = _exact(z, ids, t)
    f = gp.vocab_distill(h, w, ids, t, tail=True)
    gp.check()
    # (z and log q below 16: 1 and 8 roundings of exponents, 12 of each probability's own, sums)
    p_err, q_err = (8 * 2 + 4 + 64 + 16) * U, 8 * U
    tol = p_err * ref["p"] + q_err * ref["q"]
    err = (f["delta"].double() - ref["delta"]).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    err = (f["rest"].double() - ref["rest"]).abs()
    assert bool((err <= tol.sum(1)).all()), float((err / tol.sum(1)).max())
    # log q_r and log p_r are log1p of the entries' sums
    assert bool((ref["qr"] > 0.5).all()) and bool((ref["pr"] > 0.5).all())
    terms = ref["q"] * (ref["lq"] - ref["lp"])
    want = terms.sum(1) + ref["qr"] * (torch.log1p(-ref["q"].sum(1)) - torch.log1p(-ref["p"].sum(1)))
    tol = (ref["q"] * (p_err + 8 * U * (ref["lq"].abs() + ref["lp"].abs())) + 40 * U * terms.abs()).sum(1) + 2 * tol.sum(1)
    err = (f["loss"].double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
