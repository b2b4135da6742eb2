"""Statistics of adjusted logits that are asked for alone, with and without a target, on the GPU against the formulas in 64 bits."""
import pytest

from test_gpu_logits import CASES, P, _types, gp  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R, V, dtype, kw", CASES, ids=lambda x: str(x).replace(" ", ""))
def test_without_a_target(gp, R, V, dtype, kw):  # noqa: F811
    """Of every row, as where the adjusted logits are written, too."""
    import torch
    from logits_ref import exact, inputs, near
    z, _, how = inputs(R, V, _types()[dtype], seed=V + R, **kw)
    want = exact(z, None, how)
    for entropy in (False, True):
        f = gp.logits_adjust(z, entropy=entropy, **how)
        gp.check()
        assert set(f) == {"lse", "entropy"} - (set() if entropy else {"entropy"})
        for k in f:
            near(f[k], want[k], want["t_" + k], k)
    h = gp.logits_adjust(z, lse=False, entropy=True, **how)
    gp.check()
    assert set(h) == {"entropy"} and torch.equal(h["entropy"].view(torch.int32), f["entropy"].view(torch.int32))  # (a NaN equals itself)


# (more entries that a list names than a CTA looks at in one round, in every span and for more rows than a cluster's CTAs have; a
# vocabulary of several spans for as many rows as a batch has; everything at once)
MORE = [(2, 70001, "bf16", dict(biases=70001, masks=2)), (5, 150001, "f32", dict(biases=150001, history=20000, pad=1)),
        (200, 151936, "bf16", dict(history=9000, masks=3)), (700, 9001, "f16", dict(history=9000, biases=9001, masked=0.5, temperature=True))]


@pytest.mark.parametrize("R, V, dtype, kw", MORE, ids=lambda x: str(x).replace(" ", ""))
def test_long_lists_and_vocabularies(gp, R, V, dtype, kw):  # noqa: F811
    import torch
    from logits_ref import exact, inputs, near
    z, y, how = inputs(R, V, _types()[dtype], seed=V + R, **kw)
    g, e = torch.randn(R, device="cuda"), torch.randn(R, device="cuda") * 0.1
    ref = exact(z, y, how, g, e)
    f = gp.logits_adjust(z, y, entropy=True, **how)
    d = gp.logits_grad(z, y, f["lse"], f["logp"], g, entropy=f["entropy"], grad_entropy=e, **how)["d_logits"]
    gp.check()
    for k in f:
        near(f[k], ref[k], ref["t_" + k], k)
    near(d, torch.where(torch.isfinite(ref["d_logits"]), ref["d_logits"], 0.0), ref["t_d_logits"], "d_logits")


@pytest.mark.parametrize("R, V, dtype, kw", [(1, 20000, "bf16", dict(masks=1)), (40, 5001, "f16", dict(masked=0.4, biases=20, masks=3, pad=1)),
                                             (700, 1003, "f32", dict(masked=0.4, temperature=True))], ids=lambda x: str(x).replace(" ", ""))
def test_written_with_a_target(gp, R, V, dtype, kw):  # noqa: F811
    """Logits and log-probabilities in one call: rows without a target have logp 0, and lse and entropy of what is written."""
    import torch
    from logits_ref import exact, inputs, near
    from vocab_ref import EPS, TINY
    dt = _types()[dtype]
    z, y, how = inputs(R, V, dt, seed=V + R, **kw)
    z = torch.where(torch.isnan(z) & (y < 0)[:, None], 0.5, z)  # (rows without a target are read here)
    ref, every = exact(z, y, how), exact(z, None, how)
    f = gp.logits_adjust(z, y, write=dt, entropy=True, **how)
    gp.check()
    near(f["logp"], ref["logp"], ref["t_logp"], "logp")
    for k in ("lse", "entropy"):
        near(f[k], every[k], every["t_" + k], k)
    t = every["t_logits"] + EPS.get(dt, 2.0 ** -24) * torch.where(torch.isfinite(every["logits"]), every["logits"].abs(), 0.0) + TINY.get(dt, 0.0)
    near(f["logits"], every["logits"].to(dt).double().where(torch.isinf(every["logits"].to(dt)), every["logits"]), t, "logits")
