"""Entropies of rows that are nearly certain of one token: their digits."""
import pytest

from test_gpu_logits import P, _types, gp  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("R, V, pad", [(1, 40000, 0), (24, 9001, 1), (700, 1037, 3), (6, 140007, 2), (40, 20, 5)])
def test_entropy_of_nearly_certain_rows(gp, R, V, pad, dtype):  # noqa: F811
    """The largest logit lies 12 to 24 above a normal law's others, at any place, among special entries and at the row's ends too.
    The entropy is log(1 + s) + sum p d, of positive terms, s the others' sum relative to the largest and d the distance from it,
    whose relative error is that of s and of d.  (Where another logit is within 4 of it, in units of log 2, the largest may be in
    the sum, whose error is then one of 1 + s; the entropy is 0.2 or more.)  An exponent is a difference of products, each rounded, of up to the adjusted
    logits' size in units of log 2 (below 3 of theirs for both and the scale's rounding), an adjusted logit takes up to 8
    roundings, an exponential is good to 2^-22, sums of a thread and the joins to V / 256 + 128 roundings."""
    import math
    import torch
    from logits_ref import exact, inputs
    from vocab_ref import U
    dt = _types()[dtype]
    for kw in (dict(history=0, penalties=False), dict(history=40, biases=9, temperature=True), dict(masks=2, history=20)):
        z, y, how = inputs(R, V, dt, seed=R + V, pad=pad, **kw)
        g = torch.Generator(device="cuda")
        g.manual_seed(R)
        z.copy_(torch.where(torch.isfinite(z) & (z.abs() < 1e30), torch.randn(R, V, generator=g, device="cuda"), z.float()))
        y = y.long()
        y[::3] = torch.randint(0, min(V, 5), (len(y[::3]),), generator=g, device="cuda")
        y[1::7] = V - 1
        z[torch.arange(R, device="cuda"), y] = (12 + 12 * torch.rand(R, generator=g, device="cuda")).to(dt)
        ref = exact(z, None, how)
        want = ref["entropy"]
        left = torch.where(torch.isfinite(ref["logits"]), ref["logits"].abs(), 0.0).amax(1)
        tol = torch.where(want < 0.2, want, want + 1.0) * U * (V / 256 + 128 + 4 + (8 + 3) * (left + 30) * 1.4427) + 1e-12  # (64 bits: 1e-14 of lse)
        calls = [dict(), dict(write=torch.float32), dict(write=dt), dict(target=torch.full((R,), -1, device="cuda"), write=dt)]
        for call in calls:
            f = gp.logits_adjust(z, entropy=True, **call, **how)
            gp.check()
            err = (f["entropy"].double() - want).abs()
            assert bool((err <= tol).all()), (kw, call, float((err / want.clamp(min=1e-30)).max()), int((err > tol).sum()))
        own = z.clone(memory_format=torch.preserve_format)
        f = gp.logits_adjust(own, out={"logits": own, "entropy": torch.empty(R, device="cuda"), "lse": torch.empty(R, device="cuda")}, **how)
        gp.check()
        assert bool(((f["entropy"].double() - want).abs() <= tol).all())
        fine = torch.isfinite(ref["lse"])
        assert bool(((f["lse"].double() - ref["lse"])[fine].abs() <= ref["t_lse"][fine]).all())


def test_what_is_no_number_stays_so(gp):  # noqa: F811
    """NaN and +inf among the entries of a row, before or behind its largest; equal largest entries; rows of which nothing is left."""
    import math
    import torch
    V = 5000
    for dt in _types().values():
        for at in (0, 17, 2000, V - 1):
            for bad in (math.nan, math.inf):
                for top in (3, 1999, V - 2):
                    z = torch.randn(2, V, device="cuda").to(dt)
                    z[:, top] = 20.0
                    z[0, at] = bad
                    f = gp.logits_adjust(z, entropy=True)
                    gp.check()
                    assert math.isnan(f["lse"][0]) and math.isnan(f["entropy"][0]) and math.isfinite(f["lse"][1]) and math.isfinite(f["entropy"][1])
        z = torch.full((4, V), -math.inf, device="cuda", dtype=dt)
        z[1, 7] = 2.0
        z[2, [7, 8]] = 2.0      # (in one vector)
        z[3, [7, 4000]] = 2.0
        f = gp.logits_adjust(z, entropy=True)
        gp.check()
        for k, want in (("lse", [-math.inf, 2.0, 2 + math.log(2), 2 + math.log(2)]), ("entropy", [0.0, 0.0, math.log(2), math.log(2)])):
            for i, v in enumerate(want):
                assert float(f[k][i]) == v or abs(float(f[k][i]) - v) < 1e-6, (k, i, float(f[k][i]))
        for n in (3, 16, 17, 700):  # n equal entries anywhere
            z = torch.full((1, V), -math.inf, device="cuda", dtype=dt)
            z[0, torch.randperm(V, device="cuda")[:n]] = -4.5
            f = gp.logits_adjust(z, entropy=True)
            gp.check()
            assert abs(float(f["entropy"]) - math.log(n)) < 4e-6 and abs(float(f["lse"]) - math.log(n) + 4.5) < 4e-6
