"""Logits of hidden rows that are zeros but for one entry: their products add without a rounding, so that what is given
back for the tensor cores' dropped bits is the error.  It stays within its documented size: per 16 products of a run
(128 up to 16 tokens, else 512), 0.12 (bf16) or 0.17 (fp16) of 2^-23 of the logit."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T", [9, 200])
@pytest.mark.parametrize("d", [16, 136, 1024])
def test_one_entry_per_row(dtype, T, d):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as P
    P.build()
    gp = P.GraphPO()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float16
    V = 20003
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d)
    w = (torch.randn(V, d, generator=gen, device="cuda") * 4).to(dt)
    h = torch.zeros(T, d, device="cuda", dtype=dt)
    h[torch.arange(T), torch.arange(T) * 7 % d] = 4.0
    y = torch.randint(0, V, (T,), generator=gen, device="cuda")
    out = gp.vocab_logp(h, w, y)
    gp.check()
    z = h.double() @ w.double().t()
    lse = torch.logsumexp(z, 1)
    zy = z.gather(1, y[:, None])[:, 0]
    run = min(-(-d // 16) * 16, 128 if T <= 16 else 512)
    given = (0.17 if dtype == "f16" else 0.12) * (run / 16) * 2.0 ** -23
    # the scale's change on the logits, and a few roundings of logits, scale, maximum and results (each 2^-24 of the
    # largest logit), and of the sums' logarithm
    big = z.abs().amax(1)
    tol = (given + 8 * 2.0 ** -24) * big + 64 * 2.0 ** -24
    assert torch.all((out["lse"].double() - lse).abs() <= tol), float(((out["lse"].double() - lse).abs() / tol).max())
    tol = (given + 8 * 2.0 ** -24) * (big + zy.abs()) + 64 * 2.0 ** -24
    assert torch.all((out["logp"].double() - (zy - lse)).abs() <= tol)
