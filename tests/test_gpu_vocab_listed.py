"""Log-probabilities of a short masked batch under a large head: up to 256 tokens, whose parts one CTA per row joins,
and so many products that the tokens with a target are listed and their rows gathered first."""
import pytest

pytestmark = pytest.mark.gpu

LISTED = 1 << 37  # products from which on the tokens are listed


@pytest.fixture(scope="module")
def gp():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as pkg
    pkg.build()
    return pkg.GraphPO()


def _masks(T):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    at = torch.arange(T, device="cuda")
    return {"some": torch.rand(T, generator=g, device="cuda") < 0.4, "the first": at == 0, "the last": at == T - 1,
            "all but one": at != T // 3, "all": at >= 0, "none": at < 0}


@pytest.mark.parametrize("shape", [(256, 131072, 4096, "bf16"), (140, 129000, 8192, "f16")])
def test_short_masked_batch(gp, shape):
    import torch
    from vocab_ref import close, head_exact, head_inputs
    T, V, d, dtype = shape
    assert T * V * d >= LISTED
    h, w, y0 = head_inputs(T, V, d, torch.bfloat16 if dtype == "bf16" else torch.float16, seed=T)
    ref = head_exact(h, w, y0, 1.0)  # (a token's results do not depend on which others are masked)
    for what, drop in _masks(T).items():
        y = torch.where(drop, -1, y0)
        hidden = torch.where(drop[:, None], float("nan"), h)
        # what an earlier call left in the workspace is not this call's result
        gp.vocab_logp(h.flip(0), w, y0.flip(0), entropy=True)
        out = gp.vocab_logp(hidden, w, y, entropy=True)
        plain = gp.vocab_logp(hidden, w, y)
        gp.check()
        for k in ("logp", "lse", "entropy"):
            close(out[k][~drop], ref[k][~drop], ref["t_" + k][~drop], (what, k))
            assert not out[k][drop].any(), (what, k)
        for k in ("logp", "lse"):
            close(plain[k][~drop], ref[k][~drop], ref["t_" + k][~drop], (what, k))
            assert not plain[k][drop].any(), (what, k)


def test_a_target_past_the_vocabulary_is_reported(gp):
    import torch
    import paper_2606_18954_gb300 as P
    from vocab_ref import head_inputs
    T, V, d = 256, 131072, 4096
    h, w, y = head_inputs(T, V, d, torch.bfloat16, seed=1)
    for at in (0, 100, T - 1):
        bad = y.clone()
        bad[at] = V
        gp.vocab_logp(h, w, bad)
        with pytest.raises(P.GraphPOError) as e:
            gp.check()
        assert e.value.code == 2
    gp.vocab_logp(h, w, y)
    gp.check()
