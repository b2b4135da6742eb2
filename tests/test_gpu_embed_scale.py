"""The embedding's scale multiplies in fp32: one that is infinite there is refused, the largest that is not is taken."""
import pytest

pytestmark = pytest.mark.gpu


def test_scales_at_the_ends_of_fp32():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as P
    P.build()
    gp = P.GraphPO()
    table = torch.tensor([[0.5, -0.25, 0.0, 0.125]], device="cuda").repeat(3, 1)
    ids = torch.tensor([0, -1, 2], device="cuda")
    top = float(torch.finfo(torch.float32).max)
    x = gp.embed(table, ids, scale=top)
    gp.check()
    assert torch.equal(x, torch.where((ids >= 0)[:, None], table * top, 0.0))
    for scale in (1e39, -1e39, 1e300):
        for call in (lambda: gp.embed(table, ids, scale=scale), lambda: gp.embed_grad(table, ids, 3, scale=scale)):
            with pytest.raises(P.GraphPOError) as e:
                call()
            assert e.value.code == 1
    gp.check()
