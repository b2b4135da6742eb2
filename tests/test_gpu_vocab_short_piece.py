"""A vocabulary whose last piece has fewer steps of k than d_hidden's k has parts: the first part of that piece is empty,
and its epilogue still has to add what the rounding of dz took at the targets of the piece's rows."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gp():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as pkg
    pkg.build()
    return pkg.GraphPO()


def test_targets_in_the_last_rows(gp):
    import torch
    # T x V in pieces of at most 512 MiB of dz: 117 pieces of 29952 rows, the last of 16 (one step of 64 k), d_hidden's
    # k in two parts
    T, V, d = 8777, 3474448, 8
    assert V % 29952 == 16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    w = (torch.randn(V, d, generator=gen, device="cuda") * 0.5).bfloat16()
    h = torch.randn(T, d, generator=gen, device="cuda").bfloat16()
    y = torch.full((T,), -1, device="cuda", dtype=torch.int32)
    at = torch.arange(0, T, 50, device="cuda")
    y[at] = (V - 16 + torch.arange(len(at), device="cuda") % 16).int()
    g = torch.where(torch.rand(T, generator=gen, device="cuda") < 0.5, -1.0, 1.0) * (1 + torch.rand(T, generator=gen, device="cuda"))
    f = gp.vocab_logp(h, w, y)
    out = gp.vocab_grad(h, w, y, f["lse"], g, d_weight=False)
    gp.check()
    err = once = 0.0
    for a in at.split(16):
        z = h[a].double() @ w.double().t()
        dz = -g[a].double()[:, None] * torch.softmax(z, 1)
        dz[torch.arange(len(a), device="cuda"), y[a].long()] += g[a].double()
        want = dz @ w.double()
        err += float((out["d_hidden"][a].double() - want).square().sum())
        once += float((want.bfloat16().double() - want).square().sum())
        del z, dz
    # p of the others is below 1e-4: next to nothing of dz's own rounding remains beside the target's, which is kept; without
    # it that entry's rounding alone is as large as the result's: a ratio of sqrt(2)
    assert (err / once) ** 0.5 < 1.1, (err / once) ** 0.5
    assert not out["d_hidden"][y < 0].any()
