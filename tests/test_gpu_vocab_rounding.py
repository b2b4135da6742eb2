"""How far the gradients are from one rounding of their exact values, where dz's own rounding to 16 bits is not kept: rows
of d_weight that are no token's target, and a policy that is sure of another token than the sampled one.  An entry of dz
rounds as the result does, to the same relative error; a sum of terms of random sign and direction then carries an
error of the size of the sum's own rounding beside it: together sqrt(2) of it, and a tenth more is left for the draw."""
import math

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


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("sure", ["of the target", "of another"])
@pytest.mark.parametrize("shape", [(500, 4000, 256), (2000, 6000, 1024), (5000, 3000, 128)])
def test_at_most_two_roundings(gp, dtype, sure, shape):
    import torch
    T, V, d = shape
    dt = torch.bfloat16 if dtype == "bf16" else torch.float16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    w = (torch.randn(V, d, generator=gen, device="cuda") * 2 / d ** 0.5).to(dt)
    y, other = (torch.randint(0, V // 2, (T,), generator=gen, device="cuda") for _ in range(2))
    row = w[y if sure == "of the target" else other].float()
    lean = torch.rand(T, 1, generator=gen, device="cuda") * 12
    h = (0.5 * torch.randn(T, d, generator=gen, device="cuda") + row * (lean / row.square().sum(1, keepdim=True))).to(dt)
    g = torch.randn(T, generator=gen, device="cuda") * (512.0 if dtype == "f16" else 1.0) / T
    f = gp.vocab_logp(h, w, y)
    out = gp.vocab_grad(h, w, y, f["lse"], g, logp=f["logp"])
    gp.check()
    dz = -g.double()[:, None] * torch.softmax(h.double() @ w.double().t(), 1)
    dz[torch.arange(T, device="cuda"), y] += g.double()
    target = torch.zeros(V, dtype=torch.bool, device="cuda")
    target[y] = True
    assert not target[V // 2:].any()
    for k, want, rows in (("d_hidden", dz @ w.double(), slice(None)), ("d_weight", dz.t() @ h.double(), slice(None)),
                          ("d_weight", dz.t() @ h.double(), target), ("d_weight", dz.t() @ h.double(), ~target)):
        # (beside what is below the type's normal numbers, whose roundings are absolute)
        once = (want.to(dt).double() - want)[rows].norm()
        err = (out[k].double() - want)[rows].norm()
        assert float(err / once) < 1.1 * math.sqrt(2), (k, float(err / once))
