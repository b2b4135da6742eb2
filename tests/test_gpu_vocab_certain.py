"""The gradient of nearly certain tokens: with vocab_logp's logp, dz at the target is 1 - p to its own last digits.

Each token's gradient is held against 64 bits by itself (a norm over all of them would be that of the uncertain ones).
Bounds, per element of d_hidden: dz is rounded to the type (its target's entry to 2^-17 at most, the rounding's rest being
kept), each p has the relative error of the logits and lse, (2 d / 16 + 32) roundings of the sum of |products| each, 1 - p as
a sum of the others' p has the same, and the result is rounded once; an fp16 dz is a multiple of 2^-25 2^-13 of the
call's largest gradient at worst."""
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
@pytest.mark.parametrize("shape", [(64, 4000, 256, False), (64, 4000, 256, True), (300, 1000, 2304, True), (5000, 600, 64, False)])
def test_nearly_certain_tokens(gp, dtype, shape):
    import torch
    from vocab_ref import EPS, TINY, U
    T, V, d, entropy = shape
    dt = torch.bfloat16 if dtype == "bf16" else torch.float16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T + d)
    w = (torch.randn(V, d, generator=gen, device="cuda") * (1.5 / d ** 0.5)).to(dt)
    y = torch.randint(0, V, (T,), generator=gen, device="cuda")
    row = w[y].float()
    h = (row * (torch.linspace(13.0, 25.0, T, device="cuda")[:, None] / row.square().sum(1, keepdim=True))).to(dt)
    g = torch.where(torch.rand(T, generator=gen, device="cuda") < 0.5, -1024.0, 1024.0)
    e = torch.full((T,), 8.0, device="cuda") if entropy else None
    f = gp.vocab_logp(h, w, y, entropy=True)
    kw = dict(entropy=f["entropy"], grad_entropy=e, logp=f["logp"])
    out = gp.vocab_grad(h, w, y, f["lse"], g, **kw)
    gp.check()
    z = h.double() @ w.double().t()
    logq = torch.log_softmax(z, 1)
    p = logq.exp()
    at = torch.arange(T, device="cuda")
    others = p.clone()
    others[at, y] = 0
    one_less = others.sum(1)                                    # 1 - p of the target, with all its digits
    assert 1e-9 < float(one_less.min()) < 1e-6 and float(one_less.max()) > 1e-3
    logq[at, y] = torch.log1p(-one_less)
    ent = -(p * logq).sum(1)
    dz = -g.double()[:, None] * p
    dz[at, y] = g.double() * one_less
    if entropy:
        dz = dz - e.double()[:, None] * p * (logq + ent[:, None])
    want = dz @ w.double()
    tz = (2 * d / 16 + 32) * U * (h.double().abs() @ w.double().abs().t()).amax(1)
    rel = 4 * tz + 64 * U * (torch.logsumexp(z, 1) + 1)
    ez = (EPS[dt] + rel[:, None] * (1 + (logq.abs() if entropy else 0))) * dz.abs()
    if entropy:  # the entropy's own error, a sum of terms p |log p| with the errors of p
        ez = ez + e.double()[:, None] * p * (rel * (ent + (p * logq.abs()).sum(1)))[:, None]
    # (the target's entry: the terms of its two parts, which may cancel)
    part = g.double().abs() * one_less + (e.double() * (logq[at, y].abs() + ent) if entropy else 0)
    ez[at, y] = (2.0 ** -17 + 4 * rel) * part
    if dtype == "f16":
        ez = ez + 2.0 ** -25 * 2.0 ** -13 * (1024.0 + 24 * 8.0 * entropy)
    tol = (ez @ w.double().abs()) * (1 + EPS[dt]) + EPS[dt] * want.abs() + TINY[dt] + (2 * V / 16 + 32) * U * (dz.abs() @ w.double().abs())
    err = (out["d_hidden"].double() - want).abs()
    bad = (err > tol).any(1)
    assert not bad.any(), (int(bad.sum()), one_less[bad][:5], (err / tol).amax(1)[bad][:5])
    # the same bits again, and a token's gradient is the same for either output alone
    again = gp.vocab_grad(h, w, y, f["lse"], g, d_weight=False, **kw)
    assert torch.equal(again["d_hidden"], out["d_hidden"])


def test_without_logp_as_before_and_refusals(gp):
    """Without logp the gradient is the difference's; a logp of another type, size or device is refused."""
    import torch
    from vocab_ref import close, head_exact, head_inputs
    T, V, d = 200, 700, 96
    h, w, y = head_inputs(T, V, d, torch.bfloat16, masked=0.2, seed=4)
    g = torch.randn(T, device="cuda")
    f = gp.vocab_logp(h, w, y)
    ref = head_exact(h, w, y, 1.0, g)
    for lp in (None, f["logp"]):
        out = gp.vocab_grad(h, w, y, f["lse"], g, logp=lp)
        gp.check()
        for k in out:
            close(out[k], ref[k], ref["t_" + k], (k, lp is None))
    with pytest.raises(TypeError):
        gp.vocab_grad(h, w, y, f["lse"], g, logp=f["logp"].double())
    with pytest.raises(ValueError):
        gp.vocab_grad(h, w, y, f["lse"], g, logp=f["logp"][1:])
    with pytest.raises(ValueError):
        gp.vocab_grad(h, w, y, f["lse"], g, logp=f["logp"].cpu())


def test_at_the_c_entries(gp):
    """gpo_vocab_grad is gpo_vocab_grad_logp without logp; a logp off its 4 bytes is refused."""
    import ctypes

    import torch
    import paper_2606_18954_gb300 as P
    from paper_2606_18954_gb300 import binding as B
    from vocab_ref import head_inputs
    L = P.load()
    T, V, d = 100, 300, 64
    h, w, y = head_inputs(T, V, d, torch.bfloat16, seed=6)
    g = torch.randn(T + 1, device="cuda")[:T]
    f = gp.vocab_logp(h, w, y)
    want = {lp is None: gp.vocab_grad(h, w, y, f["lse"], g, logp=lp) for lp in (None, f["logp"])}
    gp.check()
    v = B.CVocab(T, V, d, d, d, h.data_ptr(), w.data_ptr(), y.data_ptr(), 0, 4, 1.0)
    gi = B.VocabGradInputs(f["lse"].data_ptr(), g.data_ptr(), None, None)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    vg = B.VocabGrads(dh.data_ptr(), dw.data_ptr(), d, d, 0)
    room = torch.empty(B.vocab_workspace_size(v, True), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    tail = (ctypes.byref(vg), room.data_ptr(), room.numel(), stream)
    for lp in (None, 0, f["logp"].data_ptr()):
        if lp is None:
            assert L.gpo_vocab_grad(gp._h, ctypes.byref(v), ctypes.byref(gi), *tail) == 0
        else:
            assert L.gpo_vocab_grad_logp(gp._h, ctypes.byref(v), ctypes.byref(gi), lp, *tail) == 0
        gp.check()
        assert torch.equal(dh, want[not lp]["d_hidden"]) and torch.equal(dw, want[not lp]["d_weight"])
    assert L.gpo_vocab_grad_logp(gp._h, ctypes.byref(v), ctypes.byref(gi), f["logp"].data_ptr() + 2, *tail) == 5
    assert L.gpo_vocab_grad_logp(None, ctypes.byref(v), ctypes.byref(gi), None, *tail) == 1
