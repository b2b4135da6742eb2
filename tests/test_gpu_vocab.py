"""gpo_vocab_logp and gpo_vocab_grad against their formulas in 64 bits (vocab_ref).

Sizes around the tiles (256 tokens x 256 vocabulary rows, 64 columns of k), single tokens, odd
widths and vocabularies, wider rows, masks that leave no token, masked rows full of NaN and
infinities, tokens without a gradient, several pieces of the vocabulary, added gradients, other
streams, captured calls, refusals.  A gradient is also held against differences of the loss."""
import ctypes
import math

import pytest

pytestmark = pytest.mark.gpu

SHAPE, INVALID, UNSUPPORTED, WORKSPACE, TIMEOUT = 2, 1, 5, 8, 7


@pytest.fixture(scope="module")
def gp():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as pkg
    pkg.build()
    return pkg.GraphPO()


def _types():
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16}


FORWARD = [  # tokens, vocabulary, width, pad, masked, scale
    (1, 1, 8, 0, 0.0, 1.0),
    (1, 2, 1, 0, 0.0, 0.5),
    (1, 1000, 64, 0, 0.0, 1.0),
    (2, 257, 65, 0, 0.0, 1.0),
    (5, 255, 63, 1, 0.5, 2.0),
    (127, 256, 128, 0, 0.0, 1.0),
    (129, 513, 200, 1, 0.2, 1.25),
    (255, 3001, 1024, 0, 0.0, 1.0),
    (256, 128, 333, 0, 1.0, 1.0),
    (257, 1025, 72, 0, 0.4, 0.7),
    (300, 700, 40, 0, 1.0, 1.0),
    (1000, 5003, 136, 1, 0.3, 1.0),
    (2561, 777, 320, 0, 0.05, 1.0),
    (9000, 300, 64, 0, 0.6, 1.0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", FORWARD)
def test_logp(gp, dtype, shape):
    import torch
    from vocab_ref import close, head_exact, head_inputs
    T, V, d, pad, masked, scale = shape
    h, w, y = head_inputs(T, V, d, _types()[dtype], pad, masked, seed=T, id_dtype=torch.int64 if T % 2 else torch.int32)
    out = gp.vocab_logp(h, w, y, scale=scale, entropy=True)
    plain = gp.vocab_logp(h, w, y, scale=scale)
    again = gp.vocab_logp(h, w, y, scale=scale, entropy=True)
    gp.check()
    ref = head_exact(h, w, y, scale)
    for k in ("logp", "lse", "entropy"):
        assert out[k].dtype == torch.float32 and out[k].shape == (T,)
        close(out[k], ref[k], ref["t_" + k], k)
        assert torch.equal(out[k], again[k]), k
        assert torch.equal(out[k][y < 0], torch.zeros_like(out[k][y < 0]))
    for k in ("logp", "lse"):
        close(plain[k], ref[k], ref["t_" + k], k)


def test_logp_of_listed_tokens(gp):
    """So many products that the tokens with a target are listed and their rows gathered first."""
    import torch
    from vocab_ref import close, head_exact, head_inputs
    T, V, d = 9000, 30011, 520
    assert T * V * d >= 1 << 37
    for masked in (0.4, 0.0):
        h, w, y = head_inputs(T, V, d, torch.bfloat16, masked=masked, seed=31)
        out = gp.vocab_logp(h, w, y, entropy=True)
        gp.check()
        for a in range(0, T, 3000):
            b = a + 3000
            ref = head_exact(h[a:b], w, y[a:b], 1.0)
            for k in ("logp", "lse", "entropy"):
                close(out[k][a:b], ref[k], ref["t_" + k], k)
                assert not out[k][a:b][y[a:b] < 0].any()
            del ref
    bad = y.clone()
    bad[17] = V
    import paper_2606_18954_gb300 as P
    gp.vocab_logp(h, w, bad)
    with pytest.raises(P.GraphPOError) as e:
        gp.check()
    assert e.value.code == SHAPE


def test_logp_is_as_exact_as_32_bits(gp):
    """2-norm errors of lse and logp against torch's own 32-bit products and sums of the same logits."""
    import torch
    from vocab_ref import head_exact, head_inputs
    for dtype in (torch.bfloat16, torch.float16):
        for T, V, d in ((40, 3000, 1024), (400, 6000, 2048)):
            h, w, y = head_inputs(T, V, d, dtype, seed=T)
            out = gp.vocab_logp(h, w, y)
            gp.check()
            ref = head_exact(h, w, y, 1.0)
            z = h.float() @ w.float().t()
            lse = torch.logsumexp(z, 1)
            plain = {"lse": lse, "logp": z.gather(1, y.long()[:, None])[:, 0] - lse}
            for k in plain:
                err = lambda x: float((x.double() - ref[k]).norm() / ref[k].norm())  # noqa: E731
                assert err(out[k]) <= max(1e-6, 1.5 * err(plain[k])), (k, dtype, T, err(out[k]), err(plain[k]))


def test_a_certain_token_keeps_its_digits(gp):
    """log pi of a token with almost all the probability is -(the others' sum), a number far below
    the logits' own rounding to 1: relative to it the error is that of the logits' differences."""
    import torch
    V, d = 5000, 64
    w = torch.zeros(V, d, device="cuda", dtype=torch.bfloat16)
    w[:, 0] = -1.0
    w[7, 0] = 1.0
    h = torch.zeros(3, d, device="cuda", dtype=torch.bfloat16)
    h[:, 0] = torch.tensor([10.0, 12.0, 8.0])
    out = gp.vocab_logp(h, w, torch.full((3,), 7, device="cuda", dtype=torch.int32), entropy=True)
    gp.check()
    z = 2.0 * h[:, 0].double()  # the target's logit above the others', exact
    others = (V - 1) * torch.exp(-z)
    want = -torch.log1p(others)
    assert torch.all((out["logp"].double() - want).abs() <= 64 * 2.0 ** -24 * 30 * want.abs())
    ent = torch.log1p(others) + others * z / (1 + others)
    assert torch.all((out["entropy"].double() - ent).abs() <= 64 * 2.0 ** -24 * 30 * ent)


def test_logp_extremes(gp):
    """Rows whose logits are NaN or infinite give what the formulas give (NaN); the others are not
    touched by them.  Large finite logits do not overflow."""
    import torch
    from vocab_ref import close, head_exact, head_inputs
    h, w, y = head_inputs(40, 600, 96, torch.bfloat16, seed=5)
    h = h.clone()
    h[3, 5] = math.nan
    h[9] = h[9] * 1e4
    h[17] = 0.0
    out = gp.vocab_logp(h, w, y, entropy=True)
    gp.check()
    assert math.isnan(float(out["logp"][3])) and math.isnan(float(out["lse"][3]))
    fine = torch.arange(40, device="cuda") != 3
    ref = head_exact(h[fine].contiguous(), w, y[fine].contiguous(), 1.0)
    for k in ("logp", "lse", "entropy"):
        close(out[k][fine], ref[k], ref["t_" + k], k)
    assert abs(float(out["lse"][17]) - math.log(600)) < 1e-5 and abs(float(out["entropy"][17]) - math.log(600)) < 1e-5


GRAD = [  # tokens, vocabulary, width, pad, masked, entropy, scale
    (1, 1, 8, 0, 0.0, False, 1.0),
    (1, 300, 1, 0, 0.0, True, 1.0),
    (3, 257, 65, 0, 0.0, False, 1.0),
    (63, 256, 264, 0, 0.0, True, 2.0),
    (64, 511, 256, 1, 0.0, False, 1.0),
    (65, 1000, 100, 0, 0.3, True, 1.0),
    (256, 129, 513, 0, 0.2, False, 0.7),
    (257, 2049, 128, 1, 0.0, True, 1.0),
    (700, 3003, 330, 0, 0.5, False, 1.25),
    (300, 500, 64, 0, 1.0, True, 1.0),
    (2200, 1500, 72, 0, 0.3, True, 1.0),
]


def _grads(T, y, seed, entropy, to=1.0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    gl = torch.randn(T, generator=g, device="cuda") * (to / T)
    gl[torch.rand(T, generator=g, device="cuda") < 0.3] = 0.0   # clipped tokens
    gl[y < 0] = math.nan                                       # never read
    ge = None
    if entropy:
        ge = torch.randn(T, generator=g, device="cuda") * (0.05 * to / T)
        ge[torch.rand(T, generator=g, device="cuda") < 0.3] = 0.0
        ge[y < 0] = math.nan
    return gl, ge


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", GRAD)
def test_grad(gp, dtype, shape):
    import torch
    from vocab_ref import close, head_exact, head_inputs
    T, V, d, pad, masked, entropy, scale = shape
    h, w, y = head_inputs(T, V, d, _types()[dtype], pad, masked, seed=T + 7)
    gl, ge = _grads(T, y, T, entropy, 512.0 if dtype == "f16" else 1.0)
    f = gp.vocab_logp(h, w, y, scale=scale, entropy=entropy)
    kw = dict(scale=scale, entropy=f.get("entropy"), grad_entropy=ge)
    out = gp.vocab_grad(h, w, y, f["lse"], gl, **kw)
    again = gp.vocab_grad(h, w, y, f["lse"], gl, **kw)
    gp.check()
    live = (torch.nan_to_num(gl) != 0) | (torch.nan_to_num(ge) != 0 if ge is not None else False)
    ref = head_exact(h, w, y, scale, torch.nan_to_num(gl), None if ge is None else torch.nan_to_num(ge))
    for k in ("d_hidden", "d_weight"):
        close(out[k], ref[k], ref["t_" + k], k)
        assert torch.equal(out[k], again[k]), k
    assert torch.equal(out["d_hidden"][~live | (y < 0)], torch.zeros_like(out["d_hidden"][~live | (y < 0)]))
    # one of the two alone
    only = gp.vocab_grad(h, w, y, f["lse"], gl, d_weight=False, **kw)
    assert set(only) == {"d_hidden"} and torch.equal(only["d_hidden"], out["d_hidden"])
    only = gp.vocab_grad(h, w, y, f["lse"], gl, d_hidden=False, **kw)
    assert set(only) == {"d_weight"} and torch.equal(only["d_weight"], out["d_weight"])
    gp.check()


# wide rows (logits of several accumulations), more tokens than are looked at in one go, all tokens on few targets
GRAD_MORE = [  # tokens, vocabulary, width, pad, masked, entropy, targets
    (70, 600, 2100, 0, 0.2, True, "any"),
    (300, 1000, 4096, 1, 0.0, False, "any"),
    (260, 300, 2056, 0, 0.3, True, "two"),
    (500, 900, 200, 0, 0.1, False, "one"),
    (4500, 700, 136, 0, 0.4, True, "two"),
    (9000, 300, 40, 0, 0.3, True, "any"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", GRAD_MORE)
def test_grad_wide_rows_and_frequent_targets(gp, dtype, shape):
    import torch
    from vocab_ref import close, head_exact, head_inputs
    T, V, d, pad, masked, entropy, which = shape
    h, w, y = head_inputs(T, V, d, _types()[dtype], pad, masked, seed=T + 70, sure=8.0, id_dtype=torch.int64)
    few = torch.tensor([V - 1, V - 1 if which == "one" else 5], device="cuda")
    if which != "any":
        y = torch.where(y < 0, y, few[torch.arange(T, device="cuda") % 2])
    gl, ge = _grads(T, y, T + 1, entropy, 512.0 if dtype == "f16" else 1.0)
    f = gp.vocab_logp(h, w, y, entropy=entropy)
    kw = dict(entropy=f.get("entropy"), grad_entropy=ge)
    out = gp.vocab_grad(h, w, y, f["lse"], gl, **kw)
    again = gp.vocab_grad(h, w, y, f["lse"], gl, **kw)
    gp.check()
    ref = head_exact(h, w, y, 1.0, torch.nan_to_num(gl), None if ge is None else torch.nan_to_num(ge))
    for k in ("d_hidden", "d_weight"):
        close(out[k], ref[k], ref["t_" + k], k)
        assert torch.equal(out[k], again[k]), k


@pytest.mark.parametrize("T", [4095, 4096, 4097, 5000])
def test_grad_of_many_tokens(gp, T):
    """Around the number of tokens from which on they are sorted: 32-bit ids, tokens without a target or a
    gradient, a vocabulary of fewer rows than there are SMs, and an id past the vocabulary."""
    import torch
    import paper_2606_18954_gb300 as P
    from vocab_ref import close, head_exact, head_inputs
    V, d = 150, 24
    h, w, y = head_inputs(T, V, d, torch.float16, 0, 0.3, seed=T, sure=6.0)
    gl, ge = _grads(T, y, T, True, 512.0)
    f = gp.vocab_logp(h, w, y, entropy=True)
    kw = dict(entropy=f["entropy"], grad_entropy=ge)
    out = gp.vocab_grad(h, w, y, f["lse"], gl, **kw)
    gp.check()
    ref = head_exact(h, w, y, 1.0, torch.nan_to_num(gl), torch.nan_to_num(ge))
    for k in ("d_hidden", "d_weight"):
        close(out[k], ref[k], ref["t_" + k], k)
    still = (y < 0) | ((torch.nan_to_num(gl) == 0) & (torch.nan_to_num(ge) == 0))
    assert still.any() and not out["d_hidden"][still].any()
    bad = y.clone()
    bad[T - 1] = V
    gp.vocab_grad(h, w, bad, f["lse"], gl, **kw)
    with pytest.raises(P.GraphPOError) as e:
        gp.check()
    assert e.value.code == SHAPE


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_grad_is_as_exact_as_one_rounding(gp, dtype):
    """The 2-norm error of the gradients against that of their exact values rounded once to the type: dz's own
    rounding to 16 bits, whose largest part (at the targets) is kept in fp32, may add little to it.  Its other
    entries are p g with sum of squares at most max p over the non-targets times (1 - p_target)^2, here below 0.2
    of the target's square: with the targets' part kept, sqrt(1 + 0.2) bounds the ratio."""
    import torch
    from vocab_ref import head_exact, head_inputs
    T, V, d = 500, 4000, 256
    h, w, y = head_inputs(T, V, d, _types()[dtype], seed=21, sure=6.0)
    gl = torch.randn(T, device="cuda") * (512.0 if dtype == "f16" else 1.0) / T
    f = gp.vocab_logp(h, w, y)
    out = gp.vocab_grad(h, w, y, f["lse"], gl)
    gp.check()
    ref = head_exact(h, w, y, 1.0, gl)
    z = h.double() @ w.double().t()
    p = torch.softmax(z, 1)
    at = torch.arange(T, device="cuda")
    py = p[at, y.long()].clone()
    p[at, y.long()] = 0
    share = (gl.double()[:, None] * p).square().sum() / (gl.double() * (1 - py)).square().sum()
    assert float(share) < 0.2
    for k in ("d_hidden", "d_weight"):
        once = (ref[k].to(out[k].dtype).double() - ref[k]).norm()
        assert float((out[k].double() - ref[k]).norm() / once) < math.sqrt(1.2), k


def test_grad_against_differences(gp):
    """The directional derivative of L = sum g logp + sum e entropy, by central differences in 64 bits."""
    import torch
    from vocab_ref import head_exact, head_inputs
    T, V, d = 90, 700, 48
    h, w, y = head_inputs(T, V, d, torch.float16, seed=3, sure=6.0)
    gl, ge = torch.randn(T, device="cuda"), torch.randn(T, device="cuda") * 0.3
    f = gp.vocab_logp(h, w, y, entropy=True)
    out = gp.vocab_grad(h, w, y, f["lse"], gl, entropy=f["entropy"], grad_entropy=ge)
    gp.check()
    ref = head_exact(h, w, y, 1.0, gl, ge)

    def loss(hh, ww):
        z = hh @ ww.t()
        q = torch.log_softmax(z, 1)
        at = torch.arange(T, device="cuda")
        return (gl.double() * q[at, y.long()]).sum() - (ge.double() * (q.exp() * q).sum(1)).sum()

    for k in range(4):
        torch.manual_seed(k)
        for name, dh, dw in (("d_hidden", torch.randn(T, d, device="cuda").double(), 0.0),
                             ("d_weight", 0.0, torch.randn(V, d, device="cuda").double())):
            e = 1e-5
            num = (loss(h.double() + e * dh, w.double() + e * dw) - loss(h.double() - e * dh, w.double() - e * dw)) / (2 * e)
            dirn = dh if name == "d_hidden" else dw
            got = (out[name].double() * dirn).sum()
            # the sum of the elements' bounds, and the differences' own error (e^2 third derivatives, 1e-16 L / e)
            tol = (ref["t_" + name] * dirn.abs()).sum() + 1e-6 * num.abs() + 1e-6
            assert abs(float(got - num)) <= float(tol), (name, float(got), float(num))


def test_grad_in_pieces(gp):
    """A vocabulary of several pieces (dz of one is at most 512 MiB): sums of d_hidden across them."""
    import torch
    from paper_2606_18954_gb300 import binding as B
    T, V, d = 30000, 20011, 16
    torch.manual_seed(1)
    w = (torch.randn(V, d, device="cuda") / 2).bfloat16()
    h = torch.randn(T, d, device="cuda").bfloat16()
    y = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    v = B.CVocab(T, V, d, d, d, None, None, None, 0, 4, 1.0)
    assert B.vocab_workspace_size(v, True) < 2 * T * V  # more than one piece
    gl = torch.randn(T, device="cuda")
    f = gp.vocab_logp(h, w, y)
    out = gp.vocab_grad(h, w, y, f["lse"], gl)
    gp.check()
    from vocab_ref import EPS, U
    W = w.double()
    dw = torch.zeros(V, d, device="cuda", dtype=torch.float64)
    tw = torch.zeros_like(dw)
    for a in range(0, T, 3000):
        H = h[a:a + 3000].double()
        p = torch.softmax(H @ W.t(), 1)
        dz = -gl[a:a + 3000, None].double() * p
        dz[torch.arange(3000), y[a:a + 3000].long()] += gl[a:a + 3000].double()
        want = dz @ W
        # as in vocab_ref, with the logits' error (d = 16: far below 1e-4 of p) in the rounding's slack
        tol = (EPS[torch.bfloat16] + 1e-4) * (dz.abs() @ W.abs()) + EPS[torch.bfloat16] * want.abs() + \
            (2 * V / 16 + 64) * U * (dz.abs() @ W.abs())
        err = (out["d_hidden"][a:a + 3000].double() - want).abs()
        assert torch.all(err <= tol), float((err - tol).max())
        dw += dz.t() @ H
        tw += dz.abs().t() @ H.abs()
    tol = (EPS[torch.bfloat16] + 1e-4 + (2 * T / 16 + 64) * U) * tw + EPS[torch.bfloat16] * dw.abs()
    assert torch.all((out["d_weight"].double() - dw).abs() <= tol)


def test_grad_added_to_what_is_there(gp):
    import torch
    from vocab_ref import EPS, close, head_exact, head_inputs
    T, V, d = 200, 900, 104
    h, w, y = head_inputs(T, V, d, torch.bfloat16, masked=0.2, seed=11)
    gl, _ = _grads(T, y, 4, False)
    f = gp.vocab_logp(h, w, y)
    base = (torch.randn(V, d, device="cuda") * 1e-3).bfloat16()
    for stride in (d, d + 3):  # with 16-byte rows and without
        wide = torch.zeros(V, stride, device="cuda", dtype=torch.bfloat16)
        dw = wide[:, :d]
        dw.copy_(base)
        out = gp.vocab_grad(h, w, y, f["lse"], gl, out={"d_weight": dw}, accumulate=True)
        gp.check()
        assert out["d_weight"] is dw and "d_hidden" not in out
        ref = head_exact(h, w, y, 1.0, torch.nan_to_num(gl))
        want = ref["d_weight"] + base.double()
        close(dw, want, ref["t_d_weight"] + EPS[torch.bfloat16] * want.abs(), "d_weight")
        assert not wide[:, d:].any()


def test_outputs_of_any_stride_stay_inside(gp):
    import torch
    from vocab_ref import close, head_exact, head_inputs
    T, V, d = 130, 513, 77
    h, w, y = head_inputs(T, V, d, torch.float16, masked=0.3, seed=12)
    gl, _ = _grads(T, y, 5, False, 64.0)
    f = gp.vocab_logp(h, w, y)
    bh = torch.full((T + 2, d + 5), 3.0, device="cuda", dtype=torch.float16)
    bw = torch.full((V + 2, d + 1), 3.0, device="cuda", dtype=torch.float16)
    out = {"d_hidden": bh[1:T + 1, 2:d + 2], "d_weight": bw[1:V + 1, 1:]}
    gp.vocab_grad(h, w, y, f["lse"], gl, out=out)
    gp.check()
    ref = head_exact(h, w, y, 1.0, torch.nan_to_num(gl))
    for k in out:
        close(out[k], ref[k], ref["t_" + k], k)
    out["d_hidden"].fill_(3.0)
    out["d_weight"].fill_(3.0)
    assert torch.all(bh == 3.0) and torch.all(bw == 3.0)


@pytest.mark.parametrize("d", [1, 5, 29, 37, 62, 63, 77, 100, 260, 333])
def test_what_lies_beside_the_gradients_rows_stays(gp, d):
    """Rows on 16-byte boundaries whose width is no multiple of 16 bytes: nothing past the width is written."""
    import torch
    from vocab_ref import close, head_exact, head_inputs
    T, V, stride = 130, 300, (d + 7) // 8 * 8 + (8 if d % 8 == 0 else 0)
    h, w, y = head_inputs(T, V, d, torch.bfloat16, seed=d, sure=6.0)
    gl, _ = _grads(T, y, 5, False)
    f = gp.vocab_logp(h, w, y)
    bh = torch.full((T, stride), 7.0, device="cuda", dtype=torch.bfloat16)
    bw = torch.full((V, stride), 7.0, device="cuda", dtype=torch.bfloat16)
    out = {"d_hidden": bh[:, :d], "d_weight": bw[:, :d]}
    gp.vocab_grad(h, w, y, f["lse"], gl, out=out)
    gp.check()
    ref = head_exact(h, w, y, 1.0, torch.nan_to_num(gl))
    for k in out:
        close(out[k], ref[k], ref["t_" + k], k)
    assert torch.all(bh[:, d:] == 7.0) and torch.all(bw[:, d:] == 7.0)


def test_no_tokens(gp):
    import torch
    w = torch.randn(300, 64, device="cuda").bfloat16()
    h = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    y = torch.empty(0, device="cuda", dtype=torch.int32)
    f = gp.vocab_logp(h, w, y, entropy=True)
    assert all(t.numel() == 0 for t in f.values())
    e = torch.empty(0, device="cuda")
    out = gp.vocab_grad(h, w, y, e, e)
    gp.check()
    assert out["d_hidden"].shape == (0, 64) and not out["d_weight"].any()
    keep = torch.ones_like(w)
    gp.vocab_grad(h, w, y, e, e, out={"d_weight": keep}, accumulate=True)
    gp.check()
    assert torch.all(keep == 1)


def test_target_outside_the_vocabulary(gp):
    """Reported, and the next call is not disturbed by it."""
    import torch
    import paper_2606_18954_gb300 as P
    from vocab_ref import head_inputs
    for T in (20, 400):
        h, w, y = head_inputs(T, 300, 64, torch.bfloat16, seed=2)
        good = gp.vocab_logp(h, w, y)
        gp.check()
        bad = y.clone()
        bad[T // 2] = 300
        gp.vocab_logp(h, w, bad)
        with pytest.raises(P.GraphPOError) as e:
            gp.check()
        assert e.value.code == SHAPE
        gl = torch.ones(T, device="cuda")
        gp.vocab_grad(h, w, bad, good["lse"], gl)
        with pytest.raises(P.GraphPOError) as e:
            gp.check()
        assert e.value.code == SHAPE
        again = gp.vocab_logp(h, w, y)
        gp.check()
        assert torch.equal(again["logp"], good["logp"])


def test_two_streams_at_once(gp):
    """Calls of one context on two streams, not ordered with one another: each stream has its own workspace, and
    what a call with `stream` allocates is that stream's."""
    import torch
    from vocab_ref import head_inputs
    cases = [head_inputs(T, V, d, torch.bfloat16, seed=T) for T, V, d in ((700, 9000, 256), (300, 30000, 128))]
    ids = torch.randint(0, 500, (4000,), device="cuda", dtype=torch.int32)
    rows = torch.randn(4000, 64, device="cuda")

    def run(c, stream):
        h, w, y = c
        f = gp.vocab_logp(h, w, y, stream=stream)
        d = gp.vocab_grad(h, w, y, f["lse"], f["logp"], stream=stream)
        x = gp.embed(w, y, stream=stream)
        e = gp.embed_grad(rows, ids, 500, stream=stream)
        return [f["logp"], d["d_hidden"], d["d_weight"], x, e]

    want = [run(c, None) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(20):
        got.append([run(c, s) for c, s in zip(cases, streams)])
    torch.cuda.synchronize()
    for g in got:
        for a, b in zip(g, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_another_stream_and_a_graph(gp):
    import torch
    from vocab_ref import head_inputs
    h, w, y = head_inputs(600, 2000, 128, torch.bfloat16, masked=0.2, seed=8)
    gl, _ = _grads(600, y, 6, False)
    want = gp.vocab_logp(h, w, y)
    wg = gp.vocab_grad(h, w, y, want["lse"], gl)
    gp.check()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = gp.vocab_logp(h, w, y)
        gg = gp.vocab_grad(h, w, y, got["lse"], gl)
    gp.check(s)
    assert all(torch.equal(got[k], want[k]) for k in want) and all(torch.equal(gg[k], wg[k]) for k in wg)
    # captured: the workspace and the outputs are the caller's, inputs change between replays
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    h2, out, og = h.clone(), {k: torch.empty_like(t) for k, t in want.items()}, {k: torch.empty_like(t) for k, t in wg.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gp.vocab_logp(h2, w, y, out=out, workspace=ws)
        gp.vocab_grad(h2, w, y, out["lse"], gl, out=og, workspace=ws)
    for k in range(2):
        h2.copy_(h if k else h.flip(0))
        graph.replay()
    gp.check()
    assert all(torch.equal(out[k], want[k]) for k in want) and all(torch.equal(og[k], wg[k]) for k in wg)


def test_refusals(gp):
    import torch
    import paper_2606_18954_gb300 as P
    B = P.binding
    bf = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    y = torch.zeros(4, device="cuda", dtype=torch.int32)

    def refused(code, *a, **k):
        with pytest.raises(P.GraphPOError) as e:
            gp.vocab_logp(*a, **k)
        assert e.value.code == code, (e.value.code, gp.last_error())

    refused(UNSUPPORTED, torch.zeros(4, 64, device="cuda"), torch.zeros(9, 64, device="cuda"), y)   # fp32 operands
    refused(UNSUPPORTED, bf(4, 65), bf(9, 65), y)                                     # rows off their boundary
    refused(UNSUPPORTED, bf(4, 72)[:, 1:65], bf(9, 64), y)
    refused(INVALID, bf(4, 64), bf(9, 64), y, scale=0.0)
    refused(INVALID, bf(4, 64), bf(9, 64), y, scale=math.nan)
    refused(INVALID, bf(4, 64), bf(9, 64), y, scale=-1.0)
    refused(INVALID, bf(4, 64), bf(0, 64), y)                                         # no vocabulary
    refused(INVALID, bf(1, 64).expand(4, 64), bf(9, 64), y)                            # rows on top of each other
    refused(WORKSPACE, bf(4, 64), bf(9, 64), y, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(TypeError):
        gp.vocab_logp(bf(4, 64), bf(9, 64).half(), y)
    with pytest.raises(TypeError):
        gp.vocab_logp(bf(4, 64), bf(9, 64), y.to(torch.int16))
    with pytest.raises(TypeError):
        gp.vocab_logp(bf(4, 64).to(torch.float64), bf(9, 64).to(torch.float64), y)
    with pytest.raises(ValueError):
        gp.vocab_logp(bf(4, 64), bf(9, 72), y)
    with pytest.raises(ValueError):
        gp.vocab_logp(bf(4, 64), bf(9, 64), y[:3])
    with pytest.raises(ValueError):
        gp.vocab_logp(bf(4, 64), bf(9, 64), y.cpu())
    with pytest.raises(ValueError):
        gp.vocab_logp(bf(64, 4).t(), bf(9, 64), y)
    f = torch.zeros(4, device="cuda")
    with pytest.raises(ValueError):
        gp.vocab_grad(bf(4, 64), bf(9, 64), y, f, f, accumulate=True)
    with pytest.raises(ValueError):
        gp.vocab_grad(bf(4, 64), bf(9, 64), y, f, f, grad_entropy=f)
    with pytest.raises(TypeError):
        gp.vocab_grad(bf(4, 64), bf(9, 64), y, f.double(), f)
    with pytest.raises(P.GraphPOError) as e:
        gp.vocab_grad(bf(4, 64), bf(9, 64), y, f, f, d_hidden=False, d_weight=False)
    assert e.value.code == INVALID
    # at the C entry: NULL arrays and contexts
    L = P.load()
    v = B.CVocab(4, 9, 64, 64, 64, None, None, None, 0, 4, 1.0)
    vo = B.VocabOutputs(None, None, None)
    assert L.gpo_vocab_logp(gp._h, ctypes.byref(v), ctypes.byref(vo), None, 0, None) == INVALID
    assert L.gpo_vocab_logp(None, ctypes.byref(v), ctypes.byref(vo), None, 0, None) == INVALID
    assert L.gpo_vocab_grad(gp._h, None, None, None, None, 0, None) == INVALID
    torch.cuda.synchronize()


def test_refusals_of_misaligned_and_huge_arrays(gp):
    """At the C entry: pointers that are no multiple of their elements, gradient strides past any memory."""
    import torch
    import paper_2606_18954_gb300 as P
    from paper_2606_18954_gb300 import binding as B
    L = P.load()
    T, V, d = 100, 300, 64
    h = torch.zeros(T, d, device="cuda", dtype=torch.bfloat16)
    w = torch.zeros(V, d, device="cuda", dtype=torch.bfloat16)
    y = torch.zeros(T, device="cuda", dtype=torch.int32)
    f = torch.zeros(T + 1, device="cuda")
    v = B.CVocab(T, V, d, d, d, h.data_ptr(), w.data_ptr(), y.data_ptr(), 0, 4, 1.0)
    room = torch.empty(max(B.vocab_workspace_size(v), B.vocab_workspace_size(v, True)), dtype=torch.uint8, device="cuda")

    def forward(**k):
        o = {"logp": f.data_ptr(), **k}
        vo = B.VocabOutputs(*(o.get(n) for n in ("logp", "lse", "entropy")))
        return L.gpo_vocab_logp(gp._h, ctypes.byref(v), ctypes.byref(vo), room.data_ptr(), room.numel(), None)

    def gradient(ins=(), **k):
        i = {"lse": f.data_ptr(), "grad_logp": f.data_ptr(), **dict(ins)}
        gi = B.VocabGradInputs(*(i.get(n) for n in ("lse", "grad_logp", "entropy", "grad_entropy")))
        g = {"d_hidden": h.data_ptr(), "d_weight": w.data_ptr(), "d_hidden_stride": d, "d_weight_stride": d, **k}
        vg = B.VocabGrads(g["d_hidden"], g["d_weight"], g["d_hidden_stride"], g["d_weight_stride"], 0)
        return L.gpo_vocab_grad(gp._h, ctypes.byref(v), ctypes.byref(gi), ctypes.byref(vg), room.data_ptr(), room.numel(), None)

    for name in ("logp", "lse", "entropy"):
        assert forward(**{name: f.data_ptr() + 2}) == UNSUPPORTED, name
    for name in ("lse", "grad_logp", "entropy", "grad_entropy"):
        both = {"entropy": f.data_ptr(), "grad_entropy": f.data_ptr(), name: f.data_ptr() + 2}
        assert gradient(both) == UNSUPPORTED, name
    for name in ("d_hidden", "d_weight"):
        assert gradient(**{name: h.data_ptr() + 1}) == UNSUPPORTED, name
        assert gradient(**{name + "_stride": 1 << 40}) == UNSUPPORTED, name
        assert gradient(**{name + "_stride": d - 1}) == INVALID, name
    torch.cuda.synchronize()


def test_forced_timeout_then_a_normal_call(gp):
    """The bounded waits' failure path (GPO_FLAG_DEBUG_TIMEOUT): the status, then a correct call."""
    import torch
    import paper_2606_18954_gb300 as P
    from vocab_ref import close, head_exact, head_inputs
    h, w, y = head_inputs(600, 3000, 512, torch.bfloat16, seed=9)
    gl, _ = _grads(600, y, 7, False)
    forced = P.GraphPO(flags=P.binding.FLAG_DEBUG_TIMEOUT)
    lse = gp.vocab_logp(h, w, y)["lse"]
    for _ in range(2):
        forced.vocab_logp(h, w, y)
        with pytest.raises(P.GraphPOError) as e:
            forced.check()
        assert e.value.code == TIMEOUT
        forced.vocab_grad(h, w, y, lse, gl)
        with pytest.raises(P.GraphPOError) as e:
            forced.check()
        assert e.value.code == TIMEOUT
    out = gp.vocab_logp(h, w, y, entropy=True)
    gp.check()
    ref = head_exact(h, w, y, 1.0)
    for k in out:
        close(out[k], ref[k], ref["t_" + k], k)
