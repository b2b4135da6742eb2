"""Adjusted logits and their gradient on the GPU against the formulas in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as pkg
    pkg.build()
    return pkg


@pytest.fixture(scope="module")
def gp(P):
    return P.GraphPO()


def _types():
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# rows, vocabulary, type, arguments: one entry, slices that end inside a vector, a word, a row; clusters of every size; more
# rows than CTAs; rows on every 16-byte offset; everything at once
CASES = [
    (1, 1, "f32", {}), (3, 7, "bf16", dict(history=4)), (2, 31, "f16", dict(masks=1)), (5, 33, "f32", dict(masks=3, pad=1)),
    (1, 6144, "f32", dict(masks=2)), (1, 6145, "f32", dict(biases=9)), (2, 12288, "bf16", dict(pad=3, biases=5)),
    (1, 12289, "f16", dict(masks=2, temperature=True)), (3, 24577, "bf16", dict(masks=1, pad=2)), (4, 40000, "bf16", dict(pad=5, masks=3, biases=50, temperature=True)),
    (1, 131072, "bf16", dict(history=3000, masks=2, biases=300)), (1, 131073, "f32", dict(history=3000)),
    (33, 50021, "f16", dict(pad=1, history=900, biases=70, temperature=True)), (77, 20011, "f32", dict(pad=2, masks=4, history=300)),
    (9, 140007, "f16", dict(pad=7, masks=3, history=2000, biases=30)), (400, 1001, "bf16", dict(masks=5, pad=1, temperature=True)),
    (700, 5003, "f16", dict(masks=3, masked=0.4, biases=20)), (320, 9001, "f32", dict(masked=0.5, masks=2)),
    (6, 3001, "bf16", dict(penalties=False, biases=40)), (6, 3001, "bf16", dict(penalties=False, history=0, masks=2)),
    (6, 3001, "bf16", dict(history=0, penalties=False)), (2, 131072, "f32", dict(history=20000, biases=9000, masks=2)),
    (1, 270001, "bf16", dict(history=9000, pad=1)), (3, 263001, "f32", dict(history=300, pad=3, masks=2)), (2, 300007, "f16", dict(penalties=False, history=0)),
    (4, 5, "f16", dict(pad=9, history=9)), (3, 17, "f32", dict(pad=5, biases=4, masks=2)), (64, 16390, "bf16", dict(pad=2)), (5, 2000, "f16", dict(biases=2000, history=5000)),
]


@pytest.mark.parametrize("ids", ["int32", "int64"])
@pytest.mark.parametrize("R, V, dtype, kw", CASES, ids=lambda x: str(x).replace(" ", ""))
def test_both_directions(gp, R, V, dtype, kw, ids):
    import torch
    from logits_ref import exact, inputs, near
    from vocab_ref import EPS, TINY
    dt = _types()[dtype]
    kw = dict(kw)
    z, y, how = inputs(R, V, dt, seed=V + R, ids=getattr(torch, ids), **kw)
    raw = z.clone()
    g = torch.randn(R, device="cuda")
    e = torch.randn(R, device="cuda") * 0.1
    if R > 4:
        g[::5] = 0.0
        e[::10] = 0.0
    for entropy in (False, True):
        ref = exact(z, y, how, g, e if entropy else None)
        f = gp.logits_adjust(z, y, entropy=entropy, **how)
        gp.check()
        assert set(f) == {"logp", "lse", "entropy"} - (set() if entropy else {"entropy"})
        for k in f:
            near(f[k], ref[k], ref["t_" + k], k)
        d = gp.logits_grad(z, y, f["lse"], f["logp"], g, entropy=f.get("entropy"), grad_entropy=e if entropy else None, **how)
        gp.check()
        want = torch.where(torch.isfinite(ref["d_logits"]), ref["d_logits"], 0.0)
        near(d["d_logits"], want, ref["t_d_logits"], "d_logits")
        # a sampler's call: no target, every row
        every = exact(z, None, how)
        for write in {dt, torch.float32}:
            s = gp.logits_adjust(z, write=write, entropy=entropy, **how)
            gp.check()
            # (an fp16 result below 2^-14 is a multiple of 2^-24: its rounding is off by up to 2^-25)
            t = every["t_logits"] + EPS[write] * torch.where(torch.isfinite(every["logits"]), every["logits"].abs(), 0.0) + TINY[write]
            near(s["logits"], every["logits"].to(write).double().where(torch.isinf(every["logits"].to(write)), every["logits"]), t, "logits")
            for k in ("lse", "entropy") if entropy else ("lse",):
                near(s[k], every[k], every["t_" + k], k)
    assert torch.equal(torch.nan_to_num(raw.float(), 7.0), torch.nan_to_num(z.float(), 7.0))


@pytest.mark.parametrize("R, V, pad", [(1, 30011, 0), (50, 7001, 1), (400, 900, 0)])
def test_in_place_and_other_strides(gp, R, V, pad):
    import torch
    from logits_ref import inputs
    for dt in (torch.bfloat16, torch.float32):
        z, y, how = inputs(R, V, dt, seed=5, pad=pad, masks=3, biases=10, temperature=True)
        f = gp.logits_adjust(z, write=dt, **how)
        for extra in (0, 1, 2, 8):
            wide = torch.full((R + 1, V + extra + 8), 3.5, dtype=dt, device="cuda")
            to = wide[:R, extra:extra + V]
            gp.logits_adjust(z, out={"logits": to}, **how)
            gp.check()
            assert torch.equal(torch.nan_to_num(to.float(), 7.0), torch.nan_to_num(f["logits"].float(), 7.0))
            assert bool((wide[:R, :extra] == 3.5).all()) and bool((wide[:R, extra + V:] == 3.5).all()) and bool((wide[R] == 3.5).all())
        t = gp.logits_adjust(z, y, **how)
        g = torch.randn(R, device="cuda")
        d = gp.logits_grad(z, y, t["lse"], t["logp"], g, **how)["d_logits"]
        own = torch.empty_strided(z.shape, z.stride(), dtype=dt, device="cuda")
        own.copy_(z)
        gp.logits_grad(own, y, t["lse"], t["logp"], g, out={"d_logits": own}, **how)
        gp.check()
        assert torch.equal(own, d)
        own.copy_(z)
        got = gp.logits_adjust(own, out={"logits": own, "lse": torch.empty(R, device="cuda")}, **how)
        gp.check()
        assert torch.equal(torch.nan_to_num(own.float(), 7.0), torch.nan_to_num(f["logits"].float(), 7.0))
        assert torch.equal(got["lse"], f["lse"])


def test_gradient_against_differences(gp):
    """Central differences of logp and entropy in 64 bits, of the plain formulas; the kernel's gradient of fp32 logits."""
    import torch
    from logits_ref import exact, inputs
    R, V = 4, 40
    z, y, how = inputs(R, V, torch.float32, seed=3, history=30, masks=2, biases=6, temperature=True)
    how["mask_row"][:] = torch.tensor([-1, 0, 0, -1], device="cuda")
    y = torch.tensor([3, 0, 12, 7], device="cuda", dtype=torch.int32)  # (words 0, 3, .. of every mask allow all)
    g, e = torch.randn(R, device="cuda"), torch.randn(R, device="cuda")
    z = torch.where(torch.isfinite(z) & (z.abs() < 1e30), z, 0.0)
    z = torch.where(z.abs() < 0.01, 0.5, z)  # (away from where the repetition's slope changes)
    f = gp.logits_adjust(z, y, entropy=True, **how)
    d = gp.logits_grad(z, y, f["lse"], f["logp"], g, entropy=f["entropy"], grad_entropy=e, **how)["d_logits"].double()
    gp.check()

    def loss(x):
        r = exact(x, y, how)
        return r["logp"] * g.double() + r["entropy"] * e.double()
    step = 1e-5
    for v in range(V):
        a, b = z.double().clone(), z.double().clone()
        a[:, v] += step
        b[:, v] -= step
        slope = (loss(a.requires_grad_(False)) - loss(b)) / (2 * step)
        # differences: third derivatives, below 10 (g + e) (s rho)^3, and 64-bit roundings of sums of about 20; the kernel: test_both_directions
        tol = 10 * (g.abs() + e.abs()).double() * 8 * step ** 2 + 20 * 2.0 ** -52 / step * 8 + 1e-4 * (g.abs() + e.abs()).double()
        assert bool(((d[:, v] - slope).abs() <= tol).all()), (v, d[:, v], slope)


def test_rows_of_the_lowest_value_and_infinities(gp):
    import torch
    for dt in (torch.bfloat16, torch.float32):
        low = torch.finfo(dt).min
        z = torch.full((6, 1000), low, dtype=dt, device="cuda")
        z[1, 5] = 2.0
        z[2] = -math.inf
        z[3, 7], z[3, 8] = 1.0, -math.inf
        z[4] = 1.0
        z[4, 3] = math.nan
        z[5] = 1.0
        z[5, 3] = math.inf
        y = torch.tensor([0, 5, 3, 7, 9, 9], device="cuda")
        f = gp.logits_adjust(z, y, entropy=True)
        d = gp.logits_grad(z, y, f["lse"], f["logp"], torch.ones(6, device="cuda"), entropy=f["entropy"],
                           grad_entropy=torch.ones(6, device="cuda"))["d_logits"]
        s = gp.logits_adjust(z, write=torch.float32, entropy=True)
        gp.check()
        for i in (0, 2):  # nothing is left
            assert f["lse"][i] == -math.inf and f["logp"][i] == -math.inf and f["entropy"][i] == 0 and bool((d[i] == 0).all())
            assert s["lse"][i] == -math.inf and s["entropy"][i] == 0
        for i, v in ((1, 2.0), (3, 1.0)):  # one token is
            # (lse goes through units of log 2: two roundings)
            assert abs(f["lse"][i] - v) <= 4e-7 and f["logp"][i] == 0 and f["entropy"][i] == 0 and bool((d[i] == 0).all())
            assert abs(s["lse"][i] - v) <= 4e-7 and s["entropy"][i] == 0
        for i in (4, 5):
            assert math.isnan(f["lse"][i]) and math.isnan(f["logp"][i]) and bool(torch.isnan(d[i].float()).all())
        assert torch.equal(torch.nan_to_num(s["logits"], 7.0), torch.nan_to_num(z.float(), 7.0))


def test_shared_lists_without_spans_or_rows(gp):
    """One list of biases and one mask for all rows; histories of rows that share their tokens."""
    import torch
    from logits_ref import exact, inputs, near
    R, V = 12, 2500
    z, y, how = inputs(R, V, torch.bfloat16, seed=11, history=0, penalties=False)
    seq = torch.randint(0, 60, (40,), device="cuda")
    how.update(history=seq, spans=torch.tensor([[0, 10, 10 + 2 * i] for i in range(R)], device="cuda"), repetition=1.2, presence=0.3,
               frequency=0.1, bias_ids=torch.tensor([0, 7, 31, 32, 2499], device="cuda", dtype=torch.int32),
               bias=torch.tensor([1.0, -2.0, 3.0, 0.5, -math.inf], device="cuda"),
               mask=torch.randint(-2 ** 31, 2 ** 31 - 1, (1, 100), device="cuda").to(torch.int32))
    y[:] = -1
    s = gp.logits_adjust(z, write=torch.float32, entropy=True, **how)
    gp.check()
    plain = dict(how, bias=torch.where(torch.isinf(how["bias"]), -1e300, how["bias"].double()))
    ref = exact(z, None, plain)
    want = torch.where(ref["logits"] < -1e200, -math.inf, ref["logits"])
    near(s["logits"], want, ref["t_logits"].clamp(max=1e-3) + 2.0 ** -24 * torch.where(torch.isfinite(want), want.abs(), 0.0), "logits")
    near(s["lse"], ref["lse"], ref["t_lse"], "lse")
    near(s["entropy"], ref["entropy"], ref["t_entropy"], "entropy")


def test_nothing_to_do(gp):
    import torch
    z = torch.zeros(0, 50, device="cuda")
    f = gp.logits_adjust(z, torch.zeros(0, dtype=torch.int32, device="cuda"), write=torch.float32)
    assert f["logits"].shape == (0, 50)
    assert gp.logits_grad(z, torch.zeros(0, dtype=torch.int32, device="cuda"), f["lse"], f["logp"], f["lse"])["d_logits"].shape == (0, 50)
    gp.check()
    # an empty history, no biases, no token in a history
    z = torch.randn(3, 50, device="cuda")
    a = gp.logits_adjust(z, write=torch.float32)
    b = gp.logits_adjust(z, write=torch.float32, history=torch.full((4,), -1, device="cuda"), repetition=2.0,
                         spans=torch.tensor([[0, 0, 0], [4, 4, 4], [0, 2, 4]], device="cuda"), bias=torch.zeros(0, device="cuda"),
                         bias_ids=torch.zeros(0, dtype=torch.int32, device="cuda"))
    gp.check()
    assert torch.equal(a["logits"], z) and torch.equal(b["logits"], z) and torch.equal(a["lse"], b["lse"])


def test_the_same_on_every_run_and_stream(gp):
    import torch
    from logits_ref import inputs
    for R, V in ((2, 60000), (500, 3000)):
        z, y, how = inputs(R, V, torch.bfloat16, seed=2, masks=2, history=2000, biases=40)
        one = gp.logits_adjust(z, y, entropy=True, **how)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        two = gp.logits_adjust(z, y, entropy=True, stream=s, **how)
        g = torch.randn(R, device="cuda")
        s.wait_stream(torch.cuda.current_stream())
        d2 = gp.logits_grad(z, y, two["lse"], two["logp"], g, stream=s, **how)["d_logits"]
        d1 = gp.logits_grad(z, y, one["lse"], one["logp"], g, **how)["d_logits"]
        torch.cuda.synchronize()
        gp.check()
        assert all(torch.equal(one[k], two[k]) for k in one) and torch.equal(d1, d2)


def test_replays(gp):
    """A captured call, replayed on changed inputs, with another call between."""
    import torch
    from logits_ref import inputs
    z, y, how = inputs(20, 5000, torch.bfloat16, seed=4, masks=2, biases=5)
    g = torch.randn(20, device="cuda")

    def step():
        f = gp.logits_adjust(z, y, **how)
        return f["logp"], f["lse"], gp.logits_grad(z, y, f["lse"], f["logp"], g, **how)["d_logits"]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(3):
        z.copy_(inputs(20, 5000, torch.bfloat16, seed=40 + i, masks=2, biases=5)[0].nan_to_num(0.5, 1.0, 1.0))
        graph.replay()
        torch.cuda.synchronize()
        have = [t.clone() for t in got]
        want = step()
        gp.check()
        bits = lambda x: x.view(torch.int16 if x.dtype is torch.bfloat16 else torch.int32)  # noqa: E731  (a NaN equals itself)
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(have, want))


SHAPE, ARG = 2, 1


def test_what_the_kernel_refuses(P, gp):
    import torch
    V = 100
    z = torch.zeros(3, V, device="cuda")
    t = lambda *v, dt=torch.int64: torch.tensor(v, device="cuda", dtype=dt)  # noqa: E731
    seq = t(1, 2, 3, 4)
    ok = dict(history=seq, spans=t([0, 1, 2], [0, 0, 0], [1, 2, 4]), repetition=1.5)
    bad = [
        (dict(ok, spans=t([0, 1, 2], [0, 0, 5], [1, 2, 4])), SHAPE), (dict(ok, spans=t([0, 1, 2], [-1, 0, 1], [1, 2, 4])), SHAPE),
        (dict(ok, spans=t([0, 3, 2], [0, 0, 1], [1, 2, 4])), SHAPE), (dict(ok, history=t(1, V, 3, 4)), SHAPE),
        (dict(ok, history=t(1, 2 ** 40, 3, 4)), SHAPE), (dict(ok, repetition=t(1.0, 0.0, 2.0, dt=torch.float32)), ARG),
        (dict(ok, repetition=t(1.0, math.nan, 2.0, dt=torch.float32)), ARG), (dict(ok, presence=t(1.0, math.inf, 2.0, dt=torch.float32)), ARG),
        (dict(scale=t(1.0, 1.0, 0.0, dt=torch.float32)), ARG), (dict(scale=t(1.0, 1.0, 2e4, dt=torch.float32)), ARG),
        (dict(target=t(1, V, 2)), SHAPE), (dict(bias=torch.zeros(3, device="cuda"), bias_ids=t(1, 1, 2)), SHAPE),
        (dict(bias=torch.zeros(3, device="cuda"), bias_ids=t(5, 1, 2)), SHAPE), (dict(bias=torch.zeros(3, device="cuda"), bias_ids=t(1, 2, V)), SHAPE),
        (dict(bias=torch.zeros(3, device="cuda"), bias_ids=t(-1, 1, 2)), SHAPE),
        (dict(bias=torch.zeros(3, device="cuda"), bias_ids=t(0, 1, 2), bias_spans=t([0, 3], [0, 4], [0, 0])), SHAPE),
        (dict(bias=torch.zeros(3, device="cuda"), bias_ids=t(0, 1, 2), bias_spans=t([0, 3], [2, 1], [0, 0])), SHAPE),
        (dict(mask=torch.ones(2, 4, dtype=torch.int32, device="cuda"), mask_row=t(0, 2, -1, dt=torch.int32)), SHAPE),
    ]
    want = gp.logits_adjust(z, write=torch.float32, **ok)
    gp.check()
    for kw, code in bad:
        gp.logits_adjust(z, write=torch.float32, **kw)
        again = gp.logits_adjust(z, write=torch.float32, **ok)
        with pytest.raises(P.GraphPOError) as e:
            gp.check()
        assert e.value.code == code, (kw, e.value)
        gp.check()
        assert torch.equal(again["logits"], want["logits"])
    host = [dict(scale=0.0), dict(scale=math.nan), dict(repetition=0.0), dict(repetition=-1.0), dict(presence=math.inf), dict(frequency=math.nan)]
    for kw in host:
        with pytest.raises(P.GraphPOError) as e:
            gp.logits_adjust(z, **kw)
        assert e.value.code == ARG
    with pytest.raises(P.GraphPOError):  # rows that overlap the raw ones
        buf = torch.zeros(4 * V, device="cuda")
        gp.logits_adjust(buf[:2 * V].view(2, V), out={"logits": buf[V:3 * V].view(2, V)})
    buf = torch.randn(3, 2 * V, device="cuda")  # (side by side they do not)
    assert torch.equal(gp.logits_adjust(buf[:, :V], out={"logits": buf[:, V:]}, scale=2.0)["logits"], 2 * buf[:, :V])
    for a, b in ((0, V - 1), (V - 1, 0), (1, V), (V, 1)):
        with pytest.raises(P.GraphPOError):
            gp.logits_adjust(buf[:, a:a + V], out={"logits": buf[:, b:b + V]})
    with pytest.raises(P.GraphPOError):  # no output
        gp.logits_adjust(z, lse=False)
    gp.check()


def test_replays_keep_their_errors_until_check(P, gp):
    """Of a captured call the replays' errors are raised once each, and disturb no other replay."""
    import torch
    z, ids = torch.randn(3, 100, device="cuda"), torch.tensor([1, 2, 3, 4], device="cuda")
    how = dict(history=ids, spans=torch.tensor([[0, 0, 2], [1, 2, 4], [2, 2, 4]], device="cuda"), repetition=1.5, frequency=0.5)
    step = lambda: gp.logits_adjust(z, write=torch.float32, **how)["logits"]  # noqa: E731
    want = step().clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        ids[1] = 100
        graph.replay()
        ids[1] = 2
        graph.replay()
        with pytest.raises(P.GraphPOError) as e:
            gp.check()
        assert e.value.code == SHAPE
        gp.check()
        assert torch.equal(got, want)


def test_limits(P, gp):
    """What the library refuses by its sizes alone, before it looks at any memory."""
    import ctypes
    import torch
    from paper_2606_18954_gb300 import binding as B
    L, out = B.load(), torch.zeros(1, device="cuda")
    for R, V, code in ((1, 2 ** 30 + 1, 5), (2 ** 31, 1, 5), (2 ** 12, 2 ** 29, 5), (1, 0, 1), (-1, 5, 1)):
        args = B.CLogits(R, V, V, out.data_ptr(), 1, 4, 4, 4, *([None] * 4), 1.0, 1.0, 0.0, 0.0)
        outs = B.LogitsOutputs(None, V, 1, None, out.data_ptr(), None)
        assert L.gpo_logits_adjust(gp._h, ctypes.byref(args), ctypes.byref(outs), None) == code, (R, V)


def test_offsets_past_32_bits(gp):
    """More than 2^31 entries: the last rows are what a call on them alone gives (of 400 rows, too, each is one CTA's)."""
    import torch
    R, V, n = 33000, 65600, 400
    assert R * V > 2 ** 31
    z = torch.empty(R, V, device="cuda", dtype=torch.float16).normal_()
    y = torch.randint(0, V, (R,), device="cuda")
    g, s = torch.randn(R, device="cuda"), torch.rand(R, device="cuda") + 0.5
    ids = torch.randint(0, V, (3000,), device="cuda")
    spans = torch.tensor([[0, 1000, 3000]], device="cuda").repeat(R, 1)
    mask = torch.randint(-2 ** 31, 2 ** 31, (R, (V + 31) // 32), device="cuda").to(torch.int32)
    how = lambda a: dict(scale=s[a:], history=ids, spans=spans[a:], repetition=1.2, presence=0.1, frequency=0.05, mask=mask[a:])  # noqa: E731
    tail = z[-n:].clone()
    f = gp.logits_adjust(z, y, write=torch.float16, **how(0))
    e = gp.logits_adjust(tail, y[-n:], write=torch.float16, **how(R - n))
    d = gp.logits_grad(z, y, f["lse"], f["logp"], g, out={"d_logits": z}, **how(0))["d_logits"]
    c = gp.logits_grad(tail, y[-n:], e["lse"], e["logp"], g[-n:], **how(R - n))["d_logits"]
    gp.check()
    for k in f:
        assert torch.equal(f[k][-n:], e[k]), k
    assert torch.equal(d[-n:], c)
