"""Distillation from a teacher's top tokens on the GPU against the formulas in 64 bits."""
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


# tokens, vocabulary, width, entries, type, arguments: one token; one entry; all of the vocabulary; entries of neighbouring
# tokens that share tiles; widths of several accumulations; several row tiles; more tokens than one CTA lists at a time; two
# pieces of the vocabulary; listed tokens
CASES = [
    (1, 1000, 64, 1, "bf16", {}), (1, 70, 72, 70, "f16", dict(tail=True)), (5, 40, 72, 40, "bf16", {}), (17, 300, 64, 8, "f16", dict(short=True, pad=8)),
    (16, 9001, 256, 3, "bf16", dict(tail=True, teacher="bf16")), (60, 8191, 512, 8, "f16", dict(teacher="f16", ids="int64")),
    (257, 1025, 328, 300, "bf16", dict(tail=True, short=True)), (300, 3000, 264, 33, "f16", dict(masked=0.3, teacher_scale=0.5)),
    (700, 5003, 1000, 64, "bf16", dict(masked=0.3, short=True, tail=True, pad=8)), (100, 600, 136, 512, "f16", dict(tail=True)),
    (300, 700, 2104, 20, "bf16", dict(scale=0.7)), (300, 700, 2104, 20, "f16", dict(short=True, tail=True, pad=16)),
    (4500, 700, 64, 16, "bf16", dict(masked=0.5, ids="int64")), (4300, 66000, 40, 5, "f16", dict(masked=0.2, tail=True)),
    (256, 131072, 4096, 32, "bf16", dict(masked=0.4, tail=True)), (3, 131072, 128, 64, "bf16", dict(short=True)),
]


@pytest.mark.parametrize("T, V, d, k, dtype, kw", CASES, ids=lambda x: str(x).replace(" ", ""))
def test_both_directions(gp, T, V, d, k, dtype, kw):
    import torch
    from distill_ref import exact, inputs, near
    kw = dict(kw)
    scale, ts, tail = kw.pop("scale", 1.0), kw.get("teacher_scale", 1.0), kw.get("tail", False)
    kw["teacher"], kw["ids"] = _types()[kw.get("teacher", "f32")], getattr(torch, kw.get("ids", "int32"))
    dt = _types()[dtype]
    h, w, ids, t = inputs(T, V, d, k, dt, seed=T + V, **kw)
    to = 1024.0 if dtype == "f16" else 1.0
    g = torch.randn(T, device="cuda") * to / T
    if T > 4:
        g[::5] = 0.0
    ref = exact(h, w, ids, t, scale, ts, tail, g)
    f = gp.vocab_distill(h, w, ids, t, scale=scale, teacher_scale=ts, tail=tail, lse=True)
    gp.check()
    for name in ("lse", "rest_lse", "rest", "delta", "loss"):
        near(f[name], ref[name], ref["t_" + name], name)
    r = gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g, scale=scale)
    gp.check()
    for name in ("d_hidden", "d_weight"):
        near(r[name], ref[name], ref["t_" + name], name)
    # one of them alone, added to what is there, rows of any alignment; the same bits
    out = {"d_hidden": torch.empty(T, d + 1, dtype=dt, device="cuda")[:, 1:]}
    assert torch.equal(gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g, scale=scale, out=out)["d_hidden"], r["d_hidden"])
    base = torch.randn(V, d, device="cuda").to(dt) * 1e-3 * to
    out = {"d_weight": base.clone()}
    gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g, scale=scale, accumulate=True, out=out)
    gp.check()
    want = ref["d_weight"] + base.double()
    near(out["d_weight"], want, ref["t_d_weight"] + 2.0 ** (-8 if dtype == "bf16" else -11) * want.abs(), "d_weight added")


def test_certain_students(gp):
    """A student that is nearly certain of a teacher's token, which is, too: p - q of it, the others' share and the gradient keep
    their digits."""
    import torch
    from distill_ref import exact, inputs, near
    for dt in (torch.bfloat16, torch.float16):
        for tail in (False, True):
            h, w, ids, t = inputs(200, 2000, 256, 16, dt, sure=40.0, seed=9, tail=tail, spread=0.5)
            g = torch.full((200,), 1.0, device="cuda")
            ref = exact(h, w, ids, t, tail=tail, g=g)
            sure = ref["delta"].abs().amax(1) < 1e-3
            assert int(sure.sum()) >= 10  # (some rows are)
            f = gp.vocab_distill(h, w, ids, t, tail=tail)
            gp.check()
            for name in ("rest_lse", "rest", "delta", "loss"):
                near(f[name], ref[name], ref["t_" + name], name)
            if not tail:  # (with tail 1 - q comes from the teacher's log-probability of 32 bits)
                err = (f["delta"].double() - ref["delta"]).norm(dim=1)[sure]
                # 1 - p and 1 - q move by twice the logits' and half the teacher's error, relative to themselves
                size = ((f["delta"].double().abs().sum(1)) + 2 * (ref["rest"].abs()))[sure]
                assert bool((err <= 1e-3 * size + 1e-9).all()), float((err / size).max())
            r = gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g)
            gp.check()
            for name in ("d_hidden", "d_weight"):
                near(r[name], ref[name], ref["t_" + name], name)


def test_gradient_against_differences(gp):
    """Central differences of the loss in 64 bits, of the plain formulas, in some directions."""
    import torch
    from distill_ref import exact, inputs
    T, V, d, k = 6, 50, 16, 5
    for tail in (False, True):
        h, w, ids, t = inputs(T, V, d, k, torch.float16, seed=3, short=True, tail=tail, sure=3.0)
        g = torch.rand(T, device="cuda") + 0.5
        f = gp.vocab_distill(h, w, ids, t, scale=1.25, tail=tail)
        r = gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g, scale=1.25)
        gp.check()
        ref = exact(h, w, ids, t, 1.25, 1.0, tail, g)

        def loss(hh, ww):
            from distill_ref import EPS, TINY
            EPS.setdefault(torch.float64, 0.0)
            TINY.setdefault(torch.float64, 0.0)
            return float((exact(hh, ww, ids, t, 1.25, 1.0, tail)["loss"] * g.double()).sum())
        gen = torch.Generator(device="cuda")
        gen.manual_seed(1)
        for _ in range(4):
            dh, dw = (torch.randn(x.shape, generator=gen, device="cuda", dtype=torch.float64) for x in (h, w))
            step = 1e-5
            slope = (loss(h.double() + step * dh, w.double() + step * dw) - loss(h.double() - step * dh, w.double() - step * dw)) / (2 * step)
            got = float((r["d_hidden"].double() * dh).sum() + (r["d_weight"].double() * dw).sum())
            tol = float((ref["t_d_hidden"] * dh.abs()).sum() + (ref["t_d_weight"] * dw.abs()).sum())
            # (differences: third derivatives of logits that move by about 20 a step, and roundings of the loss)
            assert abs(got - slope) <= tol + 1e3 * 20 ** 3 * step ** 2 + 1e-8, (got, slope, tol)


def test_strides_and_outputs(gp):
    import torch
    from distill_ref import inputs
    T, V, d, k = 40, 900, 64, 7
    h, w, ids, t = inputs(T, V, d, k, torch.bfloat16, seed=1, masked=0.2)
    f = gp.vocab_distill(h, w, ids, t, lse=True)
    wide = lambda x: torch.full((T, k + 5), 7, dtype=x.dtype, device="cuda")  # noqa: E731
    i2, t2, d2 = wide(ids), wide(t), wide(f["delta"])
    i2[:, 2:2 + k], t2[:, 3:3 + k] = ids, t
    out = {"loss": torch.empty(T, device="cuda"), "rest": torch.empty(T, device="cuda"), "rest_lse": torch.empty(T, device="cuda"), "delta": d2[:, 1:1 + k]}
    gp.vocab_distill(h, w, i2[:, 2:2 + k], t2[:, 3:3 + k], out=out)
    gp.check()
    for name in out:
        assert torch.equal(out[name], f[name]), name
    assert bool((d2[:, :1] == 7).all()) and bool((d2[:, 1 + k:] == 7).all())
    g = torch.rand(T, device="cuda")
    a = gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g)
    b = gp.vocab_distill_grad(h, w, i2[:, 2:2 + k], out["delta"], out["rest"], out["rest_lse"], g)
    gp.check()
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_nothing_to_learn(gp):
    """No tokens; no entries; teachers of -inf alone; gradients of 0."""
    import torch
    w = torch.randn(50, 64, device="cuda").bfloat16()
    e = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    h = e(0, 64, dt=torch.bfloat16)
    f = gp.vocab_distill(h, w, e(0, 4, dt=torch.int32), e(0, 4))
    r = gp.vocab_distill_grad(h, w, e(0, 4, dt=torch.int32), f["delta"], f["rest"], f["rest_lse"], f["loss"])
    gp.check()
    assert r["d_hidden"].shape == (0, 64) and not r["d_weight"].any()
    h = torch.full((20, 64), math.nan, device="cuda").bfloat16()
    for ids, t in ((torch.full((20, 4), -1, device="cuda"), e(20, 4)), (torch.arange(4, device="cuda").repeat(20, 1), e(20, 4) - math.inf)):
        f = gp.vocab_distill(h, w, ids, t, lse=True)
        gp.check()
        assert not any(f[k].any() for k in f)
        r = gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], e(20))
        gp.check()
        assert not r["d_hidden"].any() and not r["d_weight"].any()


def test_together_with_the_sampled_tokens(gp):
    """A policy's step on its rollouts: sampled from adjusted logits, their log-probabilities, a teacher on the same tokens; the two
    gradients of the matrix are added."""
    import torch
    from distill_ref import exact, near, rows
    from vocab_ref import head_exact
    torch.manual_seed(0)
    T, V, d, k = 120, 3000, 128, 12
    h, w = rows(torch.randn(T, d, device="cuda"), torch.bfloat16, 0), rows(torch.randn(V, d, device="cuda") / 6, torch.bfloat16, 0)
    z = h.float() @ w.float().t()
    seq = torch.randint(0, V, (T,), device="cuda")
    spans = torch.stack([torch.zeros(T, dtype=torch.int64, device="cuda"), torch.full((T,), 10, device="cuda"),
                         torch.arange(T, device="cuda").clamp(min=10)], 1)
    s = gp.logits_adjust(z, write=torch.float32, history=seq, spans=spans, repetition=1.1, frequency=0.05, scale=1.25)
    y = (s["logits"] + -torch.log(-torch.log(torch.rand(T, V, device="cuda").clamp(1e-9, 1 - 1e-7)))).argmax(1)
    f = gp.logits_adjust(z, y, history=seq, spans=spans, repetition=1.1, frequency=0.05, scale=1.25)
    assert bool(((s["logits"].gather(1, y[:, None])[:, 0] - s["lse"] - f["logp"]).abs() < 1e-4).all())
    t, ids = torch.log_softmax(h.float() @ (w.float() + 0.05 * torch.randn(V, d, device="cuda")).t(), 1).topk(k, dim=1)
    head = gp.vocab_logp(h, w, y, entropy=True)
    taught = gp.vocab_distill(h, w, ids, t, tail=True)
    g1, g2 = torch.randn(T, device="cuda") / T, torch.full((T,), 0.5 / T, device="cuda")
    a = gp.vocab_grad(h, w, y, head["lse"], g1, logp=head["logp"])
    b = gp.vocab_distill_grad(h, w, ids, taught["delta"], taught["rest"], taught["rest_lse"], g2, out=dict(a, d_hidden=torch.empty_like(h)),
                              accumulate=True)
    gp.check()
    r1, r2 = head_exact(h, w, y, 1.0, g1), exact(h, w, ids, t, tail=True, g=g2)
    near(taught["loss"], r2["loss"], r2["t_loss"], "loss")
    near(b["d_hidden"], r2["d_hidden"], r2["t_d_hidden"], "d_hidden")
    want = r1["d_weight"] + r2["d_weight"]
    near(a["d_weight"], want, r1["t_d_weight"] + r2["t_d_weight"] + 2.0 ** -8 * (want.abs() + r1["d_weight"].abs()), "d_weight")


def test_streams_and_replays(gp):
    import torch
    from distill_ref import inputs
    h, w, ids, t = inputs(300, 900, 128, 9, torch.bfloat16, seed=5, masked=0.1)
    g = torch.rand(300, device="cuda")

    def step(stream=None):
        f = gp.vocab_distill(h, w, ids, t, stream=stream)
        r = gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g, stream=stream)
        return [f["loss"], f["delta"], f["rest"], f["rest_lse"], r["d_hidden"], r["d_weight"]]
    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = step(s)
    torch.cuda.synchronize()
    gp.check()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    big = inputs(3000, 5000, 256, 30, torch.bfloat16, seed=6)
    gp.vocab_distill(*big)  # (a larger workspace in between)
    for i in range(3):
        for x, y in zip((h, w, ids, t), inputs(300, 900, 128, 9, torch.bfloat16, seed=50 + i)):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        have = [x.clone() for x in got]
        want = step()
        gp.check()
        assert all(torch.equal(a, b) for a, b in zip(want, have))


SHAPE, NONFINITE, ARG, TIMEOUT = 2, 4, 1, 7


def test_refusals(P, gp):
    import torch
    from distill_ref import inputs
    T, V, d, k = 33, 500, 64, 6
    h, w, ids, t = inputs(T, V, d, k, torch.bfloat16, seed=2)
    want = gp.vocab_distill(h, w, ids, t)
    g = torch.rand(T, device="cuda")

    def at(x, r, c, v):
        x = x.clone()
        x[r, c] = v
        return x
    for i, v, code in ((at(ids, 3, 2, V), t, SHAPE), (at(ids, 3, 2, int(ids[3, 4])), t, SHAPE), (ids, at(t, 5, 0, math.nan), NONFINITE),
                       (ids, at(t, 5, 0, math.inf), NONFINITE)):
        gp.vocab_distill(h, w, i, v)
        again = gp.vocab_distill(h, w, ids, t)
        with pytest.raises(P.GraphPOError) as e:
            gp.check()
        assert e.value.code == code
        gp.check()
        assert all(torch.equal(again[n], want[n]) for n in want)
    gp.vocab_distill_grad(h, w, at(ids, 3, 2, V), want["delta"], want["rest"], want["rest_lse"], g)
    with pytest.raises(P.GraphPOError) as e:
        gp.check()
    assert e.value.code == SHAPE
    for kw in (dict(scale=0.0), dict(teacher_scale=math.nan), dict(teacher_scale=2.0, tail=True)):
        with pytest.raises(P.GraphPOError) as e:
            gp.vocab_distill(h, w, ids, t, **kw)
        assert e.value.code == ARG
    with pytest.raises(P.GraphPOError):
        gp.vocab_distill(h, w, ids.repeat(1, 100), t.repeat(1, 100))
    for bad in (lambda: gp.vocab_distill(h, w, ids[:, :3], t), lambda: gp.vocab_distill(h, w, ids.float(), t),
                lambda: gp.vocab_distill(h, w.half(), ids, t), lambda: gp.vocab_distill(h, w, ids, t, workspace=torch.empty(1 << 20, dtype=torch.uint8)),
                lambda: gp.vocab_distill_grad(h, w, ids, want["delta"][:, :3], want["rest"], want["rest_lse"], g),
                lambda: gp.vocab_distill_grad(h, w, ids, want["delta"], want["rest"], want["rest_lse"], g, accumulate=True)):
        with pytest.raises((ValueError, TypeError)):
            bad()
    with pytest.raises(P.GraphPOError) as e:  # a workspace too small
        gp.vocab_distill(h, w, ids, t, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 8
    gp.check()


def test_replays_keep_their_errors_until_check(P, gp):
    """Of captured calls the replays' errors are raised once each, and disturb no other replay; rows listed or not."""
    import torch
    from distill_ref import inputs
    for T, V, d in ((33, 500, 64), (2100, 66000, 1000)):
        h, w, ids, t = inputs(T, V, d, 6, torch.bfloat16, seed=2)
        good, g = ids.clone(), torch.rand(T, device="cuda")

        def step():
            f = gp.vocab_distill(h, w, ids, t)
            return f, gp.vocab_distill_grad(h, w, good, f["delta"], f["rest"], f["rest_lse"], g)["d_hidden"]
        want = [x.clone() for x in (step()[0]["loss"], step()[1])]
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            got = step()
        for code, bad in ((SHAPE, V), (SHAPE, int(ids[3, 4]))):
            ids[3, 2] = bad
            graph.replay()
            ids.copy_(good)
            graph.replay()
            with pytest.raises(P.GraphPOError) as e:
                gp.check()
            assert e.value.code == code
            gp.check()
            assert torch.equal(got[0]["loss"], want[0]) and torch.equal(got[1], want[1])


def test_a_wait_that_runs_out(P):
    """The tensor-core kernels' first wait gives up (about a millisecond): the call returns an error, the next one is right."""
    import torch
    from distill_ref import inputs
    h, w, ids, t = inputs(300, 900, 128, 9, torch.bfloat16, seed=5)
    slow = P.GraphPO(flags=P.binding.FLAG_DEBUG_TIMEOUT)
    f = slow.vocab_distill(h, w, ids, t)
    with pytest.raises(P.GraphPOError) as e:
        slow.check()
    assert e.value.code == TIMEOUT
    good = P.GraphPO()
    f = good.vocab_distill(h, w, ids, t)
    good.check()
    g = torch.ones(300, device="cuda")
    slow.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g)
    with pytest.raises(P.GraphPOError) as e:
        slow.check()
    assert e.value.code == TIMEOUT
    good.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], g)
    good.check()
