"""Log-probabilities of up to 16 tokens, one launch (gpo_vocab_few.cu), over that kernel's range: token counts on both
sides of its two column halves, vocabularies of one box of 32 rows up to several whole tiles of 128 per CTA (the running
maximum and sum carried on), widths of several accumulations of 128 and of more steps than its ring holds, odd ends of
each, masked and NaN rows, targets outside the vocabulary, given-up waits, captured calls and two streams."""
import math

import pytest

pytestmark = pytest.mark.gpu

SHAPE, TIMEOUT = 2, 7


@pytest.fixture(scope="module")
def gp():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as pkg
    pkg.build()
    return pkg.GraphPO()


def _type(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16}[name]


CASES = [  # tokens, vocabulary, width, pad, masked, scale
    (1, 32, 64, 0, 0.0, 1.0),
    (6, 33, 128, 0, 0.0, 1.0),
    (8, 4864, 129, 0, 0.0, 1.0),           # one box per CTA of 152, one column past an accumulation
    (9, 4865, 192, 1, 0.3, 1.25),
    (15, 14591, 256, 0, 0.0, 1.0),         # three boxes per CTA, the last row missing
    (16, 19456, 136, 0, 0.4, 1.0),         # one whole tile per CTA
    (7, 19457, 520, 1, 0.0, 0.7),          # a second tile for some
    (16, 40001, 264, 0, 0.2, 1.0),         # two tiles and more, the last of few rows
    (12, 100003, 200, 0, 0.0, 1.0),
    (1, 131072, 333, 0, 0.0, 1.0),
    (10, 20011, 1024, 0, 0.0, 1.0),        # 16 steps of 64 k a tile: the ring and the four accumulators go round
    (3, 50021, 4096, 0, 0.5, 1.0),
    (16, 30000, 2056, 1, 0.3, 2.0),
    (11, 25000, 24, 0, 1.0, 1.0),          # no token at all
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", CASES)
def test_few_tokens(gp, dtype, shape):
    import torch
    from vocab_ref import close, head_exact, head_inputs
    T, V, d, pad, masked, scale = shape
    h, w, y = head_inputs(T, V, d, _type(dtype), pad, masked, seed=V + T, id_dtype=torch.int64 if T % 2 else torch.int32)
    gp.vocab_logp(h, w, y.flip(0))  # leaves its own parts and marks behind
    out = gp.vocab_logp(h, w, y, scale=scale, entropy=True)
    plain = gp.vocab_logp(h, w, y, scale=scale)
    again = gp.vocab_logp(h, w, y, scale=scale, entropy=True)
    gp.check()
    ref = head_exact(h, w, y, scale)
    for k in ("logp", "lse", "entropy"):
        close(out[k], ref[k], ref["t_" + k], k)
        assert torch.equal(out[k], again[k]), k
        assert not out[k][y < 0].any()
    for k in ("logp", "lse"):
        close(plain[k], ref[k], ref["t_" + k], k)


@pytest.mark.parametrize("T", list(range(1, 18)))
def test_every_number_of_tokens(gp, T):
    """And each token in every column: its results do not depend on which column it is in, nor on the others."""
    import torch
    from vocab_ref import close, head_exact, head_inputs
    V, d = 20001, 144
    h, w, y = head_inputs(17, V, d, torch.bfloat16, seed=5)
    at = (torch.arange(T, device="cuda") + 3) % 17
    out = gp.vocab_logp(h[at].contiguous(), w, y[at].contiguous(), entropy=True)
    gp.check()
    ref = head_exact(h[at].contiguous(), w, y[at], 1.0)
    for k in ("logp", "lse", "entropy"):
        close(out[k], ref[k], ref["t_" + k], k)


@pytest.mark.parametrize("T", [1, 8, 16])
def test_targets_everywhere(gp, T):
    """The target in the first and last row of a box, of a tile, of a CTA's share and of the vocabulary."""
    import torch
    from vocab_ref import close, head_exact, head_inputs
    V, d = 40003, 72
    h, w, _ = head_inputs(T, V, d, torch.float16, seed=9)
    for first in (0, 31, 32, 127, 128, 263, 264, 20000, V - 33, V - 20):
        y = (first + torch.arange(T, device="cuda")).clamp(max=V - 1).int()
        out = gp.vocab_logp(h, w, y, entropy=True)
        ref = head_exact(h, w, y, 1.0)
        for k in ("logp", "lse", "entropy"):
            close(out[k], ref[k], ref["t_" + k], (k, first))
    gp.check()


def test_as_exact_as_32_bits(gp):
    """2-norm errors against torch's own 32-bit products and sums, as for more tokens: no more than 1.5 times theirs or 1e-6."""
    import torch
    from vocab_ref import head_exact, head_inputs
    for dtype in (torch.bfloat16, torch.float16):
        for T, V, d in ((16, 30000, 2048), (7, 20000, 4096), (1, 50000, 1024)):
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
    import torch
    V, d = 40000, 256
    w = torch.zeros(V, d, device="cuda", dtype=torch.bfloat16)
    w[:, 200] = -1.0
    w[39999, 200] = 1.0
    h = torch.zeros(12, d, device="cuda", dtype=torch.bfloat16)
    h[:, 200] = torch.linspace(8.0, 13.0, 12)
    out = gp.vocab_logp(h, w, torch.full((12,), 39999, device="cuda", dtype=torch.int32), entropy=True)
    gp.check()
    z = 2.0 * h[:, 200].double()
    others = (V - 1) * torch.exp(-z)
    want = -torch.log1p(others)
    assert torch.all((out["logp"].double() - want).abs() <= 64 * 2.0 ** -24 * 30 * want.abs())
    ent = torch.log1p(others) + others * z / (1 + others)
    assert torch.all((out["entropy"].double() - ent).abs() <= 64 * 2.0 ** -24 * 30 * ent)


def test_nan_rows_and_large_logits(gp):
    import torch
    from vocab_ref import close, head_exact, head_inputs
    h, w, y = head_inputs(14, 21000, 160, torch.bfloat16, seed=5)
    h = h.clone()
    h[3, 5] = math.nan
    h[9] = h[9] * 1e4
    h[12] = 0.0
    out = gp.vocab_logp(h, w, y, entropy=True)
    gp.check()
    assert math.isnan(float(out["logp"][3])) and math.isnan(float(out["lse"][3]))
    fine = torch.arange(14, device="cuda") != 3
    ref = head_exact(h[fine].contiguous(), w, y[fine].contiguous(), 1.0)
    for k in ("logp", "lse", "entropy"):
        close(out[k][fine], ref[k], ref["t_" + k], k)
    assert abs(float(out["lse"][12]) - math.log(21000)) < 1e-5 and abs(float(out["entropy"][12]) - math.log(21000)) < 1e-5


@pytest.mark.parametrize("T", [1, 8, 16])
def test_target_outside_the_vocabulary(gp, T):
    import torch
    import paper_2606_18954_gb300 as P
    from vocab_ref import head_inputs
    h, w, y = head_inputs(T, 20500, 136, torch.bfloat16, seed=2)
    good = gp.vocab_logp(h, w, y)
    gp.check()
    for id_dtype, past in ((torch.int32, 20500), (torch.int64, 1 << 40)):
        bad = y.to(id_dtype, copy=True)
        bad[T // 2] = past
        gp.vocab_logp(h, w, bad)
        with pytest.raises(P.GraphPOError) as e:
            gp.check()
        assert e.value.code == SHAPE
    again = gp.vocab_logp(h, w, y)
    gp.check()
    assert torch.equal(again["logp"], good["logp"])


def test_forced_timeout_then_a_normal_call(gp):
    import torch
    import paper_2606_18954_gb300 as P
    from vocab_ref import close, head_exact, head_inputs
    h, w, y = head_inputs(13, 40000, 512, torch.bfloat16, seed=9)
    forced = P.GraphPO(flags=P.binding.FLAG_DEBUG_TIMEOUT)
    room = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")  # both contexts' in turn
    for _ in range(2):
        forced.vocab_logp(h, w, y, workspace=room)
        with pytest.raises(P.GraphPOError) as e:
            forced.check()
        assert e.value.code == TIMEOUT
        out = gp.vocab_logp(h, w, y, entropy=True, workspace=room)
        gp.check()
        ref = head_exact(h, w, y, 1.0)
        for k in out:
            close(out[k], ref[k], ref["t_" + k], k)


def test_a_graph_and_two_streams(gp):
    """Replays share one call's mark, so they clear the marks: new inputs, new results; and calls of two streams at once."""
    import torch
    from vocab_ref import head_inputs
    cases = [head_inputs(T, V, d, torch.bfloat16, seed=T) for T, V, d in ((16, 30000, 256), (5, 60000, 512))]
    want = [gp.vocab_logp(*c, entropy=True) for c in cases]
    gp.check()
    h, w, y = cases[0]
    room = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    h2, out = h.clone(), {k: torch.empty_like(t) for k, t in want[0].items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gp.vocab_logp(h2, w, y, out=out, workspace=room)
    flipped = gp.vocab_logp(h.flip(0).contiguous(), w, y, entropy=True)
    for k in range(6):
        h2.copy_(h if k % 2 else h.flip(0))
        graph.replay()
        gp.check()
        assert all(torch.equal(out[n], (want[0] if k % 2 else flipped)[n]) for n in out), k
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for _ in range(30):
        got.append([gp.vocab_logp(*c, entropy=True, stream=s) for c, s in zip(cases, streams)])
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a[n], b[n]) for a, b in zip(g, want) for n in b)
    gp.check()
