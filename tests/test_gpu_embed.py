"""gpo_embed and gpo_embed_grad against their formulas in 64 bits.

Every type, widths around the 512-byte column blocks, rows off their 16-byte boundaries, tables
around the rows a CTA of the sort owns, pieces of the sorted tokens that cut runs, one token for
the whole batch, no token at all, ids below 0, added gradients, refusals.  The gradient is linear in
its input, so that holding it against the formula also holds it against differences."""
import math

import pytest

pytestmark = pytest.mark.gpu

SHAPE, INVALID, UNSUPPORTED, WORKSPACE = 2, 1, 5, 8


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
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


def _ids(kind, T, V, seed, dtype):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    if kind == "uniform":
        x = (u * V).long()
    elif kind == "zipf":
        x = (torch.exp(u * math.log(V + 1)) - 1).long()
    elif kind == "one":
        x = torch.full((T,), V // 2, device="cuda")
    elif kind == "none":
        x = torch.full((T,), -1, device="cuda")
    else:  # "few": some rows, the last among them, and tokens without an id
        x = torch.where(u < 0.3, -5, torch.where(u < 0.6, V - 1, (u * 3).long()))
    return x.clamp(max=V - 1).to(dtype)


LOOK = [(1, 1, 1, 0), (1, 50, 4096, 0), (3, 10, 7, 0), (16, 1000, 256, 0), (100, 3000, 257, 1), (1001, 77, 1000, 4), (5000, 900, 64, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", LOOK)
def test_embed(gp, dtype, shape):
    import torch
    from vocab_ref import EPS
    T, V, d, off = shape
    table = torch.randn(V, d + off, device="cuda").to(_type(dtype))[:, off:]
    ids = _ids("few" if T > 3 else "uniform", T, V, T, torch.int64 if T % 2 else torch.int32)
    for scale in (1.0, 1.7):
        got = gp.embed(table, ids, scale=scale)
        gp.check()
        keep = (ids >= 0)[:, None]
        want = torch.where(keep, table[ids.clamp(min=0).long()].double() * scale, 0.0)
        assert got.dtype == table.dtype and got.shape == (T, d)
        # scale in fp32, the product in fp32, one rounding to the type
        tol = (EPS[table.dtype] * (1 + 2.0 ** -20) + 2.0 ** -23) * want.abs() + 2.0 ** -25
        assert torch.all((got.double() - want).abs() <= tol)
        if scale == 1.0:
            assert torch.equal(got, torch.where(keep, table[ids.clamp(min=0).long()], torch.zeros((), dtype=table.dtype, device="cuda")))


GRAD = [  # tokens, vocabulary, width, offset of the rows, ids
    (1, 1, 1, 0, "uniform"),
    (1, 33, 40, 0, "uniform"),
    (31, 5, 264, 0, "zipf"),
    (32, 4, 128, 0, "one"),
    (33, 4, 128, 0, "one"),
    (64, 64, 300, 1, "uniform"),
    (1000, 300, 257, 0, "few"),
    (1000, 200000, 16, 0, "uniform"),
    (4097, 1025, 72, 4, "zipf"),
    (5000, 3, 513, 0, "uniform"),
    (16385, 5000, 24, 0, "one"),
    (20000, 40000, 136, 8, "zipf"),
    (70001, 900, 8, 0, "zipf"),
    (300, 400, 48, 0, "none"),
    (0, 400, 48, 0, "none"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", GRAD)
def test_embed_grad(gp, dtype, shape):
    import torch
    from vocab_ref import EPS, TINY
    T, V, d, off, kind = shape
    torch.manual_seed(T)
    grad = (torch.randn(T, d + off, device="cuda") / 4).to(_type(dtype))[:, off:]
    ids = _ids(kind, T, V, T, torch.int64 if T % 2 else torch.int32)
    if (ids < 0).any():
        grad = grad.clone()
        grad[ids < 0] = math.nan  # reaches nothing
    scale = 0.75 if T % 3 else 1.0
    got = gp.embed_grad(grad, ids, V, scale=scale)
    again = gp.embed_grad(grad, ids, V, scale=scale)
    gp.check()
    keep = ids >= 0
    y, x = ids[keep].long(), grad[keep].double()
    want = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_put_((y,), x, accumulate=True) * scale
    size = torch.zeros_like(want).index_put_((y,), x.abs(), accumulate=True) * scale
    count = torch.bincount(y, minlength=V)[:, None].double()
    # a chain of at most count fp32 additions, the scale, one rounding
    eps = EPS[grad.dtype]
    tol = (count + 4) * 2.0 ** -24 * size * (1 + eps) + eps * want.abs() * (1 + 2.0 ** -10) + TINY[grad.dtype]
    assert got.dtype == grad.dtype and got.shape == (V, d)
    assert torch.all((got.double() - want).abs() <= tol)
    assert torch.equal(got, again)
    assert not got[count[:, 0] == 0].any()
    # added to a gradient that is there; rows without tokens keep what they hold
    base = torch.randn(V, d, device="cuda").to(grad.dtype)
    acc = base.clone()
    assert gp.embed_grad(grad, ids, V, scale=scale, out=acc, accumulate=True) is acc
    gp.check()
    both = want + base.double()
    tol = (count + 4) * 2.0 ** -24 * (size + base.double().abs()) * (1 + eps) + eps * both.abs() * (1 + 2.0 ** -10) + TINY[grad.dtype]
    assert torch.all((acc.double() - both).abs() <= tol)
    assert torch.equal(acc[count[:, 0] == 0], base[count[:, 0] == 0])


def test_outputs_stay_inside(gp):
    import torch
    T, V, d = 500, 130, 37
    for dtype in (torch.bfloat16, torch.float32):
        wide = torch.full((V + 2, d + 3), 3.0, device="cuda", dtype=dtype)
        ids = _ids("zipf", T, V, 1, torch.int32)
        gp.embed_grad(torch.randn(T, d, device="cuda").to(dtype), ids, V, out=wide[1:V + 1, 2:d + 2])
        rows = torch.full((T + 2, d + 3), 3.0, device="cuda", dtype=dtype)
        gp.embed(torch.randn(V, d, device="cuda").to(dtype), ids, out=rows[1:T + 1, 2:d + 2])
        gp.check()
        wide[1:V + 1, 2:d + 2] = 3.0
        rows[1:T + 1, 2:d + 2] = 3.0
        assert torch.all(wide == 3.0) and torch.all(rows == 3.0)


def test_another_stream_and_a_graph(gp):
    import torch
    T, V, d = 3000, 700, 96
    grad = torch.randn(T, d, device="cuda").bfloat16()
    ids = _ids("zipf", T, V, 3, torch.int64)
    want, look = gp.embed_grad(grad, ids, V), None
    look = gp.embed(want, ids)
    gp.check()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = gp.embed_grad(grad, ids, V)
        rows = gp.embed(got, ids)
    gp.check(s)
    assert torch.equal(got, want) and torch.equal(rows, look)
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    out, ids2 = torch.empty_like(want), ids.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gp.embed_grad(grad, ids2, V, out=out, workspace=ws)
    for k in range(2):
        ids2.copy_(ids if k else ids.flip(0))
        graph.replay()
    gp.check()
    assert torch.equal(out, want)


def test_refusals(gp):
    import torch
    import paper_2606_18954_gb300 as P
    table = torch.zeros(50, 64, device="cuda")
    ids = torch.zeros(5, device="cuda", dtype=torch.int32)

    def refused(code, f):
        with pytest.raises(P.GraphPOError) as e:
            f()
            gp.check()
        assert e.value.code == code, (e.value.code, gp.last_error())

    refused(INVALID, lambda: gp.embed(table, ids, scale=math.inf))
    refused(INVALID, lambda: gp.embed(table[:0], ids))
    refused(INVALID, lambda: gp.embed(table[:1].expand(50, 64), ids))
    refused(WORKSPACE, lambda: gp.embed_grad(torch.zeros(5, 64, device="cuda"), ids, 50, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")))
    refused(SHAPE, lambda: gp.embed(table, ids + 50))
    refused(SHAPE, lambda: gp.embed_grad(torch.zeros(5, 64, device="cuda"), ids + 50, 50))
    for f in (lambda: gp.embed(table.double(), ids), lambda: gp.embed(table, ids.short()),
              lambda: gp.embed(table, ids, out=torch.zeros(5, 64, device="cuda", dtype=torch.float16))):
        with pytest.raises(TypeError):
            f()
    for f in (lambda: gp.embed(table.t(), ids), lambda: gp.embed(table, ids.cpu()),
              lambda: gp.embed_grad(torch.zeros(5, 64, device="cuda"), ids[:4], 50),
              lambda: gp.embed_grad(torch.zeros(5, 64, device="cuda"), ids, 50, accumulate=True),
              lambda: gp.embed(table, ids, out=torch.zeros(4, 64, device="cuda"))):
        with pytest.raises(ValueError):
            f()
    assert torch.equal(gp.embed(table + 1, ids), torch.ones(5, 64, device="cuda"))
    gp.check()
