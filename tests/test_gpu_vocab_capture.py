"""Captured calls of the vocabulary ends without a workspace of the caller's: theirs comes from the graph's memory, not
from the context's, which later calls may replace or use on other streams."""
import pytest


def test_a_captured_call_leaves_the_contexts_workspaces_alone(monkeypatch):
    import torch
    from paper_2606_18954_gb300 import binding
    gp = object.__new__(binding.GraphPO)
    gp._device, gp._sizes, gp._rooms = 0, {}, {}
    capturing = False
    monkeypatch.setattr(binding, "_capturing", lambda: capturing)
    room = lambda n: gp._room(n, lambda: n, "cpu", None, 7)[0]  # noqa: E731
    own = room(1000)
    assert room(500) is own and gp._rooms == {7: own}
    capturing = True
    taken = room(1000)
    assert taken is not own and taken.numel() >= 1000 and gp._rooms[7] is own
    assert room(5000).numel() >= 5000 and gp._rooms[7] is own
    capturing = False
    assert room(1000) is own
    assert room(5000) is gp._rooms[7] and gp._rooms[7] is not own


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as pkg
    pkg.build()
    return pkg


def _step(gp, case):
    h, w, y = case
    f = gp.vocab_logp(h, w, y, entropy=True)
    d = gp.vocab_grad(h, w, y, f["lse"], f["entropy"], logp=f["logp"])
    x = gp.embed(w, y)
    e = gp.embed_grad(x, y, w.shape[0])
    return [f["logp"], f["lse"], f["entropy"], d["d_hidden"], d["d_weight"], x, e]


@pytest.mark.gpu
@pytest.mark.parametrize("T", [9, 300])
def test_replays_after_a_larger_call(P, T):
    import torch
    from vocab_ref import head_inputs
    gp = P.GraphPO()
    case = head_inputs(T, 900, 128, torch.bfloat16, seed=T)
    large = head_inputs(3000, 9000, 256, torch.bfloat16, seed=1)
    want = [t.clone() for t in _step(gp, case)]
    gp.check()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        _step(gp, case)  # the stream has a workspace already
        with torch.cuda.graph(graph, stream=s):
            got = _step(gp, case)
        _step(gp, large)  # which this call replaces
        gp.check(s)
        # what the allocator has free now belongs to these
        held = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in (1 << 12, 1 << 16, 1 << 18, 1 << 20, 1 << 22) * 8]
        for t in got:
            t.zero_()
        graph.replay()
        _step(gp, large)
        graph.replay()
        gp.check(s)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(bool((t == 7).all()) for t in held)


@pytest.mark.gpu
def test_two_graphs_on_two_streams(P):
    """Captured on one stream, replayed on two at the same time."""
    import torch
    from vocab_ref import head_inputs
    gp = P.GraphPO()
    cases = [head_inputs(T, V, d, torch.bfloat16, seed=T) for T, V, d in ((700, 9000, 256), (300, 30000, 128))]
    want = [[t.clone() for t in _step(gp, c)] for c in cases]
    gp.check()
    graphs, outs = [], []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_step(gp, c))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    gp.check()
    for got, ref in zip(outs, want):
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.gpu
def test_close_releases_the_workspaces(P):
    import torch
    from vocab_ref import head_inputs
    gp = P.GraphPO()
    _step(gp, head_inputs(300, 900, 128, torch.bfloat16, seed=2))
    gp.check()
    assert gp._rooms
    gp.close()
    assert not gp._rooms
