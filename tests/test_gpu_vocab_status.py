"""check() after several calls of the vocabulary ends: the first error of any of them is raised, once, whatever was
enqueued after it, and the failing call disturbs none of the others."""
import pytest

pytestmark = pytest.mark.gpu

SHAPE, REWARD, TIMEOUT = 2, 3, 7


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as pkg
    pkg.build()
    return pkg


def raised(P, gp, code, stream=None):
    with pytest.raises(P.GraphPOError) as e:
        gp.check(stream)
    assert e.value.code == code, (e.value.code, gp.last_error())
    gp.check(stream)  # once


class Calls:
    """The four operators on small inputs, with one id past the vocabulary on request."""

    def __init__(self, gp, T=40, V=300, d=64):
        import torch
        from vocab_ref import head_inputs
        self.gp, self.V = gp, V
        self.h, self.w, self.y = head_inputs(T, V, d, torch.bfloat16, seed=T)
        self.bad = self.y.clone()
        self.bad[T // 2] = V
        self.g = torch.randn(T, device="cuda")
        self.lse = gp.vocab_logp(self.h, self.w, self.y)["lse"]
        gp.check()

    def run(self, name, bad=False, stream=None):
        y = self.bad if bad else self.y
        if name == "logp":
            return self.gp.vocab_logp(self.h, self.w, y, stream=stream)["logp"]
        if name == "grad":
            return self.gp.vocab_grad(self.h, self.w, y, self.lse, self.g, stream=stream)["d_weight"]
        if name == "embed":
            return self.gp.embed(self.w, y, stream=stream)
        return self.gp.embed_grad(self.h, y, self.V, stream=stream)


NAMES = ("logp", "grad", "embed", "embed_grad")


@pytest.mark.parametrize("T", [9, 40, 4500])
@pytest.mark.parametrize("name", NAMES)
def test_an_error_is_kept_until_check(P, name, T):
    import torch
    gp = P.GraphPO()
    c = Calls(gp, T)
    want = {n: c.run(n).clone() for n in NAMES}
    gp.check()
    c.run(name, bad=True)
    got = {n: c.run(n) for n in NAMES}
    raised(P, gp, SHAPE)
    for n in NAMES:
        assert torch.equal(got[n], want[n]), n
    assert all(torch.equal(c.run(n), want[n]) for n in NAMES)
    gp.check()


def test_many_calls_later(P):
    """More calls than there are status words: an error in the first of them is raised all the same."""
    gp = P.GraphPO()
    c = Calls(gp, 9)
    c.run("embed", bad=True)
    for _ in range(700):
        c.run("embed")
    raised(P, gp, SHAPE)
    for i in range(700):
        c.run("embed", bad=i % 50 == 0)
    raised(P, gp, SHAPE)


def test_calls_of_other_kinds_between(P):
    """The advantage path's and the loss's own status, as before: the last call's; neither hides the other."""
    import torch
    from paper_2606_18954_gb300 import workloads as W
    b = W.make_batch(W.CONFIGS["tiny"].scaled(2))
    gp = P.GraphPO(kappa=b["kappa"], w=b["w"], lambda_eff=b["lambda_eff"])
    batch = P.Batch.from_arrays(b, device="cuda")
    c = Calls(gp)
    c.run("logp", bad=True)
    adv = gp(batch, nodes=True)
    lp = -torch.rand(batch.total_tokens, device="cuda")
    gp.token_loss(batch, gp.loss_plan(batch), lp, lp, edge_adv=adv["edge_adv"])
    raised(P, gp, SHAPE)
    good = batch.reward.clone()
    batch.reward[0] = 7
    gp(batch)
    c.run("embed")
    with pytest.raises(P.GraphPOError) as e:
        gp.check()
    assert e.value.code == REWARD
    c.run("embed")  # what has been raised is not this call's
    gp.check()
    batch.reward.copy_(good)
    gp(batch)
    gp.check()


def test_two_streams(P):
    import torch
    gp = P.GraphPO()
    c = Calls(gp)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    c.run("logp", bad=True, stream=streams[0])
    c.run("embed", stream=streams[1])
    c.run("embed", stream=streams[0])
    raised(P, gp, SHAPE, streams[0])
    gp.check(streams[1])


def test_a_timeout_is_kept(P):
    forced = P.GraphPO(flags=P.binding.FLAG_DEBUG_TIMEOUT)
    gp = P.GraphPO()
    for T in (9, 40):
        c = Calls(gp, T)
        c.gp = forced
        c.run("logp")
        c.run("embed")
        c.run("embed_grad")
        raised(P, forced, TIMEOUT)


@pytest.mark.parametrize("T", [9, 40])
def test_captured_calls(P, T):
    """Every captured call has status words of its own: the first call's error is not cleared by the second, a replay
    with valid inputs raises nothing, and a graph may be replayed when its context is gone."""
    import torch
    gp = P.GraphPO()
    c = Calls(gp, T)
    y = c.y.clone()
    room = torch.empty(8 << 20, dtype=torch.uint8, device="cuda")
    out, x = {"logp": torch.empty(T, device="cuda")}, torch.empty_like(c.h)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gp.vocab_logp(c.h, c.w, y, out=out, workspace=room)
        gp.embed(c.w, c.y, out=x, workspace=room)
    want = c.run("logp").clone()
    gp.check()
    for bad in (False, True, False, True, True, False):
        y.copy_(c.bad if bad else c.y)
        graph.replay()
        c.run("embed")  # (an eager call after it)
        if bad:
            raised(P, gp, SHAPE)
        else:
            gp.check()
            assert torch.equal(out["logp"], want)
    y.copy_(c.y)
    del gp, c.gp
    out["logp"].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out["logp"], want)


@pytest.mark.parametrize("T", [9, 40, 4500])
def test_replays_keep_their_errors_until_check(P, T):
    """A replay's error is raised though others with valid inputs follow it, which it does not disturb; every kernel that
    comes first in a call is captured once."""
    import torch
    gp = P.GraphPO()
    c = Calls(gp, T)
    want = {n: c.run(n).clone() for n in NAMES}
    gp.check()
    for name in NAMES:
        bad, c.bad = c.bad, c.y.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = c.run(name, bad=True)  # (reads c.bad, which the replays change)
        for _ in range(3):
            c.bad.copy_(bad)
            graph.replay()
            c.bad.copy_(c.y)
            for _ in range(2):
                got.zero_()
                graph.replay()
                assert torch.equal(got, want[name]), name
            raised(P, gp, SHAPE)
        graph.replay()
        gp.check()
        c.bad = bad


def test_a_replay_after_one_that_gave_up(P):
    import torch
    forced = P.GraphPO(flags=P.binding.FLAG_DEBUG_TIMEOUT)
    for T in (9, 40):
        c = Calls(P.GraphPO(), T)
        graph = torch.cuda.CUDAGraph()
        c.gp = forced
        with torch.cuda.graph(graph):
            c.run("logp")
        for _ in range(2):
            graph.replay()
            graph.replay()  # (with the first one's status still there)
            raised(P, forced, TIMEOUT)
        c.run("embed")
        forced.check()
