"""Adjusted logits and distillation on two streams at once, eager and replayed: each has the bits that it has alone."""
import pytest

from test_gpu_logits import P, gp  # noqa: F401

pytestmark = pytest.mark.gpu


def _steps(gp, seed):  # noqa: F811
    import torch
    import distill_ref
    import logits_ref
    z, y, how = logits_ref.inputs(150 + 200 * seed, 20011, torch.bfloat16, seed=seed, masks=2, history=900, biases=30, pad=seed)
    h, w, ids, t = distill_ref.inputs(700 + 900 * seed, 5003, 264, 24, torch.float16, seed=seed, masked=0.2, short=True, tail=True)
    g, k = torch.randn(len(y), device="cuda"), torch.rand(len(h), device="cuda")

    def step():
        a = gp.logits_adjust(z, y, entropy=True, **how)
        b = gp.logits_adjust(z, write=torch.bfloat16, entropy=True, **how)
        d = gp.logits_grad(z, y, a["lse"], a["logp"], g, entropy=a["entropy"], grad_entropy=g, **how)
        f = gp.vocab_distill(h, w, ids, t, tail=True)
        r = gp.vocab_distill_grad(h, w, ids, f["delta"], f["rest"], f["rest_lse"], k)
        return [x for o in (a, b, d, f, r) for x in o.values()]
    return step


def _same(a, b):
    import torch
    bits = lambda x: x.view(torch.int16 if x.element_size() == 2 else torch.int32)  # noqa: E731  (a NaN equals itself)
    return all(torch.equal(bits(x), bits(y)) for x, y in zip(a, b))


def test_two_streams_at_once(gp):  # noqa: F811
    import torch
    steps = [_steps(gp, i) for i in range(2)]
    want = [s() for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(steps[i]())
    torch.cuda.synchronize()
    gp.check()
    assert all(_same(o, want[i]) for i in range(2) for o in got[i])


def test_two_graphs_at_once(gp):  # noqa: F811
    import torch
    steps = [_steps(gp, i) for i in range(2)]
    want = [s() for s in steps]
    torch.cuda.synchronize()
    graphs, got = [torch.cuda.CUDAGraph() for _ in steps], []
    for g, s in zip(graphs, steps):
        with torch.cuda.graph(g):
            got.append(s())
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for o in got:
            for x in o:
                x.zero_()
        torch.cuda.synchronize()
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                graphs[i].replay()
                graphs[i].replay()
        steps[0]()  # (an eager call beside them)
        torch.cuda.synchronize()
        gp.check()
        assert all(_same(o, w) for o, w in zip(got, want))
