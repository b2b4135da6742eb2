"""The vocabulary ends take arrays and workspaces of the context's own device only: everything else is refused before a
launch."""
import pytest


def _cpu_context():
    from paper_2606_18954_gb300 import binding
    gp = object.__new__(binding.GraphPO)
    gp._device, gp._sizes, gp._rooms = 0, {}, {}
    return gp


def test_a_workspace_of_the_host_is_refused():
    import torch
    gp = _cpu_context()
    with pytest.raises(ValueError):
        gp._room((0,), lambda: 256, "cpu", torch.empty(1024, dtype=torch.uint8), 0)


def test_another_device_is_refused():
    import torch
    gp = _cpu_context()
    gp._device = 3  # (tensors of the host are on device -1)
    h, w, y = torch.zeros(4, 64).bfloat16(), torch.zeros(9, 64).bfloat16(), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: gp.vocab_logp(h, w, y), lambda: gp.vocab_grad(h, w, y, y.float(), y.float()), lambda: gp.embed(w, y),
                 lambda: gp.embed_grad(h, y, 9), lambda: gp._elsewhere(-1)):
        with pytest.raises(ValueError):
            call()


def _calls(gp):
    import torch
    h = torch.zeros(20, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.zeros(300, 64, device="cuda", dtype=torch.bfloat16)
    y = torch.zeros(20, device="cuda", dtype=torch.int32)
    f = torch.zeros(20, device="cuda")
    return [lambda **k: gp.vocab_logp(h, w, y, **k), lambda **k: gp.vocab_grad(h, w, y, f, f, **k),
            lambda **k: gp.embed(w, y, **k), lambda **k: gp.embed_grad(h, y, 300, **k)]


@pytest.mark.gpu
def test_refusals_on_the_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("a CUDA device is required for -m gpu tests")
    import paper_2606_18954_gb300 as P
    P.build()
    gp = P.GraphPO()
    good = torch.empty(1 << 20, device="cuda")  # (4 MB, whatever its type)
    for call in _calls(gp):
        for bad in (torch.empty(1 << 22, dtype=torch.uint8), torch.empty(1 << 22, dtype=torch.uint8).pin_memory(),
                    torch.empty(1 << 20, 2, device="cuda", dtype=torch.int32)[:, 0]):
            with pytest.raises(ValueError):
                call(workspace=bad)
        call(workspace=good)
        gp.check()
        own = gp._device
        gp._device = own + 1  # as if the context were another device's
        try:
            with pytest.raises(ValueError):
                call()
            with pytest.raises(ValueError):
                call(workspace=good)
        finally:
            gp._device = own
        call()
        gp.check()
