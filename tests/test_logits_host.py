"""The adjusted logits' host side without a device: struct layouts against the header, refusals."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2606_18954_gb300 import binding, build
    build()
    binding.load()
    return binding


def test_structs_match_the_header(B):
    import struct

    from test_abi import struct_fields
    for cls, name in ((B.CLogits, "gpo_logits"), (B.LogitsOutputs, "gpo_logits_outputs"), (B.LogitsGradInputs, "gpo_logits_grad_inputs")):
        assert [f for f, _ in cls._fields_] == struct_fields(name), name
    # the packed images are the structs'
    c = B.CLogits(*range(1, 13), *[float(x) for x in range(13, 17)], *range(17, 29))
    assert bytes(c) == B._PACK_LOGITS(*range(1, 13), *[float(x) for x in range(13, 17)], *range(17, 29))
    assert ctypes.sizeof(B.LogitsOutputs) == len(B._PACK_LOGITS_OUT(1, 2, 1, 4, 5, 6)) == 48
    got = struct.unpack("@Qqi3Q", bytes(B.LogitsOutputs(1, 2, 1, 4, 5, 6)))
    assert got == (1, 2, 1, 4, 5, 6)


def test_null_arguments(B):
    L = B.load()
    assert L.gpo_logits_adjust(None, ctypes.byref(B.CLogits()), None, None) == 1
    assert L.gpo_logits_grad(None, ctypes.byref(B.CLogits()), None, None, 0, None) == 1


def _context():
    """A context's binding without its device: what it refuses before the library is called."""
    from paper_2606_18954_gb300 import binding
    gp = object.__new__(binding.GraphPO)
    gp._device, gp._sizes, gp._rooms = -1, {}, {}  # (the host's tensors are on device -1)
    return gp


def test_the_binding_refuses(monkeypatch):
    import torch

    from paper_2606_18954_gb300 import binding
    monkeypatch.setattr(binding, "_matrix", lambda t, what, dev, rows, cols, dtype: _checked(t, what, rows, cols, dtype))

    def _checked(t, what, rows, cols, dtype):
        if tuple(t.shape) != (rows, cols):
            raise ValueError(what)
        if t.dtype is not dtype:
            raise TypeError(what)
        return t.stride(0)
    gp = _context()
    z = torch.zeros(3, 70)
    i32 = torch.int32
    v = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt)  # noqa: E731
    for bad, error in (
            (dict(scale=v(2)), ValueError), (dict(repetition=v(3).double()), TypeError), (dict(history=v(5, i32)), ValueError),
            (dict(spans=torch.zeros(3, 3, dtype=torch.int64)), ValueError), (dict(history=v(5), spans=v(9, torch.int64).view(3, 3)), TypeError),
            (dict(history=v(5, i32), spans=v(9, i32).view(3, 3)), TypeError), (dict(history=v(5, i32), spans=v(6, torch.int64).view(3, 2)), ValueError),
            (dict(bias=v(4)), ValueError), (dict(bias=v(4), bias_ids=v(5, i32)), ValueError), (dict(bias=v(4).double(), bias_ids=v(4, i32)), TypeError),
            (dict(bias=v(4), bias_ids=v(4, i32), bias_spans=v(9, torch.int64).view(3, 3)), ValueError),
            (dict(mask=v(4, i32).view(2, 2)), ValueError), (dict(mask=v(9, torch.int64).view(3, 3)), TypeError),
            (dict(mask=v(6, i32).view(2, 3)), ValueError), (dict(mask=v(6, i32).view(2, 3), mask_row=v(3, torch.int64)), TypeError),
            (dict(mask=v(0, i32).view(0, 3), mask_row=v(3, i32)), ValueError), (dict(target=v(3)), TypeError), (dict(target=v(4, i32)), ValueError),
            (dict(write=torch.float16), TypeError), (dict(bias_spans=v(6, torch.int64).view(3, 2)), ValueError),
            (dict(mask_row=v(3, i32)), ValueError)):
        with pytest.raises(error):
            gp.logits_adjust(z, **bad)
    for bad, error in ((dict(target=None), ValueError), (dict(lse=v(2)), ValueError), (dict(logp=v(3).double()), TypeError),
                       (dict(grad_entropy=v(3)), ValueError), (dict(out={"d_logits": z.half()}), TypeError)):
        args = dict(target=v(3, i32), lse=v(3), logp=v(3), grad_logp=v(3))
        args.update(bad)
        with pytest.raises(error):
            gp.logits_grad(z, **args)
    with pytest.raises(TypeError):
        gp.logits_adjust(z.double())
    with pytest.raises(ValueError):
        gp.logits_adjust(z[0])
    gp._device = 0
    with pytest.raises(ValueError):
        gp.logits_adjust(z)
