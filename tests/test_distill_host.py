"""The distillation's host side without a device: struct layouts against the header, workspace sizes, refusals."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2606_18954_gb300 import binding, build
    build()
    binding.load()
    return binding


def test_structs_match_the_header(B):
    from test_abi import struct_fields
    for cls, name in ((B.CTeacher, "gpo_teacher"), (B.DistillOutputs, "gpo_distill_outputs"), (B.DistillGradInputs, "gpo_distill_grad_inputs")):
        assert [f for f, _ in cls._fields_] == struct_fields(name), name
    assert bytes(B.CTeacher(*range(1, 9), 9.0)) == B._PACK_TEACHER(*range(1, 9), 9.0)
    assert bytes(B.DistillOutputs(*range(1, 7))) == B._PACK_DISTILL_OUT(*range(1, 7))
    assert bytes(B.DistillGradInputs(*range(1, 6))) == B._PACK_DISTILL_IN(*range(1, 6))


def vocab(B, **kw):
    a = dict(num_tokens=100, vocab=1000, d=64, hidden_stride=64, weight_stride=64, hidden=None, weight=None, target=None,
             dtype=0, id_bytes=0, scale=1.0)
    a.update(kw)
    return B.CVocab(*[a[f] for f, _ in B.CVocab._fields_])


def teacher(B, **kw):
    a = dict(k=8, ids_stride=8, logits_stride=8, ids=None, logits=None, id_bytes=4, dtype=1, tail=0, scale=1.0)
    a.update(kw)
    return B.CTeacher(*[a[f] for f, _ in B.CTeacher._fields_])


def test_workspace(B):
    size = lambda grad=False, k=8, **kw: B.distill_workspace_size(vocab(B, **kw), teacher(B, k=k, ids_stride=k, logits_stride=k), grad)  # noqa: E731
    assert 0 < size(num_tokens=0) < size(num_tokens=1) < size(num_tokens=1000) < size(num_tokens=5000)
    assert size(k=8) < size(k=64) < size(k=512)
    # beside the forward pass and the gradient of the products: a few words per token and entry, and forward two bytes per token and
    # 128 columns of the vocabulary (1000: 8 of them, a border more)
    for grad, words in ((False, 5), (True, 0)):
        for T, k in ((100, 8), (5000, 64), (3, 512)):
            more = size(grad, k, num_tokens=T) - B.vocab_workspace_size(vocab(B, num_tokens=max(T, 17), id_bytes=4), grad)
            assert more <= 4 * T * (words * (k + 8) + 6) + 20 * T * (not grad) + 12 * 256, (grad, T, k, more)


@pytest.mark.parametrize("bad, code", [
    (dict(k=0), 1), (dict(k=-1), 1), (dict(k=513, ids_stride=513, logits_stride=513), 5), (dict(ids_stride=7), 1), (dict(id_bytes=2), 1),
    (dict(ids_stride=1 << 40), 5)])
def test_refusals(B, bad, code):
    n = ctypes.c_size_t()
    for grad in (0, 1):
        assert B.load().gpo_vocab_distill_workspace_size(ctypes.byref(vocab(B)), ctypes.byref(teacher(B, **bad)), grad, ctypes.byref(n)) == code
    for wrong, status in ((dict(num_tokens=-1), 1), (dict(vocab=0), 1), (dict(dtype=1), 5), (dict(hidden_stride=63), 1)):
        assert B.load().gpo_vocab_distill_workspace_size(ctypes.byref(vocab(B, **wrong)), ctypes.byref(teacher(B)), 0, ctypes.byref(n)) == status
    # (the gradient does not read the teacher's logits)
    assert B.load().gpo_vocab_distill_workspace_size(ctypes.byref(vocab(B)), ctypes.byref(teacher(B, logits_stride=7)), 0, ctypes.byref(n)) == 1
    assert B.load().gpo_vocab_distill_workspace_size(ctypes.byref(vocab(B)), ctypes.byref(teacher(B, logits_stride=7)), 1, ctypes.byref(n)) == 0


def test_null_arguments(B):
    L, n = B.load(), ctypes.c_size_t()
    v, t = ctypes.byref(vocab(B)), ctypes.byref(teacher(B))
    assert L.gpo_vocab_distill_workspace_size(None, t, 0, ctypes.byref(n)) == 1
    assert L.gpo_vocab_distill_workspace_size(v, None, 0, ctypes.byref(n)) == 1
    assert L.gpo_vocab_distill_workspace_size(v, t, 0, None) == 1
    assert L.gpo_vocab_distill(None, v, t, None, None, 0, None) == 1
    assert L.gpo_vocab_distill_grad(None, v, t, None, None, None, 0, None) == 1


def test_the_binding_refuses():
    import torch

    from paper_2606_18954_gb300 import binding
    gp = object.__new__(binding.GraphPO)
    gp._device, gp._sizes, gp._rooms = 0, {}, {}
    h, w = torch.zeros(4, 64).bfloat16(), torch.zeros(9, 64).bfloat16()
    i, t, f = torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3), torch.zeros(4)
    for args in ((h, w, i, t), (h[0], w, i, t), (h, w, i[0], t), (h, w, i[:2], t)):
        with pytest.raises(ValueError):  # (the host's arrays)
            gp.vocab_distill(*args)
    for args, error in (((h, w, i.float(), t), TypeError), ((h.double(), w, i, t), TypeError)):
        with pytest.raises((error, ValueError)):
            gp.vocab_distill(*args)
    with pytest.raises(ValueError):
        gp.vocab_distill_grad(h, w, i, t, f, f, f)
