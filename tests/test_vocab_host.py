"""The vocabulary ends' host side without a device: struct layouts against the header, workspace
sizes, refusals of sizes."""
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
    for cls, name in ((B.CVocab, "gpo_vocab"), (B.VocabOutputs, "gpo_vocab_outputs"),
                      (B.VocabGradInputs, "gpo_vocab_grad_inputs"), (B.VocabGrads, "gpo_vocab_grads"),
                      (B.CEmbedding, "gpo_embedding")):
        assert [f for f, _ in cls._fields_] == struct_fields(name), name


def vocab(B, **kw):
    a = dict(num_tokens=100, vocab=1000, d=64, hidden_stride=64, weight_stride=64, hidden=None, weight=None, target=None,
             dtype=0, id_bytes=4, scale=1.0)
    a.update(kw)
    return B.CVocab(*[a[f] for f, _ in B.CVocab._fields_])


def embedding(B, **kw):
    a = dict(num_tokens=100, vocab=1000, d=64, table_stride=64, row_stride=64, ids=None, dtype=1, id_bytes=4, scale=1.0)
    a.update(kw)
    return B.CEmbedding(*[a[f] for f, _ in B.CEmbedding._fields_])


def test_vocab_workspace(B):
    size = lambda grad=False, **kw: B.vocab_workspace_size(vocab(B, **kw), grad)  # noqa: E731
    assert 0 < size(num_tokens=0) < size(num_tokens=1) == size(num_tokens=16)  # up to 16 tokens: one launch's own parts
    assert size(num_tokens=65) <= size(num_tokens=256) < size(num_tokens=257) < size(num_tokens=5000)
    # never a whole [T x V] matrix: the gradient's largest part is a piece of 512 MiB at most
    big = dict(num_tokens=1 << 17, vocab=1 << 18, d=1024, hidden_stride=1024, weight_stride=1024)
    hidden = (1 << 17) * 1024
    assert size(True, **big) < (512 << 20) + 4 * hidden + 2 * hidden + (8 << 20)
    assert size(**big) < 2 * (1 << 17) * (1 << 18) // 4
    # fp32 sums of d_hidden: none with one piece and enough row tiles for the GPU, else at most 32 of them
    wide = dict(num_tokens=4096, d=4096, hidden_stride=4096, weight_stride=4096)
    assert size(True, vocab=8192, **wide) < 2 * 4096 * 8192 + 2 * 4096 * 4096 + (1 << 20)
    assert size(True, num_tokens=300, vocab=100000) < 2 * 512 * 100352 + 32 * 4 * 512 * 64 + (1 << 20)


@pytest.mark.parametrize("bad, code", [
    (dict(num_tokens=-1), 1), (dict(vocab=0), 1), (dict(d=0), 1), (dict(hidden_stride=63), 1), (dict(weight_stride=63), 1),
    (dict(dtype=1), 5), (dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(id_bytes=2), 1), (dict(num_tokens=1 << 31), 5),
    (dict(vocab=1 << 31), 5), (dict(hidden_stride=1 << 40), 5), (dict(vocab=1 << 30, weight_stride=1 << 30), 5),
    (dict(num_tokens=(1 << 31) - 2048, vocab=(1 << 31) - 2048), 5)])
def test_vocab_refusals(B, bad, code):
    n = ctypes.c_size_t()
    for grad in (0, 1):
        assert B.load().gpo_vocab_workspace_size(ctypes.byref(vocab(B, **bad)), grad, ctypes.byref(n)) == code
    with pytest.raises(B.GraphPOError):
        B.vocab_workspace_size(vocab(B, **bad))


def test_embed_workspace(B):
    size = lambda grad=False, **kw: B.embed_workspace_size(embedding(B, **kw), grad)  # noqa: E731
    assert 0 < size() <= 256 and size() == size(num_tokens=1 << 20)
    assert size() < size(True) < size(True, num_tokens=10000)


@pytest.mark.parametrize("bad, code", [
    (dict(num_tokens=-1), 1), (dict(vocab=0), 1), (dict(d=0), 1), (dict(table_stride=63), 1), (dict(row_stride=63), 1),
    (dict(dtype=3), 1), (dict(id_bytes=1), 1), (dict(num_tokens=1 << 31), 5), (dict(vocab=1 << 31), 5),
    (dict(vocab=1 << 30, table_stride=1 << 30), 5)])
def test_embed_refusals(B, bad, code):
    n = ctypes.c_size_t()
    for grad in (0, 1):
        assert B.load().gpo_embed_workspace_size(ctypes.byref(embedding(B, **bad)), grad, ctypes.byref(n)) == code


def test_null_arguments(B):
    L, n = B.load(), ctypes.c_size_t()
    assert L.gpo_vocab_workspace_size(None, 0, ctypes.byref(n)) == 1
    assert L.gpo_vocab_workspace_size(ctypes.byref(vocab(B)), 0, None) == 1
    assert L.gpo_embed_workspace_size(None, 0, ctypes.byref(n)) == 1
    assert L.gpo_embed(None, ctypes.byref(embedding(B)), None, None, None, 0, None) == 1
    assert L.gpo_embed_grad(None, ctypes.byref(embedding(B)), None, None, 0, None, 0, None) == 1
    assert L.gpo_vocab_grad(None, ctypes.byref(vocab(B)), None, None, None, 0, None) == 1
