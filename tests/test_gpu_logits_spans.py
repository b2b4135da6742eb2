"""Rows that one CTA takes in several spans (81408 entries of 16 bits, 81664 of 32), of lengths about a span's."""
import pytest

from test_gpu_logits import P, _types, gp  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V, dtype", [(81407, "bf16"), (81408, "f16"), (81409, "bf16"), (81425, "f16"), (81664, "f32"), (81665, "f32"), (162816, "bf16"),
                                      (162835, "f16")])
def test_about_a_spans_length(gp, V, dtype):  # noqa: F811
    """310 rows: more than share an SM's places with clusters.  Histories, biases and targets at both ends of the spans."""
    import torch
    from logits_ref import exact, inputs, near
    R = 310
    z, y, how = inputs(R, V, _types()[dtype], seed=V, pad=V % 5, history=50, masks=2, biases=40)
    per = 81664 if dtype == "f32" else 81408
    head = (0 - z.data_ptr() // z.element_size()) % (32 // z.element_size())  # (of the first row; the others' differ with the stride)
    ends = [v for e in (per, 2 * per) for v in range(e + head - 20, e + head + 20) if v < V] + [V - 1]
    ends = torch.tensor(ends, device="cuda")
    h = how["history"]
    h[::3] = ends[torch.arange(len(h[::3]), device="cuda") % len(ends)].to(h.dtype)
    at = torch.arange(0, R, 2, device="cuda")
    y[at] = ends[at // 2 % len(ends)].to(y.dtype)
    z[at, y[at].long()] = 9.0
    how["mask_row"][::4] = -1  # (whose rows then hold no NaN)
    z[::4] = torch.where(z[::4].abs() < 100, z[::4], 0.5)
    g, e = torch.randn(R, device="cuda"), torch.randn(R, device="cuda") * 0.1
    ref, every = exact(z, y, how, g, e), exact(z, None, how)
    f = gp.logits_adjust(z, y, entropy=True, **how)
    d = gp.logits_grad(z, y, f["lse"], f["logp"], g, entropy=f["entropy"], grad_entropy=e, **how)["d_logits"]
    s = gp.logits_adjust(z, write=torch.float32, entropy=True, **how)
    gp.check()
    for k in f:
        near(f[k], ref[k], ref["t_" + k], k)
    near(d, ref["d_logits"], ref["t_d_logits"], "d_logits")
    for k in ("lse", "entropy"):
        near(s[k], every[k], every["t_" + k], k)
    t = every["t_logits"] + 2.0 ** -24 * torch.where(torch.isfinite(every["logits"]), every["logits"].abs(), 0.0)
    near(s["logits"], every["logits"], t, "logits")
