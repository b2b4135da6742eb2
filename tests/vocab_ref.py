"""The vocabulary ends' formulas in 64 bits (include/graphpo.h), with bounds of what the kernels'
roundings can make of them, and inputs for their tests."""
import math

import torch

U = 2.0 ** -24                                                    # unit roundoff of fp32
EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: U}  # of a value's rounding
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -126}


def rows(x, dtype, pad):
    """x in the given type, its rows on 16-byte boundaries: with `pad`, or an odd width, a view of a
    wider buffer filled with NaN."""
    n, d = x.shape
    if not pad and d % 8 == 0:
        return x.to(dtype)
    wide = torch.full((n, (d + 7) // 8 * 8 + 8 * pad), math.nan, dtype=dtype, device=x.device)
    wide[:, :d] = x
    return wide[:, :d]


def head_inputs(T, V, d, dtype, pad=0, masked=0.0, seed=0, id_dtype=torch.int32, sure=14.0):
    """hidden, weight, target of a policy head: hidden rows lean to their target's row by up to
    `sure`, rows without a target hold NaN or infinities."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 + seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    u = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    weight = n(V, d) * (1.5 / math.sqrt(d))
    target = torch.randint(0, V, (T,), generator=g, device="cuda")
    w = weight[target]
    hidden = n(T, d) + w * (u(T, 1) * sure / w.square().sum(1, keepdim=True).clamp(min=1e-3))
    drop = u(T) < masked
    bad = torch.tensor([math.nan, math.inf, -math.inf], device="cuda")
    hidden = torch.where(drop[:, None], bad[torch.arange(T, device="cuda") % 3][:, None], hidden)
    target = torch.where(drop, -1 - 99 * (torch.arange(T, device="cuda") % 2), target).to(id_dtype)
    return rows(hidden, dtype, pad), rows(weight, dtype, pad), target


def head_exact(hidden, weight, target, scale, g=None, e=None):
    """Forward results in 64 bits, and with g (and e) the gradients, each with a bound of the error.

    A logit is a sum of d products in fp32: at most 16 of its additions (a tensor-core instruction's
    k) or the order of a segment's lose an ulp of what has been added, taken here as 2 d / 16 + 32 roundings of the sum
    of |products|.  The sums over the vocabulary are relative to their maximum and good to a few
    roundings each; dz is rounded to 16 bits, and the gradients once more."""
    keep = target >= 0
    y = target.clamp(min=0).long()
    h = torch.where(keep[:, None], hidden, 0).double()
    w = weight.double()
    z = scale * (h @ w.t())
    lse = torch.logsumexp(z, 1)
    logq = z - lse[:, None]
    p = logq.exp()
    ent = -(p * torch.where(p > 0, logq, 0)).sum(1)
    d = h.shape[1]
    tz = (2 * d / 16 + 32) * U * scale * (h.abs() @ w.abs().t()).amax(1)     # of a logit
    tl = 2 * tz + 32 * U * (lse.abs() + 1)                                # of lse and logp
    te = (2 * tz + 64 * U) * (2 + ent + logq.abs().clamp(max=60).mul(p).sum(1)) + 32 * U  # of the entropy
    at = torch.arange(len(y), device=y.device)
    zero = lambda x: torch.where(keep, x, 0)  # noqa: E731
    out = dict(lse=zero(lse), logp=zero(logq[at, y]), entropy=zero(ent), t_lse=tl, t_logp=tl, t_entropy=te)
    if g is None:
        return out
    eps = EPS[hidden.dtype]
    gd = zero(g.double())
    ed = zero(e.double()) if e is not None else torch.zeros_like(gd)
    one = torch.zeros_like(p)
    one[at, y] = 1
    dz = gd[:, None] * (one - p) - ed[:, None] * p * (logq + ent[:, None])
    # dz: one rounding to 16 bits, and what lse's, the logits' and the entropy's errors make of p
    slack = (tl + tz)[:, None] * p * (gd.abs()[:, None] + ed.abs()[:, None] * ((logq + ent[:, None]).abs() + 1))
    slack = slack + p * (ed.abs() * te)[:, None] + 64 * U * (gd.abs()[:, None] * (one + p))
    tiny = TINY[hidden.dtype] * (gd.abs().amax() + 24 * ed.abs().amax()) * 2.0 ** -12
    ez = eps * dz.abs() + slack + torch.where((gd.abs() + ed.abs())[:, None] > 0, tiny, 0.0)
    small = TINY[hidden.dtype]
    for name, a, b, ea in (("d_hidden", dz, w, ez), ("d_weight", dz.t(), h, ez.t())):
        exact = scale * (a @ b)
        k = a.shape[1]
        part = scale * (ea @ b.abs()) + (2 * k / 16 + 32) * U * scale * (a.abs() @ b.abs())
        out[name] = exact
        out["t_" + name] = part * (1 + eps) + eps * exact.abs() + small
    return out


def close(got, want, tol, what):
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), (what, float(err[bad].max()), float(tol[bad].min()) if bad.any() else 0.0, int(bad.sum()))
