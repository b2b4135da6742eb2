"""The distillation's formulas in 64 bits (include/graphpo.h), with bounds of what the kernels' roundings can make of
them, and inputs for their tests."""
import math

import torch

from vocab_ref import EPS, TINY, U, rows

EX2 = 2.0 ** -21  # of an approximate exponential, and of a sum of them


def inputs(T, V, d, k, dtype, teacher=torch.float32, pad=0, masked=0.0, short=False, tail=False, ids=torch.int32, seed=0, sure=14.0, teacher_scale=1.0,
           spread=1.0):
    """hidden, weight, ids, teacher's logits: a teacher on hidden states `spread` away from the policy's, its entries in any order; with
    `short` rows of fewer entries (at any place, their logits NaN), and some of probability 0; rows without any hold NaN or infinities."""
    g = torch.Generator(device="cuda")
    g.manual_seed(500 + seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    u = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    weight = n(V, d) * (1.5 / math.sqrt(d))
    w = weight[torch.randint(0, V, (T,), generator=g, device="cuda")]
    hidden = n(T, d) + w * (u(T, 1) * sure / w.square().sum(1, keepdim=True).clamp(min=1e-3))
    z = (hidden + spread * n(T, d)) @ weight.t()
    if tail:
        z = torch.log_softmax(z, 1)
    t, i = z.topk(k, dim=1)
    order = torch.argsort(u(T, k), dim=1)
    t, i = t.gather(1, order) / (1.0 if tail else teacher_scale), i.gather(1, order)
    if short:
        off = u(T, k) < u(T, 1) * 0.9
        off[torch.arange(T, device="cuda"), torch.randint(0, k, (T,), generator=g, device="cuda")] = False
        i = torch.where(off, -1 - i, i)
        t = torch.where(off, math.nan, t)
        zero = ~off & (u(T, k) < 0.1)
        zero[torch.arange(T, device="cuda"), torch.where(off, -math.inf, t.double()).argmax(1)] = False
        t = torch.where(zero, -math.inf, t)
    drop = u(T) < masked
    bad = torch.tensor([math.nan, math.inf, -math.inf], device="cuda")
    hidden = torch.where(drop[:, None], bad[torch.arange(T, device="cuda") % 3][:, None], hidden)
    i = torch.where(drop[:, None], -1, i)
    wide = lambda x, fill: torch.cat([x, torch.full_like(x[:, :pad], fill)], 1)[:, :k]  # noqa: E731
    return rows(hidden, dtype, pad), rows(weight, dtype, pad), wide(i.to(ids), 0), wide(t.to(teacher), 1.0)


def exact(hidden, weight, ids, teacher, scale=1.0, teacher_scale=1.0, tail=False, g=None):
    """Results in 64 bits with bounds t_*: forward, and with g the gradients.

    A logit is good to 2 d / 16 + 32 roundings of the sum of |products| (vocab_ref.head_exact), a teacher's probability to a
    dozen roundings and those of its logits; a probability moves by p (1 - p) of its logit's error; sums of
    exponentials are good to EX2.  The largest entry's p - q comes from 1 - q and 1 - p, which are sums."""
    T, k = ids.shape
    V, d = weight.shape
    entry = ids >= 0
    tv = torch.where(entry, teacher.double(), -math.inf) * (1.0 if tail else teacher_scale)
    live = entry.any(1) & (tail | (tv.amax(1) > -math.inf))
    h = torch.where(live[:, None], hidden, 0).double()
    w = weight.double()
    z = scale * (h @ w.t())
    inside = torch.zeros(T, V, dtype=torch.bool, device=z.device)
    r, c = torch.nonzero(entry, as_tuple=True)
    inside[r, ids[r, c].long()] = True
    lse = torch.logsumexp(z, 1)
    lr = torch.logsumexp(torch.where(inside, -math.inf, z), 1)
    mass = torch.logsumexp(tv, 1)
    mass = mass.clamp(min=0) if tail else mass
    lq = torch.where(live[:, None], tv - mass[:, None], -math.inf)
    q = lq.exp()
    qr = (1 - q.sum(1)).clamp(min=0) * (lr > -math.inf) if tail else torch.zeros_like(lse)
    i = ids.clamp(min=0).long()
    lp = torch.where(entry, z.gather(1, i) - lse[:, None], -math.inf)
    p, pr = lp.exp(), (lr - lse).exp()
    some = live & (lr > -math.inf)
    zero = lambda x: torch.where(live, x, 0)  # noqa: E731
    plus = lambda a, x: torch.where(a, x, 0.0)  # noqa: E731
    loss = plus(entry & (q > 0), q * (lq - lp)).sum(1) + plus(qr > 0, qr * (qr.log() - (lr - lse)))
    tz = (2 * d / 16 + 32) * U * scale * (h.abs() @ w.abs().t()).amax(1)          # of a logit
    tl = 2 * tz + 32 * U * (lse.abs() + 1) + EX2                                # of lse
    tr = torch.where(some, 2 * tz + 32 * U * (lr.abs() + 1) + EX2, 0.0)         # of rest_lse
    big = torch.where(entry & (tv > -math.inf), tv.abs(), 0.0).amax(1)
    tq = 16 * U * (big + mass.abs().nan_to_num(0, 0, 0) + 4)                    # of log q
    eq = (8 * U + tq * 0.25) * float(tail)                                     # of q_r: of probabilities that sum to 1, their roundings
    gap = plus(entry & (q > 0), (lq - lp).abs())
    t_loss = (q * (tq[:, None] * (gap + 1) + (tz + tl)[:, None] + 16 * U * (1 + gap + lp.abs().clamp(max=1e4)))).nan_to_num(0, 0, 0).sum(1) + plus(
        qr > 0, qr * (tr + tl + 16 * U * (lr - lse).abs()) + eq * ((qr.log() - (lr - lse)).abs() + 2)) + 40 * U * loss.abs()
    first = torch.zeros_like(entry)
    first[torch.arange(T, device=z.device), torch.where(entry, z.gather(1, i), -math.inf).argmax(1)] = True
    sums = EX2 + (k / 32 + 64) * U
    t_delta = 2 * tz[:, None] * p * (1 - p) + q * (1 - q) * 2 * tq[:, None] + eq[:, None] * first + sums * torch.where(first, (1 - p) + (1 - q), p + q)
    # what 64 bits leave of p - q here: exponents that are differences of numbers as large as lse, the products' sums
    own = 2.0 ** -52 * (8 * (lse.abs() + mass.abs().nan_to_num(0, 0, 0) + 1) + 4 * tz / U)
    t_delta = t_delta + own[:, None] * (p + q)
    t_rest = 2 * tz * pr * (1 - pr) + 2 * eq + sums * (pr + qr) + own * (pr + qr)
    out = dict(loss=zero(loss), delta=torch.where(entry & live[:, None], p - q, 0.0), rest=zero(pr - qr), rest_lse=zero(lr), lse=zero(lse),
               t_loss=t_loss, t_delta=t_delta, t_rest=t_rest, t_rest_lse=tr, t_lse=tl)
    if g is None:
        return out
    eps = EPS[hidden.dtype]
    gd = zero(g.double())
    dense = torch.where(inside, -math.inf, z - lr[:, None]).exp().nan_to_num(0.0)  # of the others
    dz = (pr - qr)[:, None] * dense
    ez = dense * (t_rest + (pr - qr).abs() * (tz + tr + EX2 + 8 * U * lr.abs().nan_to_num(0, 0, 0)))[:, None]
    dz[r, ids[r, c].long()] = (p - q)[r, c]
    ez[r, ids[r, c].long()] = t_delta[r, c]
    dz, ez = dz.nan_to_num(0.0) * gd[:, None], ez.nan_to_num(0.0) * gd.abs()[:, None]
    tiny = TINY[hidden.dtype] * gd.abs().amax() * 2.0 ** -12
    ez = ez + (eps + 4 * U) * dz.abs() + torch.where(gd.abs()[:, None] > 0, tiny, 0.0)
    for name, a, b, ea in (("d_hidden", dz, w, ez), ("d_weight", dz.t(), h, ez.t())):
        n = a.shape[1]
        part = scale * (ea @ b.abs()) + (2 * n / 16 + 32) * U * scale * (a.abs() @ b.abs())
        out[name] = scale * (a @ b)
        out["t_" + name] = part * (1 + eps) + eps * out[name].abs() + TINY[hidden.dtype]
    return out


def near(got, want, tol, what):
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine], want[~fine]), (what, "infinities")
    err = (got - want)[fine].abs()
    tol = tol.expand_as(want)[fine]
    bad = ~(err <= tol)
    assert not bad.any(), (what, float(err[bad].max()), float(tol[bad].min()), int(bad.sum()), float((err / tol.clamp(min=1e-300)).max()))
