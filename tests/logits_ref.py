"""The adjusted logits' formulas in 64 bits (include/graphpo.h), with bounds of what the kernel's roundings can make of
them, and inputs for their tests."""
import math

import torch

from vocab_ref import EPS, TINY, U

LOG2E = 1.4426950408889634


def inputs(R, V, dtype, seed=0, pad=0, history=60, penalties=True, biases=0, masks=0, temperature=False, ids=torch.int32,
           target=True, masked=0.0, device="cuda"):
    """(logits, target, arguments of logits_adjust): rows of a view `pad` elements wider filled with NaN, histories with
    tokens often repeated and ids below 0, lists of biases that rows share, masks with words of all and of no bits, and one mask
    of nothing; logits that the masks leave out are NaN or infinite."""
    g = torch.Generator(device=device)
    g.manual_seed(77 + seed)
    rand = lambda *s: torch.rand(*s, generator=g, device=device)  # noqa: E731
    z = torch.randn(R, V, generator=g, device=device) * 3.0
    y = torch.randint(0, V, (R,), generator=g, device=device)
    z[torch.arange(R, device=device), y] += 14.0 * rand(R)
    how = dict(scale=1.0, repetition=1.0, presence=0.0, frequency=0.0)
    if history:
        n = (rand(R, 2) * (history + 1)).long() * (rand(R, 1) < 0.9)
        end = torch.cumsum(n.sum(1), 0)
        how["spans"] = torch.stack([end - n.sum(1), end - n[:, 1], end], 1).contiguous()
        u = rand(max(1, int(end[-1])))
        tokens = (V * u ** 4).long().clamp(max=V - 1)
        how["history"] = torch.where(rand(len(tokens)) < 0.05, -1 - tokens, tokens).to(ids)
    if penalties:
        pick = lambda *v: torch.tensor(v, device=device)[torch.randint(0, len(v), (R,), generator=g, device=device)]  # noqa: E731
        how.update(repetition=pick(1.0, 1.3, 0.8), presence=pick(0.0, 0.4, -0.3), frequency=pick(0.0, 0.15))
    if temperature:
        how["scale"] = 0.5 + rand(R)
    if biases:
        k = min(biases, V)
        lists = [torch.sort(torch.randperm(V, generator=g, device=device)[:max(1, k - i)]).values for i in range(3)]
        start = torch.tensor([0] + [len(x) for x in lists], device=device).cumsum(0)
        which = torch.randint(0, 4, (R,), generator=g, device=device)
        none = which == 3
        which = which.clamp(max=2)
        how.update(bias_ids=torch.cat(lists).to(ids), bias=torch.randn(int(start[-1]), generator=g, device=device) * 2,
                   bias_spans=torch.stack([start[which], torch.where(none, start[which], start[which + 1])], 1).contiguous())
    keep = rand(R) >= masked
    if masks:
        W = (V + 31) // 32
        bits = rand(masks, W, 32) < torch.linspace(0.05, 0.9, masks, device=device)[:, None, None]
        bits[:, ::3] = True
        bits[:, 1::7] = False
        if masks > 1:
            bits[-1] = False
        how["mask_row"] = torch.randint(-1, masks, (R,), generator=g, device=device).to(torch.int32)
        how["mask"] = (bits.long() << torch.arange(32, device=device)).sum(2).to(torch.int32)
        out = ~bits.view(masks, -1)[:, :V][how["mask_row"].clamp(min=0).long()] & (how["mask_row"] >= 0)[:, None]
        bad = torch.tensor([math.nan, math.inf, -math.inf, 3e38], device=device)
        z = torch.where(out, bad[torch.arange(V, device=device) % 4], z)
    z[~keep] = math.nan
    wide = torch.full((R, V + pad), math.nan, dtype=dtype, device=device)
    wide[:, pad // 2:pad // 2 + V] = z
    return wide[:, pad // 2:pad // 2 + V], torch.where(keep, y, -1 - y).to(ids) if target else None, how


def exact(logits, target, how, g=None, e=None):
    """Results in 64 bits with bounds t_*: of each row the adjusted logits, lse, logp, entropy, and with g (and e) d_logits.

    An adjusted logit takes at most 8 roundings of what it is summed from.  A thread adds up V / 384 + 40 terms at most, each of an exponential good to 2^-21 and an exponent that is a difference of two rounded numbers; the
    joins add less than 64 roundings."""
    R, V = logits.shape
    of = lambda name, r: float(how[name][r]) if isinstance(how[name], torch.Tensor) else float(how[name])  # noqa: E731
    res = {k: [] for k in ("logits", "t_logits", "lse", "t_lse", "logp", "t_logp", "entropy", "t_entropy", "d_logits", "t_d_logits")}
    small, eps = TINY.get(logits.dtype, 0.0), EPS.get(logits.dtype, U)
    for r in range(R):
        z = logits[r].double()
        whole = torch.zeros(V, dtype=torch.bool, device=z.device)
        made = torch.zeros(V, dtype=torch.float64, device=z.device)
        if how.get("spans") is not None:
            b, m, n = (int(x) for x in how["spans"][r])
            h = how["history"][b:n].long()
            whole[h[h >= 0]] = True
            h = how["history"][m:n].long()
            made.index_put_((h[h >= 0],), torch.ones((), dtype=torch.float64, device=z.device), accumulate=True)
        th = of("repetition", r)
        slope = torch.where(whole, torch.where(z > 0, 1 / th, th), 1.0)
        minus = of("frequency", r) * made + of("presence", r) * (made > 0)
        plus = torch.zeros_like(z)
        if how.get("bias") is not None:
            b, n = (int(x) for x in how["bias_spans"][r]) if how.get("bias_spans") is not None else (0, len(how["bias"]))
            plus[how["bias_ids"][b:n].long()] = how["bias"][b:n].double()
        s = of("scale", r)
        y = s * (z * slope - minus + plus)
        m = 0 if how.get("mask") is None else int(how["mask_row"][r]) if how.get("mask_row") is not None else min(r, how["mask"].shape[0] - 1)
        allowed = torch.ones_like(whole)
        if how.get("mask") is not None and m >= 0:
            v = torch.arange(V, device=z.device)
            allowed = (how["mask"][m][v >> 5].long() >> (v & 31)) & 1 > 0
        y = torch.where(allowed, y, -math.inf)
        ty = 8 * U * s * ((z * slope).abs() + minus.abs() + plus.abs())
        res["logits"].append(y)
        res["t_logits"].append(torch.where(allowed, ty, 0.0))
        t = -1 if target is None else int(target[r])
        stats = target is None or t >= 0
        left = ~(y <= -7e27)
        lse = torch.logsumexp(torch.where(left, y, -math.inf), 0)
        logq = torch.where(left, y - lse, -math.inf)
        p = torch.where(left, logq.exp(), 0.0)
        h = -torch.where(p == 0, 0.0, p * logq).sum()
        # the error of the sum of exponentials, of itself
        near = left & (logq > -40)
        top = float(y[left].max().abs()) * LOG2E if left.any() else 0.0
        dy = float(torch.where(near, ty, 0.0).max()) if near.any() else 0.0
        rel = U * (V / 384 + 104) + 2.0 ** -21 + 4 * U * (top + 40) + 2 * dy
        tl = rel + 4 * U * (abs(float(lse)) + 1) if left.any() else 0.0
        te = 8 * (rel + 4 * U * top) * (1 + float(h) + float((p * torch.where(p > 0, logq.abs(), 0.0)).sum())) + 32 * U
        zero = torch.zeros((), dtype=torch.float64, device=z.device)
        res["lse"].append(lse if stats else zero)
        res["t_lse"].append(zero + (tl if stats else 0.0))
        res["entropy"].append(h if stats else zero)
        res["t_entropy"].append(zero + (te if stats else 0.0))
        if t < 0:
            res["logp"].append(zero)
            res["t_logp"].append(zero)
        else:
            lp = logq[t]
            first = bool(left[t]) and float(y[t]) >= float(y[left].max())
            tp = 2 * rel * abs(float(lp)) + small if first else 2 * rel * (1 + abs(float(lp))) + 4 * U * abs(float(lse)) if bool(left[t]) else 0.0
            res["logp"].append(lp)
            res["t_logp"].append(zero + tp)
        if g is not None:
            if t < 0 or not left.any():
                res["d_logits"].append(torch.zeros_like(z))
                res["t_d_logits"].append(torch.zeros_like(z))
                continue
            gd, ed = float(g[r]), 0.0 if e is None else float(e[r])
            one = torch.zeros_like(z)
            one[t] = 1.0
            f = torch.where(p > 0, p * (logq + h), 0.0)
            d = gd * (one - p) - ed * f
            rp = rel + tl + 4 * U * (torch.where(left, y.abs(), 0.0) + abs(float(lse)))
            td = abs(gd) * p * rp + abs(ed) * (f.abs() * (rp + 8 * U) + p * (tl + te + 8 * U * (h + torch.where(left, logq.abs(), 0.0))))
            td = td + abs(ed) * 2.0 ** -126 * 200
            if bool(left[t]):  # (by logp: 1 - p has its digits)
                td[t] = abs(gd) * (float(p[t]) * tp + 8 * U * abs(float(torch.expm1(lp)))) + abs(ed) * float(p[t]) * (
                    abs(float(lp) + float(h)) * (tp + 8 * U) + tp + te + 4 * U * (abs(float(lp)) + float(h)))
            by = torch.where(allowed, s * slope, 0.0)
            d = torch.where(allowed, d * by, 0.0)
            res["d_logits"].append(d)
            res["t_d_logits"].append(torch.where(allowed, td * by.abs() * (1 + 8 * eps) + (eps + 8 * U) * d.abs() + small, 0.0))
    return {k: torch.stack(v) for k, v in res.items() if v}


def near(got, want, tol, what):
    """got equals want to tol; infinities and NaN in the same places."""
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), (what, "NaN")
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), (what, "infinities")
    assert bool(torch.isfinite(got[fine]).all()), (what, "not finite")
    err = (got - want)[fine].abs()
    bad = ~(err <= tol.expand_as(want)[fine])
    assert not bad.any(), (what, float(err[bad].max()), float(tol.expand_as(want)[fine][bad].min()), int(bad.sum()))
