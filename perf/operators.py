"""The vocabulary ends of a policy model as measurable cases.

What a GraphPO trainer does around the advantages and the policy loss: log-probabilities of the
sampled tokens from hidden states and the vocabulary matrix (and the entropy of Algorithm S.1's
bonus), the gradients of both from the loss's gradient, the embedding lookup of the tokens and the
gradient of its table.  Kinds of case (`op`):

  logp        log-probability, log-sum-exp (and entropy) of every token
  grad        gradients of the hidden states and the vocabulary matrix
  embed       rows of the table by token id, scaled
  embed_grad  gradient of the table

Token ids follow a Zipf law over a random order of the vocabulary.  Hidden states lean towards the
row of their target by a random amount, so that some tokens are nearly certain and some are not, as
a trained policy's are.  Tokens without a target (prompts, tool output, padding; target -1) have
undefined hidden states, every other one NaN here.  Where `pad` is set, rows are views of a wider
buffer.
"""
import math

import numpy as np
import torch

own = False

_DEVICE = "cuda"
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def _case(name, op, tokens, vocab, d, dtype="bf16", **kw):
    c = dict(name=name, op=op, tokens=tokens, vocab=vocab, d=d, dtype=dtype, pad=False, masked=0.0, entropy=False, scale=1.0)
    c.update(kw)
    return c


def listed():
    return [
        # one sequence being decoded: the log-probability of one sampled token, every weight read once
        _case("logp_one_token", "logp", 1, 131072, 4096),
        # a debugging run's last layer: bound by launches and latency
        _case("logp_small", "logp", 7, 1009, 256, "f16", entropy=True),
        # one step of a group's rollouts scored together at a sampling temperature, an odd vocabulary
        _case("logp_step", "logp", 250, 50021, 1024, "f16", entropy=True, scale=1.25),
        # a training micro-batch with its prompts masked, for the entropy bonus
        _case("logp_train", "logp", 4096, 100003, 2048, masked=0.3, entropy=True, pad=True),
        # old and reference log-probabilities of a long batch
        _case("logp_long", "logp", 8192, 131072, 2048),
        # the gradient of a debugging run
        _case("grad_small", "grad", 300, 8191, 512, "f16"),
        # a micro-batch's gradient: masked prompts, clipped tokens, the entropy bonus
        _case("grad_train", "grad", 2048, 65536, 2048, masked=0.3, entropy=True),
        # the largest: a wide model's micro-batch, every token trained on
        _case("grad_wide", "grad", 4096, 131072, 4096),
        # the tokens of 16 sequences being decoded
        _case("embed_step", "embed", 16, 131072, 4096),
        # a training batch's tokens
        _case("embed_train", "embed", 32768, 131072, 4096, scale=64.0),
        # a debugging run's table in fp32
        _case("embed_grad_small", "embed_grad", 1000, 8191, 512, "f32"),
        # a training batch's table: frequent tokens in thousands of places, most rows without any
        _case("embed_grad_train", "embed_grad", 32768, 131072, 4096),
    ]


def _spread(rng, lo, hi, step=1):
    """A size between lo and hi, its logarithm uniform, rounded up to a multiple of `step`."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = min(hi, max(lo, -(-n // step) * step))
    return n if n != 3072 else n + step


def draw(rng):
    op = rng.choice(["logp", "logp", "grad", "grad", "embed", "embed_grad"])
    head = op in ("logp", "grad")
    vocab = _spread(rng, 1000, 131072)
    d = _spread(rng, 128, 4096, 8 if rng.random() < 0.7 else 1)
    if op == "logp":
        tokens = 1 if rng.random() < 0.2 else _spread(rng, 1, 8192)
        while tokens * vocab * d > 8192 * 131072 * 2048:
            tokens = (tokens + 1) // 2
    elif op == "grad":
        tokens = _spread(rng, 16, 4096)
    else:
        tokens = _spread(rng, 1, 32768)
    return dict(op=op, tokens=tokens, vocab=vocab, d=d, dtype=rng.choice(["bf16", "f16"] if head else ["bf16", "f16", "f32"]),
                pad=d % 8 != 0 or rng.random() < 0.25, masked=rng.choice([0.0, 0.0, 0.3, 0.6]) if tokens >= 32 else 0.0, entropy=head and rng.random() < 0.4,
                scale=rng.choice([1.0, 1.25, 0.7]) if head else rng.choice([1.0, round(math.sqrt(d), 3)]))


def _zipf(vocab):
    w = 1.0 / (np.arange(vocab, dtype=np.float64) + 2.7)
    return w / w.sum()


def _ids(gen, tokens, vocab, masked):
    cdf = torch.from_numpy(np.cumsum(_zipf(vocab))).to(_DEVICE)
    u = torch.rand(tokens, generator=gen, device=_DEVICE, dtype=torch.float64)
    order = torch.randperm(vocab, generator=gen, device=_DEVICE)
    ids = order[torch.searchsorted(cdf, u).clamp_(max=vocab - 1)]
    if masked > 0.0:
        ids = torch.where(torch.rand(tokens, generator=gen, device=_DEVICE) < masked, -1, ids)
    return ids.to(torch.int32)


def _rows(values, dtype, pad):
    """`values` in the given type; with `pad` as a view of a wider buffer whose rows start on 16 bytes."""
    n, d = values.shape
    if not pad:
        return values.to(dtype)
    wide = torch.zeros(n, (d + 7) // 8 * 8 + 16, dtype=dtype, device=values.device)
    wide[:, :d] = values
    return wide[:, :d]


def prepare(case, seed):
    gen = torch.Generator(device=_DEVICE)
    gen.manual_seed(0x6E5D + 1000003 * seed)
    T, V, D, dtype = case["tokens"], case["vocab"], case["d"], _TYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=_DEVICE)  # noqa: E731
    s = dict(case=dict(case), ids=_ids(gen, T, V, case["masked"]), scale=float(case["scale"]))
    if case["op"] == "embed":
        s["table"] = _rows(normal(V, D), dtype, case["pad"])
        return s
    if case["op"] == "embed_grad":
        s["grad"] = _rows(normal(T, D) / 8.0, dtype, case["pad"])
        return s
    weight = normal(V, D).mul_(2.0 / math.sqrt(D) / s["scale"])
    keep = s["ids"] >= 0
    row = weight[s["ids"].clamp(min=0).long()]
    lean = torch.rand(T, 1, generator=gen, device=_DEVICE) * 18.0 / s["scale"]
    hidden = normal(T, D) + row * (lean / row.square().sum(1, keepdim=True))
    hidden[~keep & (torch.arange(T, device=_DEVICE) % 2 == 0)] = math.nan
    s["hidden"], s["weight"] = _rows(hidden, dtype, case["pad"]), _rows(weight, dtype, case["pad"])
    if case["op"] == "grad":
        # the forward pass's results, and the loss's gradient: a quarter of the tokens clipped, fp16 with its loss scale
        s["lse"], _, s["entropy"] = _plain_logp(s["hidden"], s["weight"], s["ids"], s["scale"])
        to = 1024.0 if case["dtype"] == "f16" else 1.0
        live = keep & (torch.rand(T, generator=gen, device=_DEVICE) >= 0.25)
        s["grad_logp"] = torch.where(live, normal(T) * (to / T), 0.0)
        s["grad_entropy"] = torch.where(keep, torch.full((T,), -0.01 * to / T, device=_DEVICE), 0.0) if case["entropy"] else None
    return s


def _logits(hidden, weight, ids, scale):
    """Scaled logits in 32 bits (0 for tokens without a target), with the operands that made them."""
    h = torch.where((ids >= 0)[:, None], hidden, 0.0).float()
    w = weight.float()
    return scale * (h @ w.t()), h, w


def _plain_logp(hidden, weight, ids, scale):
    """lse, logp and entropy in 32 bits, 0 for tokens without a target.  The target's logit and the sum over the
    others are kept apart, so that a nearly certain token's log-probability, a sum of small terms, keeps its digits."""
    z = _logits(hidden, weight, ids, scale)[0]
    keep = ids >= 0
    y = ids.clamp(min=0).long()[:, None]
    at = z.gather(1, y)[:, 0]
    z = z.scatter(1, y, -math.inf)
    most = z.amax(1)
    z = z - most[:, None]
    p = torch.exp(z)
    s = p.sum(1)
    u = torch.where(p > 0.0, p * z, 0.0).sum(1)
    top = torch.maximum(most, at)
    a, c = at - top, most - top
    others = torch.exp(c) * s
    total = others + torch.exp(a)
    log_total = torch.where(a == 0.0, torch.log1p(others), torch.log(total))
    entropy = log_total - (torch.exp(c) * (u + c * s) + torch.exp(a) * a) / total
    return torch.where(keep, top + log_total, 0.0), torch.where(keep, a - log_total, 0.0), torch.where(keep, entropy, 0.0)


def _plain_grad(s):
    z, h, w = _logits(s["hidden"], s["weight"], s["ids"], s["scale"])
    keep = s["ids"] >= 0
    z = z - s["lse"][:, None]
    p = torch.exp(z)
    g = torch.where(keep, s["grad_logp"], 0.0)
    dz = -g[:, None] * p
    if s["grad_entropy"] is not None:
        e = torch.where(keep, s["grad_entropy"], 0.0)
        dz = dz - e[:, None] * p * (z + s["entropy"][:, None])
    at = torch.arange(dz.shape[0], device=dz.device)
    dz[at, s["ids"].clamp(min=0).long()] += g
    dz = dz * s["scale"]
    return {"d_hidden": (dz @ w).to(s["hidden"].dtype), "d_weight": (dz.t() @ h).to(s["weight"].dtype)}


_gp = None


def _framework():
    global _gp
    if _gp is None:
        import paper_2606_18954_gb300 as P
        _gp = P.GraphPO()
    return _gp


def run(s):
    case = s["case"]
    op, ids = case["op"], s["ids"]
    if own:
        gp = _framework()
        if op == "logp":
            return gp.vocab_logp(s["hidden"], s["weight"], ids, scale=s["scale"], entropy=case["entropy"])
        if op == "grad":
            return gp.vocab_grad(s["hidden"], s["weight"], ids, s["lse"], s["grad_logp"], scale=s["scale"],
                                 entropy=s["entropy"] if case["entropy"] else None, grad_entropy=s["grad_entropy"])
        if op == "embed":
            return gp.embed(s["table"], ids, scale=s["scale"])
        return gp.embed_grad(s["grad"], ids, case["vocab"], scale=s["scale"])
    if op == "logp":
        lse, logp, entropy = _plain_logp(s["hidden"], s["weight"], ids, s["scale"])
        return {"logp": logp, "lse": lse, "entropy": entropy} if case["entropy"] else {"logp": logp, "lse": lse}
    if op == "grad":
        return _plain_grad(s)
    if op == "embed":
        x = s["table"][ids.clamp(min=0).long()].float() * s["scale"]
        return torch.where((ids >= 0)[:, None], x, 0.0).to(s["table"].dtype)
    g = torch.where((ids >= 0)[:, None], s["grad"].float(), 0.0)
    table = torch.zeros(case["vocab"], g.shape[1], device=g.device)
    table.index_add_(0, ids.clamp(min=0).long(), g)
    return (table * s["scale"]).to(s["grad"].dtype)


def work(case):
    T, V, D, e = case["tokens"], case["vocab"], case["d"], _SIZE[case["dtype"]]
    live = T * (1.0 - case["masked"])
    if case["op"] == "logp":
        return {"bytes": (live + V) * D * e + T * (12 + 4 * case["entropy"]), "flops": 2.0 * live * V * D}
    if case["op"] == "grad":
        if not case["entropy"]:
            live *= 0.75  # clipped tokens have no gradient
        return {"bytes": (live + T + 2 * V) * D * e + T * (12 + 8 * case["entropy"]), "flops": 6.0 * live * V * D}
    distinct = float((1.0 - (1.0 - _zipf(V)) ** live).sum())
    if case["op"] == "embed":
        return {"bytes": (distinct + T) * D * e + 4.0 * T, "flops": float(T * D)}
    return {"bytes": (live + V) * D * e + 4.0 * T, "flops": live * D}


def exact(case, seed):
    s = prepare(case, seed)
    ids = s["ids"].long()
    rows = torch.nonzero(ids >= 0)[:, 0]
    y, T, V, D = ids[rows], case["tokens"], case["vocab"], case["d"]

    def whole(part, *shape):
        out = torch.zeros(T, *shape, dtype=torch.float64, device=_DEVICE)
        out[rows] = part
        return out

    if case["op"] == "embed":
        return whole(s["table"].double()[y] * s["scale"], D)
    if case["op"] == "embed_grad":
        out = torch.zeros(V, D, dtype=torch.float64, device=_DEVICE)
        out.index_put_((y,), s["grad"][rows].double() * s["scale"], accumulate=True)
        return out
    w = s["weight"].double()
    h = s["hidden"][rows].double()
    names = ("logp", "lse", "entropy")
    got = {n: [] for n in names}
    dh, dw = [], torch.zeros(V, D, dtype=torch.float64, device=_DEVICE) if case["op"] == "grad" else None
    for a in range(0, len(rows), 1024):
        b = min(a + 1024, len(rows))
        z = torch.mm(h[a:b], w.t()) * s["scale"]
        logq = torch.log_softmax(z, dim=1)
        q = logq.exp()
        ent = -(q * logq).sum(1)
        pick = torch.arange(b - a, device=_DEVICE)
        if case["op"] == "logp":
            got["logp"].append(logq[pick, y[a:b]])
            got["lse"].append(torch.logsumexp(z, dim=1))
            got["entropy"].append(ent)
            continue
        g = s["grad_logp"][rows[a:b]].double()
        one = torch.zeros_like(q)
        one[pick, y[a:b]] = 1.0
        d = g[:, None] * (one - q)
        if case["entropy"]:
            d -= s["grad_entropy"][rows[a:b]].double()[:, None] * q * (logq + ent[:, None])
        dh.append(torch.mm(d, w) * s["scale"])
        dw += torch.mm(d.t(), h[a:b]) * s["scale"]
    if case["op"] == "logp":
        return {n: whole(torch.cat(got[n]) if got[n] else 0.0) for n in names if n != "entropy" or case["entropy"]}
    return {"d_hidden": whole(torch.cat(dh) if dh else 0.0, D), "d_weight": dw}
