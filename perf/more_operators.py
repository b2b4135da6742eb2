"""What shapes a policy's distribution over its vocabulary, as measurable cases.

When a rollout is sampled, the sampler's logits are adjusted before a token is drawn: penalties for tokens that the row
has had already, biases, a grammar's mask, the temperature.  The log-probabilities that the policy loss takes are those
of the adjusted distribution, and its gradient goes back through the adjustment.  When the policy learns from a teacher,
the loss is the Kullback-Leibler divergence from the teacher's top tokens to the policy's whole vocabulary.  Kinds of
case (`op`):

  adjust        logits as the sampler takes them, or only their log-probabilities, log-sum-exps and entropies
  adjust_grad   gradient of the raw logits from that of the log-probabilities (and entropies)
  distill       divergence of every token from hidden states, the vocabulary matrix and the teacher's top tokens
  distill_grad  its gradients of the hidden states and the matrix

Token ids follow a Zipf law over a random order of the vocabulary.  The teacher is the policy's matrix on other hidden
states near the policy's; its top tokens are those of its own logits.  Tokens that take no part (prompts, padding) have
no target or no teacher, and undefined hidden states or logits, every other one NaN here.  Where `pad` is set, rows are views
of a wider buffer.
"""
import math

import numpy as np
import torch

own = False

_DEVICE = "cuda"
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def _adjust(name, op, rows, vocab, dtype="bf16", **kw):
    """rows of logits; prompt and generated: the most tokens of a row's history; rollouts: 0 for rows with histories of their
    own, else the rows are the positions of so many rollouts; write: "f32" or "same" (the logits' type) for a sampler, that gets
    the adjusted logits, "" for a trainer, that has the sampled tokens and gets their log-probabilities; grammars: masks that the
    rows share; biases: entries of each list (one for every four rows)"""
    c = dict(name=name, op=op, rows=rows, vocab=vocab, dtype=dtype, pad=False, prompt=0, generated=0, rollouts=0, penalties=False, grammars=0, biases=0,
             temperature=False, write="", entropy=False, masked=0.0)
    c.update(kw)
    return c


def _distill(name, op, tokens, vocab, d, k, dtype="bf16", **kw):
    """k: the teacher's top tokens; tail: their log-probabilities, with the rest of the vocabulary as one more outcome"""
    c = dict(name=name, op=op, tokens=tokens, vocab=vocab, d=d, k=k, dtype=dtype, pad=False, masked=0.0, short=False, tail=False, scale=1.0, teacher="f32")
    c.update(kw)
    return c


def listed():
    return [
        # one sequence being decoded under a grammar: bound by latency
        _adjust("adjust_one", "adjust", 1, 131072, prompt=3000, generated=2000, penalties=True, grammars=1, write="same"),
        # a server's step over requests with penalties, biases and temperatures of their own, an odd vocabulary
        _adjust("adjust_odd", "adjust", 33, 50021, "f16", pad=True, prompt=1500, generated=700, penalties=True, biases=300, temperature=True, write="f32"),
        # a step of a batch of rollouts: penalties, a few grammars, the log-sum-exp and entropy of what is sampled from
        _adjust("adjust_step", "adjust", 256, 131072, prompt=6000, generated=2000, penalties=True, grammars=8, temperature=True, write="same", entropy=True),
        # a training micro-batch's log-probabilities under what the sampler had applied, from its logits
        _adjust("adjust_score", "adjust", 4096, 65536, prompt=800, generated=1024, rollouts=4, penalties=True, grammars=4, entropy=True, masked=0.3),
        # the gradient of a server's step that is trained on online
        _adjust("adjust_grad_step", "adjust_grad", 250, 50021, "f16", pad=True, prompt=1500, generated=700, penalties=True, biases=64, temperature=True),
        # the training micro-batch's gradient, with the entropy bonus
        _adjust("adjust_grad_train", "adjust_grad", 4096, 65536, prompt=800, generated=1024, rollouts=4, penalties=True, grammars=4, entropy=True, masked=0.3),
        # a debugging run: bound by launches and latency
        _distill("distill_small", "distill", 60, 8191, 512, 8, "f16", teacher="f16"),
        # a micro-batch with its prompts masked, a teacher's log-probabilities cut where its nucleus ends
        _distill("distill_train", "distill", 2048, 65536, 2048, 32, masked=0.3, short=True, tail=True),
        # a long batch from stored top logits
        _distill("distill_long", "distill", 8192, 131072, 2048, 64, teacher="bf16"),
        # the gradient of a debugging run
        _distill("distill_grad_small", "distill_grad", 300, 8191, 512, 16, "f16", scale=1.25),
        # the micro-batch's gradient
        _distill("distill_grad_train", "distill_grad", 2048, 65536, 2048, 32, masked=0.3, short=True, tail=True),
        # the largest: a wide model's micro-batch, every token with a teacher
        _distill("distill_grad_wide", "distill_grad", 4096, 131072, 4096, 64),
    ]


def _spread(rng, lo, hi, step=1):
    """A size between lo and hi, its logarithm uniform, rounded up to a multiple of `step`."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(hi, max(lo, -(-n // step) * step))


def draw(rng):
    op = rng.choice(["adjust", "adjust", "adjust_grad", "distill", "distill", "distill_grad"])
    vocab = _spread(rng, 1000, 131072)
    if op in ("adjust", "adjust_grad"):
        rows = 1 if rng.random() < 0.15 else _spread(rng, 1, 4096)
        while rows * vocab > 4096 * 65536:
            rows = (rows + 1) // 2
        train = op == "adjust_grad" or rng.random() < 0.5
        several = train and rows >= 64 and rng.random() < 0.7
        return dict(op=op, rows=rows, vocab=vocab, dtype=rng.choice(["bf16", "f16", "f32"]), pad=rng.random() < 0.4, prompt=rng.choice([0, _spread(rng, 1, 6000 if rows <= 512 else 800)]),
                    generated=_spread(rng, 1, 2000 if rows <= 512 else 1024), rollouts=rng.choice([1, 3, 8]) if several else 0, penalties=rng.random() < 0.8,
                    grammars=rng.choice([0, 1, 5]), biases=rng.choice([0, 0, 1, 300]), temperature=rng.random() < 0.5,
                    write="" if train else rng.choice(["same", "f32"]), entropy=rng.random() < 0.4, masked=rng.choice([0.0, 0.3, 0.6]) if several else 0.0)
    d = _spread(rng, 128, 4096, 8 if rng.random() < 0.7 else 1)
    tokens = 1 if rng.random() < 0.1 else _spread(rng, 1, 8192 if op == "distill" else 4096)
    while tokens * vocab * d > 8192 * 131072 * 2048:
        tokens = (tokens + 1) // 2
    k = _spread(rng, 1, 256)
    while tokens * k > 8192 * 64:
        k = (k + 1) // 2
    return dict(op=op, tokens=tokens, vocab=vocab, d=d, k=k, dtype=rng.choice(["bf16", "f16"]), pad=d % 8 != 0 or rng.random() < 0.25,
                masked=rng.choice([0.0, 0.0, 0.3, 0.6]) if tokens >= 32 else 0.0, short=rng.random() < 0.4, tail=rng.random() < 0.5, scale=rng.choice([1.0, 1.25, 0.7]),
                teacher=rng.choice(["f32", "bf16", "f16"]))


# ---------------------------------------------------------------------------- inputs


def _zipf(vocab):
    w = 1.0 / (np.arange(vocab, dtype=np.float64) + 2.7)
    return w / w.sum()


def _ids(gen, n, vocab, order):
    cdf = torch.from_numpy(np.cumsum(_zipf(vocab))).to(_DEVICE)
    u = torch.rand(n, generator=gen, device=_DEVICE, dtype=torch.float64)
    return order[torch.searchsorted(cdf, u).clamp_(max=vocab - 1)]


def _rows(values, dtype, pad, unit):
    """`values` in the given type; with `pad` as a view of a wider buffer whose rows are `unit` elements more, or as many as make
    whole 16 bytes."""
    n, d = values.shape
    if not pad:
        return values.to(dtype)
    wide = torch.zeros(n, d + 1 if unit == 1 else (d + 7) // 8 * 8 + 16, dtype=dtype, device=values.device)
    wide[:, :d] = values
    return wide[:, :d]


def _prepare_adjust(case, gen, s):
    R, V, dtype = case["rows"], case["vocab"], _TYPES[case["dtype"]]
    rand = lambda *n: torch.rand(*n, generator=gen, device=_DEVICE)  # noqa: E731
    whole = lambda n, lo, hi: torch.randint(lo, hi + 1, (n,), generator=gen, device=_DEVICE)  # noqa: E731
    order = torch.randperm(V, generator=gen, device=_DEVICE)
    # frequent tokens have higher logits, and one token of most rows stands out
    z = torch.randn(R, V, generator=gen, device=_DEVICE).mul_(2.0)
    z[:, order] -= 0.7 * torch.log(torch.arange(V, device=_DEVICE) + 2.7)
    sampled = _ids(gen, R, V, order)
    z[torch.arange(R, device=_DEVICE), sampled] += 16.0 * rand(R)
    # histories: (begin, first generated, end) of each row in one array of tokens
    if case["rollouts"]:
        n = case["rollouts"]
        first = torch.arange(R, device=_DEVICE) * n // R
        start = torch.arange(R, device=_DEVICE) - torch.searchsorted(first, first)
        seq = case["prompt"] + int(start.max()) + 1
        begin = first * seq
        gens = start % max(1, case["generated"])
        spans = torch.stack([begin, begin + case["prompt"], begin + case["prompt"] + gens], 1)
        tokens = n * seq
    else:
        p = whole(R, 0, case["prompt"]) if R > 1 else torch.full((R,), case["prompt"], device=_DEVICE)
        g = whole(R, 0, case["generated"]) if R > 1 else torch.full((R,), case["generated"], device=_DEVICE)
        end = torch.cumsum(p + g, 0)
        spans = torch.stack([end - p - g, end - g, end], 1)
        tokens = int(end[-1])
    s["history"] = _ids(gen, max(1, tokens), V, order).to(torch.int32)
    s["spans"] = spans.contiguous()
    s["pairs"] = int((spans[:, 2] - spans[:, 0]).sum())
    pick = lambda *v: torch.tensor(v, device=_DEVICE)[whole(R, 0, len(v) - 1)]  # noqa: E731
    s["repetition"] = pick(1.0, 1.1, 1.3) if case["penalties"] else 1.0
    s["presence"] = pick(0.0, 0.2, 0.7) if case["penalties"] else 0.0
    s["frequency"] = pick(0.0, 0.1, 0.3) if case["penalties"] else 0.0
    s["scale"] = pick(1.0, 1.25, 0.7) if case["temperature"] else 1.0
    s["mask"] = s["mask_row"] = None
    if case["grammars"]:
        # every mask allows a share of the vocabulary between a hundredth and nearly all, and what its rows have sampled; the
        # last of several allows nothing, and is one row's
        M, W = case["grammars"], (V + 31) // 32
        s["mask_row"] = whole(R, -1 if R > 1 else 0, max(0, M - 2)).to(torch.int32)
        allows = rand(M, 32 * W) < torch.linspace(0.01, 0.95, M, device=_DEVICE)[:, None]
        has = s["mask_row"] >= 0
        allows[s["mask_row"][has].long(), sampled[has]] = True
        if M > 1 and R > 1:
            allows[-1] = False
            s["mask_row"][-1] = M - 1
        s["mask"] = (allows.view(M, W, 32).long() << torch.arange(32, device=_DEVICE)).sum(2).to(torch.int32)
        allowed = allows[s["mask_row"].clamp(min=0).long(), sampled] | (s["mask_row"] < 0)
    else:
        allowed = torch.ones(R, dtype=torch.bool, device=_DEVICE)
    s["bias"] = s["bias_ids"] = s["bias_spans"] = None
    if case["biases"]:
        lists, each = (R + 3) // 4, min(case["biases"], V)
        key = rand(lists, V) if lists * V <= 1 << 26 else rand(1, V).expand(lists, V)
        s["bias_ids"] = key.topk(each, dim=1).indices.sort(dim=1).values.reshape(-1).to(torch.int32)
        s["bias"] = torch.randn(lists * each, generator=gen, device=_DEVICE) * 3.0
        at = torch.arange(R, device=_DEVICE) // 4 * each
        s["bias_spans"] = torch.stack([at, at + each], 1)
    # a token that is masked, and a share of the others, takes no part
    keep = allowed & (rand(R) >= case["masked"])
    if case["masked"]:
        z[~keep & (torch.arange(R, device=_DEVICE) % 2 == 0)] = math.nan
    s["target"] = torch.where(keep, sampled, -1).to(torch.int32)
    s["logits"] = _rows(z, dtype, case["pad"], 1)
    del z
    if case["op"] == "adjust_grad":
        f = _plain_adjust(s, entropy=True)
        to = 1024.0 if case["dtype"] == "f16" else 1.0
        live = keep & (rand(R) >= (0.25 if R > 8 else 0.0))  # (a share of them clipped)
        s["lse"], s["logp"], s["entropy"] = f["lse"], f["logp"], f["entropy"]
        s["grad_logp"] = torch.where(live, torch.randn(R, generator=gen, device=_DEVICE) * (to / R), 0.0)
        s["grad_entropy"] = torch.where(keep, torch.full((R,), -0.01 * to / R, device=_DEVICE), 0.0) if case["entropy"] else None
    return s


def _prepare_distill(case, gen, s):
    T, V, D, K, dtype = case["tokens"], case["vocab"], case["d"], min(case["k"], case["vocab"]), _TYPES[case["dtype"]]
    normal = lambda *n: torch.randn(*n, generator=gen, device=_DEVICE)  # noqa: E731
    order = torch.randperm(V, generator=gen, device=_DEVICE)
    s["scale"] = float(case["scale"])
    weight = normal(V, D).mul_(2.0 / math.sqrt(D) / s["scale"])
    row = weight[_ids(gen, T, V, order)]
    lean = torch.rand(T, 1, generator=gen, device=_DEVICE) * 18.0 / s["scale"]
    hidden = normal(T, D) + row * (lean / row.square().sum(1, keepdim=True))
    taught = hidden + normal(T, D)
    keep = torch.rand(T, generator=gen, device=_DEVICE) >= case["masked"]
    ids, values = [], []
    w16 = weight.bfloat16().t()
    for a in range(0, T, 2048):
        z = (taught[a:a + 2048].bfloat16() @ w16).float() * s["scale"]
        if case["tail"]:
            z = torch.log_softmax(z, 1)
        v, i = z.topk(K, dim=1)
        ids.append(i)
        values.append(v)
    ids, values = torch.cat(ids), torch.cat(values)
    if case["short"]:  # as many as the teacher's nucleus held, one at least; what follows them is no entry
        n = torch.randint(1, K + 1, (T, 1), generator=gen, device=_DEVICE)
        off = torch.arange(K, device=_DEVICE)[None] >= n
        ids, values = torch.where(off, -1, ids), torch.where(off, math.nan, values)
    ids = torch.where(keep[:, None], ids, -1)
    hidden[~keep & (torch.arange(T, device=_DEVICE) % 2 == 0)] = math.nan
    s["ids"], s["teacher"] = ids.to(torch.int32), values.to(_TYPES[case["teacher"]])
    s["hidden"], s["weight"] = _rows(hidden, dtype, case["pad"], 8), _rows(weight, dtype, case["pad"], 8)
    if case["op"] == "distill_grad":
        f = _plain_distill(s)
        to = 1024.0 if case["dtype"] == "f16" else 1.0
        s["delta"], s["rest"], s["rest_lse"] = f["delta"], f["rest"], f["rest_lse"]
        s["grad_loss"] = torch.where(keep, (0.5 + torch.rand(T, generator=gen, device=_DEVICE)) * (to / T), 0.0)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=_DEVICE)
    gen.manual_seed(0x7A31 + 1000003 * seed)
    s = dict(case=dict(case))
    return (_prepare_adjust if case["op"] in ("adjust", "adjust_grad") else _prepare_distill)(case, gen, s)


# ---------------------------------------------------------------------------- plain forms


def _column(x):
    return x[:, None] if isinstance(x, torch.Tensor) else x


def _adjusted(s):
    """Adjusted logits in 32 bits, -inf where a mask leaves a token out, and d adjusted / d raw."""
    z = s["logits"].float()
    R, V = z.shape
    spans = s["spans"]
    n = spans[:, 2] - spans[:, 0]
    row = torch.repeat_interleave(torch.arange(R, device=z.device), n, output_size=s["pairs"])
    at = torch.arange(s["pairs"], device=z.device) - (torch.cumsum(n, 0) - n)[row] + spans[row, 0]
    tok = s["history"][at].long()
    seen = torch.zeros(R * V, device=z.device).index_add_(0, row * V + tok, torch.ones_like(tok, dtype=torch.float32)).view(R, V)
    made = torch.zeros(R * V, device=z.device).index_add_(0, row * V + tok, (at >= spans[row, 1]).float()).view(R, V)
    rep = _column(s["repetition"])
    by = torch.where(seen > 0, torch.where(z > 0, 1.0 / (rep * torch.ones_like(z)), rep * torch.ones_like(z)), 1.0)
    y = z * by - _column(s["frequency"]) * made - _column(s["presence"]) * (made > 0)
    if s["bias"] is not None:
        m = s["bias_spans"][:, 1] - s["bias_spans"][:, 0]
        each = s["bias_ids"].numel() // ((R + 3) // 4)
        at = s["bias_spans"][:, :1] + torch.arange(each, device=z.device)
        y = y.scatter_add(1, s["bias_ids"][at].long(), torch.where(torch.arange(each, device=z.device) < m[:, None], s["bias"][at], 0.0))
    y = y * _column(s["scale"])
    by = by * _column(s["scale"])
    if s["mask"] is not None:
        v = torch.arange(V, device=z.device)
        allowed = ((s["mask"][:, v >> 5] >> (v & 31)) & 1) > 0
        keep = allowed[s["mask_row"].clamp(min=0).long()] | (s["mask_row"] < 0)[:, None]
        y, by = torch.where(keep, y, -math.inf), torch.where(keep, by, 0.0)
    return y, by


def _stats(y, target):
    """lse, logp and entropy of rows of adjusted logits, 0 for rows without a target.  The target's logit and the sum over the others
    are kept apart, so that a nearly certain token's log-probability, a sum of small terms, keeps its digits.  (target None: of all rows,
    what is kept apart is the largest.)"""
    target = y.argmax(1) if target is None else target
    live = target >= 0
    t = target.clamp(min=0).long()[:, None]
    at = y.gather(1, t)[:, 0]
    z = y.scatter(1, t, -math.inf)
    most = z.amax(1)
    top = torch.maximum(most, at)
    base = torch.where(most > -math.inf, most, 0.0)
    z = z - base[:, None]
    p = torch.exp(z)
    total = p.sum(1)
    u = torch.where(p > 0.0, p * z, 0.0).sum(1)
    none = top == -math.inf
    a, c = torch.where(at > -math.inf, at - top, -math.inf), torch.where(most > -math.inf, base - top, -math.inf)
    others, one = torch.where(total > 0.0, torch.exp(c) * total, 0.0), torch.exp(a)
    log_total = torch.where(a == 0.0, torch.log1p(others), torch.log(others + one))
    entropy = log_total - (torch.where(others > 0.0, torch.exp(c) * u + others * c, 0.0) + torch.where(one > 0.0, one * a, 0.0)) / (others + one)
    zero = lambda x: torch.where(live, x, 0.0)  # noqa: E731
    return {"logp": zero(torch.where(at > -math.inf, a - log_total, -math.inf)), "lse": zero(torch.where(none, -math.inf, top + log_total)),
            "entropy": zero(torch.where(none, 0.0, entropy))}


def _plain_adjust(s, write="", entropy=False):
    y, _ = _adjusted(s)
    out = _stats(y, None if write else s["target"])
    if not entropy:
        del out["entropy"]
    if write:
        del out["logp"]
        out["logits"] = y.to(torch.float32 if write == "f32" else s["logits"].dtype)
    return out


def _plain_adjust_grad(s):
    y, by = _adjusted(s)
    live = (s["target"] >= 0) & (s["lse"] > -math.inf)
    logq = torch.where(y > -math.inf, y - s["lse"][:, None], -math.inf)
    p = torch.exp(logq)
    g = torch.where(live, s["grad_logp"], 0.0)
    dy = -g[:, None] * p
    t = s["target"].clamp(min=0).long()
    at = torch.arange(len(t), device=t.device)
    dy[at, t] = -g * torch.expm1(s["logp"])
    if s["grad_entropy"] is not None:
        e = torch.where(live, s["grad_entropy"], 0.0)
        dy = dy - e[:, None] * torch.where(p > 0.0, p * (logq + s["entropy"][:, None]), 0.0)
    return {"d_logits": torch.where(live[:, None] & (by != 0.0), dy * by, 0.0).to(s["logits"].dtype)}


def _plain_distill(s):
    """loss, delta = p - q of the teacher's entries, rest_lse = the log-sum-exp of the others, rest = their p - q."""
    ids, V = s["ids"], s["weight"].shape[0]
    entry = ids >= 0
    live = entry.any(1)
    h = torch.where(live[:, None], s["hidden"], 0.0).float()
    z = s["scale"] * (h @ s["weight"].float().t())
    i = torch.where(entry, ids, ids.amax(1, keepdim=True).clamp(min=0)).long()
    zk = torch.where(entry, z.gather(1, i), -math.inf)
    z = z.scatter_(1, i, -math.inf)
    most = z.amax(1)
    base = torch.where(most > -math.inf, most, 0.0)
    others = torch.exp(z - base[:, None]).sum(1)
    rest_lse = base + torch.log(others)
    # the teacher: of 64 bits, as 1 - sum of probabilities is a small difference of larger numbers
    t = torch.where(entry, s["teacher"].double(), -math.inf)
    t = t - (torch.logsumexp(t, 1).clamp(min=0.0) if s["case"]["tail"] else torch.logsumexp(t, 1))[:, None]
    q = torch.where(entry, torch.exp(t), 0.0)
    qr = (1.0 - q.sum(1)).clamp(min=0.0) if s["case"]["tail"] else torch.zeros_like(q[:, 0])
    a = torch.cat([zk, rest_lse[:, None]], 1).double()
    logp = a - torch.logsumexp(a, 1, keepdim=True)
    logq = torch.cat([t, torch.log(qr)[:, None]], 1)
    every = torch.exp(logq)
    loss = torch.where(every > 0.0, every * (logq - logp), 0.0).sum(1)
    delta = torch.where(entry, torch.exp(logp[:, :-1]) - q, 0.0)
    rest = torch.exp(logp[:, -1]) - qr
    zero = lambda x: torch.where(live, x, 0.0).float()  # noqa: E731
    return {"loss": zero(loss), "delta": torch.where(live[:, None], delta, 0.0).float(), "rest": zero(rest), "rest_lse": zero(rest_lse.double())}


def _plain_distill_grad(s):
    ids = s["ids"]
    entry = ids >= 0
    live = entry.any(1)
    h = torch.where(live[:, None], s["hidden"], 0.0).float()
    w = s["weight"].float()
    z = s["scale"] * (h @ w.t())
    dz = s["rest"][:, None] * torch.exp(z - s["rest_lse"][:, None])
    i = torch.where(entry, ids, ids.amax(1, keepdim=True).clamp(min=0)).long()
    first = ids.argmax(1, keepdim=True)  # (where an entry is none, the row's last id again, with its own value)
    dz = dz.scatter_(1, i, torch.where(entry, s["delta"], s["delta"].gather(1, first)))
    g = torch.where(live, s["grad_loss"], 0.0)
    dz = torch.where(live[:, None], dz * g[:, None], 0.0) * s["scale"]
    return {"d_hidden": (dz @ w).to(s["hidden"].dtype), "d_weight": (dz.t() @ h).to(s["weight"].dtype)}


# ---------------------------------------------------------------------------- one pass


_gp = None


def _framework():
    global _gp
    if _gp is None:
        import paper_2606_18954_gb300 as P
        _gp = P.GraphPO()
    return _gp


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        gp = _framework()
        if op in ("adjust", "adjust_grad"):
            how = dict(scale=s["scale"], mask=s["mask"], mask_row=s["mask_row"], history=s["history"], spans=s["spans"], repetition=s["repetition"],
                       presence=s["presence"], frequency=s["frequency"], bias=s["bias"], bias_ids=s["bias_ids"], bias_spans=s["bias_spans"])
        if op == "adjust":
            write = None if not case["write"] else torch.float32 if case["write"] == "f32" else s["logits"].dtype
            return gp.logits_adjust(s["logits"], target=None if write else s["target"], write=write, entropy=case["entropy"], **how)
        if op == "adjust_grad":
            return gp.logits_grad(s["logits"], s["target"], s["lse"], s["logp"], s["grad_logp"], entropy=s["entropy"] if case["entropy"] else None,
                                  grad_entropy=s["grad_entropy"], **how)
        if op == "distill":
            return gp.vocab_distill(s["hidden"], s["weight"], s["ids"], s["teacher"], scale=s["scale"], tail=case["tail"])
        return gp.vocab_distill_grad(s["hidden"], s["weight"], s["ids"], s["delta"], s["rest"], s["rest_lse"], s["grad_loss"], scale=s["scale"])
    if op == "adjust":
        return _plain_adjust(s, case["write"], case["entropy"])
    if op == "adjust_grad":
        return _plain_adjust_grad(s)
    if op == "distill":
        return _plain_distill(s)
    return _plain_distill_grad(s)


def work(case):
    V, e = case["vocab"], _SIZE[case["dtype"]]
    if case["op"] in ("adjust", "adjust_grad"):
        R = case["rows"]
        live = R * (1.0 - case["masked"])
        grad = case["op"] == "adjust_grad"
        # the tokens of the rollouts, or of half of every row's longest history on average
        history = case["rollouts"] * (case["prompt"] + R / max(1, case["rollouts"])) if case["rollouts"] else R * (case["prompt"] + case["generated"]) * (0.5 if R > 1 else 1.0)
        small = 4.0 * history + 24.0 * R + case["grammars"] * V / 8.0 + (8.0 * case["biases"] * ((R + 3) // 4) if case["biases"] else 0.0) + 32.0 * R
        if grad:
            return {"bytes": (live * (1.0 if case["entropy"] else 0.75) + R) * V * e + small, "flops": 12.0 * live * V}
        out = 0 if not case["write"] else 4 if case["write"] == "f32" else e
        return {"bytes": (R if out else live) * V * e + R * V * out + small, "flops": 8.0 * live * V}
    T, D, K = case["tokens"], case["d"], min(case["k"], case["vocab"])
    live = T * (1.0 - case["masked"])
    if case["op"] == "distill":
        return {"bytes": (live + V) * D * e + T * K * (8.0 + _SIZE[case["teacher"]]) + 12.0 * T, "flops": 2.0 * live * V * D}
    return {"bytes": (live + T + 2.0 * V) * D * e + T * K * 8.0 + 12.0 * T, "flops": 6.0 * live * V * D}


# ---------------------------------------------------------------------------- in 64 bits


def _exact_row(s, i, z):
    """One row's adjusted logits and their derivative with respect to z, its raw ones."""
    V = z.shape[0]
    of = lambda name: float(s[name][i]) if isinstance(s[name], torch.Tensor) else float(s[name])  # noqa: E731
    b, g, e = (int(x) for x in s["host_spans"][i])
    whole = torch.bincount(s["history"][b:e], minlength=V)
    made = torch.bincount(s["history"][g:e], minlength=V).double()
    theta = of("repetition")
    slope = torch.where(whole > 0, torch.where(z > 0, 1.0 / theta, theta), 1.0)
    y = z * slope - of("frequency") * made - of("presence") * (made > 0).double()
    if s["bias"] is not None:
        b, e = (int(x) for x in s["bias_spans"][i])
        y.index_add_(0, s["bias_ids"][b:e].long(), s["bias"][b:e].double())
    y, slope = y * of("scale"), slope * of("scale")
    m = -1 if s["mask"] is None else int(s["mask_row"][i])
    if m >= 0:
        bits = torch.bitwise_and(s["mask"][m].long()[:, None].bitwise_right_shift(torch.arange(32, device=z.device)), 1).reshape(-1)[:V]
        y[bits == 0] = -math.inf
        slope[bits == 0] = 0.0
    return y, slope


def _exact_adjust(s):
    case = s["case"]
    R, V = s["logits"].shape
    s["host_spans"] = s["spans"].cpu().numpy()
    for name in ("repetition", "presence", "frequency", "scale", "bias_spans", "mask_row", "target", "grad_logp", "grad_entropy"):
        if isinstance(s.get(name), torch.Tensor):
            s[name] = s[name].cpu()
    grad = case["op"] == "adjust_grad"
    kept = torch.empty(R, V, dtype=torch.float64, device=_DEVICE) if case["write"] else None
    d = torch.zeros(R, V, dtype=torch.float64, device=_DEVICE) if grad else None
    got = torch.zeros(R, 3, dtype=torch.float64, device=_DEVICE)
    for i in range(R):
        t = int(s["target"][i])
        if t < 0 and not case["write"]:
            continue
        y, slope = _exact_row(s, i, s["logits"][i].double())
        logq = torch.log_softmax(y, 0)
        q = logq.exp()
        h = -(torch.where(q > 0, q * logq, 0.0)).sum()
        if case["write"]:
            kept[i] = y
        if not grad:
            got[i, 0], got[i, 1], got[i, 2] = logq[max(t, 0)], torch.logsumexp(y, 0), h
            continue
        dy = -float(s["grad_logp"][i]) * q
        dy[t] += float(s["grad_logp"][i])
        if s["grad_entropy"] is not None:
            dy -= float(s["grad_entropy"][i]) * torch.where(q > 0, q * (logq + h), 0.0)
        d[i] = torch.where(slope != 0, dy * slope, 0.0)
    if grad:
        return {"d_logits": d}
    out = {"lse": got[:, 1].clone()}
    if case["entropy"]:
        out["entropy"] = got[:, 2].clone()
    if case["write"]:
        out["logits"] = kept
    else:
        out["logp"] = got[:, 0].clone()
    return out


def _exact_distill(s):
    case = s["case"]
    ids = s["ids"].long()
    T, K = ids.shape
    V, D = s["weight"].shape
    rows = torch.nonzero((ids >= 0).any(1))[:, 0]
    w = s["weight"].double()
    grad = case["op"] == "distill_grad"
    out = {"loss": torch.zeros(T, dtype=torch.float64, device=_DEVICE), "delta": torch.zeros(T, K, dtype=torch.float64, device=_DEVICE),
           "rest": torch.zeros(T, dtype=torch.float64, device=_DEVICE), "rest_lse": torch.zeros(T, dtype=torch.float64, device=_DEVICE)}
    dh = torch.zeros(T, D, dtype=torch.float64, device=_DEVICE) if grad else None
    dw = torch.zeros(V, D, dtype=torch.float64, device=_DEVICE) if grad else None
    for a in range(0, len(rows), 1024):
        r = rows[a:a + 1024]
        x, i = s["hidden"][r].double(), ids[r]
        entry = i >= 0
        z = torch.mm(x, w.t()) * s["scale"]
        at, col = torch.nonzero(entry, as_tuple=True)
        inside = torch.zeros_like(z, dtype=torch.bool)
        inside[at, i[at, col]] = True
        t = s["teacher"][r].double()
        t[~entry] = -math.inf
        mass = torch.logsumexp(t, 1)
        if case["tail"]:
            mass = mass.clamp(min=0.0)
        q = torch.exp(t - mass[:, None])
        left = (1.0 - q.sum(1)).clamp(min=0.0) if case["tail"] else torch.zeros(len(r), dtype=torch.float64, device=_DEVICE)
        p = torch.softmax(z, 1)
        logp = torch.log_softmax(z, 1)
        pr = torch.where(inside, 0.0, p).sum(1)
        lr = torch.logsumexp(torch.where(inside, -math.inf, z), 1)
        if grad:
            dense = torch.where(inside, 0.0, p * (1.0 - left / pr)[:, None])
            dense[at, i[at, col]] = (p[at, i[at, col]] - q[at, col])
            dense *= s["grad_loss"][r].double()[:, None] * s["scale"]
            dh[r] = torch.mm(dense, w)
            dw += torch.mm(dense.t(), x)
            continue
        lp = logp.gather(1, i.clamp(min=0))
        lq = t - mass[:, None]
        loss = torch.where(entry & (q > 0), q * (lq - lp), 0.0).sum(1)
        loss += torch.where(left > 0, left * (torch.log(left) - (lr - torch.logsumexp(z, 1))), 0.0)
        out["loss"][r] = loss
        out["delta"][r] = torch.where(entry, lp.exp() - q, 0.0)
        out["rest"][r] = pr - left
        out["rest_lse"][r] = lr
    return {"d_hidden": dh, "d_weight": dw} if grad else out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_adjust(s) if case["op"] in ("adjust", "adjust_grad") else _exact_distill(s)
