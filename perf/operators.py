"""The operators behind a token model's logits, timed at the sizes a program that denoises tokens or trains on
them calls them with: ``logprobs`` (log-probabilities of given tokens, entropy, the likeliest tokens), ``distill``
(loss against another evaluation's likeliest tokens, with its gradient) and ``reveal`` (which masked positions
take their candidates).

The plain forms are the definitions in elementary torch operations, in fp32; what enters the loss beside its exponentials
is in fp64, where terms of a list and its tail that cancel would otherwise leave little of it.
Vocabularies are those of the synthetic token models (1000 and 126464), one generic size, and odd ones.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
MASK = 0  # the id that marks a masked position here


def _logprobs(name, rows, vocab, dtype, top, tokens, entropy, active=1.0, scale=1.0, pad=0, banned=0):
    """`active`: the share of rows that is scored; `pad`: columns between rows; `banned`: tokens at -inf."""
    c = dict(kind="logprobs", rows=rows, vocab=vocab, dtype=dtype, top=top, tokens=tokens, entropy=entropy, active=active,
             scale=scale, pad=pad, banned=banned)
    return dict(c, name=name) if name else c


def _distill(name, rows, vocab, dtype, top, tail, grad, ignored=0.0, scale=1.0, ragged=False):
    """`grad`: the gradient's type, or "" for the loss alone; `ignored`: the share of rows of weight 0; `ragged`: lists of
    their own lengths."""
    c = dict(kind="distill", rows=rows, vocab=vocab, dtype=dtype, top=top, tail=tail, grad=grad, ignored=ignored, scale=scale,
             ragged=ragged)
    return dict(c, name=name) if name else c


def _reveal(name, batch, tokens, window, lowest):
    c = dict(kind="reveal", batch=batch, tokens=tokens, window=window, lowest=lowest)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one row: the next token's log-probability with a few alternatives, where latency is everything
        _logprobs("score one row", 1, 126464, "f16", 4, 1, True),
        # a prompt of odd length scored token by token
        _logprobs("score a prompt", 333, 126464, "f16", 0, 1, False),
        # a denoising step of the served batch: the best token of every position that is still masked, half of them
        _logprobs("candidates of a step", 4096, 126464, "f16", 1, 0, True, active=0.5),
        # the full model's likeliest tokens of every position, kept as a teacher
        _logprobs("teacher's list", 4096, 126464, "f16", 32, 0, False),
        # another vocabulary of odd size in a padded buffer, some tokens banned, a temperature
        _logprobs("odd vocabulary", 1003, 32003, "bf16", 8, 4, True, scale=1.25, pad=13, banned=7),
        # how far a scheduled evaluation is from the full one: the loss alone
        _distill("fidelity of a schedule", 1024, 126464, "f16", 32, "bucket", ""),
        # a training step of the served batch: loss and gradient
        _distill("distil a step", 4096, 126464, "f16", 32, "bucket", "bf16"),
        # cross entropy of the masked tokens (a list of one), the others ignored
        _distill("cross entropy", 2048, 32000, "bf16", 1, "renorm", "bf16", ignored=0.4),
        # logits and gradient in fp32, long lists, a temperature
        _distill("distil in fp32", 300, 126464, "f32", 64, "bucket", "f32", scale=0.5),
        # the small token model
        _distill("distil a small model", 17, 1000, "f32", 8, "renorm", "f32", ragged=True),
        # one short sample, a block of it at a time
        _reveal("reveal in a block", 1, 192, 32, False),
        # many long samples, lowest entropy first
        _reveal("reveal in a batch", 16, 4096, 0, True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["logprobs"] * 3 + ["distill"] * 3 + ["reveal"])
    if kind == "reveal":
        n = _log(rng, 32, 4096)
        return _reveal(None, _log(rng, 1, 16), n, rng.choice([0, 0, max(1, n // 8)]), rng.random() < 0.5)
    vocab = rng.choice([126464, 126464, 1000, _log(rng, 1000, 126464), _log(rng, 1000, 126464)])
    dtype = rng.choice(["f16", "f16", "bf16", "f32"])
    rows = _log(rng, 1, 4096 if dtype != "f32" else 2048)
    scale = rng.choice([1.0, 1.0, 0.5, 1.25])
    if kind == "logprobs":
        top, tokens = rng.choice([0, 1, 1, 4, 8, 32, 50]), rng.choice([0, 1, 1, 5])
        return _logprobs(None, rows, vocab, dtype, top, tokens, rng.random() < 0.6 or top + tokens == 0,
                         active=rng.choice([1.0, 1.0, 0.5, 0.1]), scale=scale, pad=rng.choice([0, 0, 8, 5]),
                         banned=rng.choice([0, 0, 1, 100]))
    grad = rng.choice(["", dtype, "bf16" if dtype == "f16" else dtype])
    return _distill(None, rows, vocab, dtype, rng.choice([1, 8, 32, 64]), rng.choice(["bucket", "renorm"]), grad,
                    ignored=rng.choice([0.0, 0.0, 0.4]), scale=scale, ragged=rng.random() < 0.3)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

CHUNK = 1 << 26  # values made at a time


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _chunks(rows, vocab):
    step = max(1, CHUNK // vocab)
    return [(a, min(rows, a + step)) for a in range(0, rows, step)]


def _rows_of_logits(g, n, vocab):
    """fp32 [n, vocab] as a trained head gives them: a wide bulk and a few tokens well above it."""
    z = 2.0 * torch.randn(n, vocab, generator=g, device="cuda")
    k = min(24, vocab)
    at = torch.randint(0, vocab, (n, k), generator=g, device="cuda")
    # (the larger of two that fall on one token: the same for the same seed)
    z.scatter_reduce_(1, at, 6.0 + 8.0 * torch.rand(n, k, generator=g, device="cuda"), "amax")
    return z


def _share(g, n, share):
    """bool [n]: round(share n) of them, at least one."""
    on = torch.zeros(n, dtype=torch.bool, device="cuda")
    on[torch.randperm(n, generator=g, device="cuda")[: max(1, round(share * n))]] = True
    return on


def prepare(case, seed):
    g, c = _generator(seed), case
    if c["kind"] == "reveal":
        B, N = c["batch"], c["tokens"]
        s = dict(case=c)
        ids = torch.randint(1, 126464, (B, N), generator=g, device="cuda", dtype=torch.int32)
        s["ids"] = torch.where(torch.rand(B, N, generator=g, device="cuda") < 0.6, MASK, ids).to(torch.int32)
        s["cand"] = torch.randint(1, 126464, (B, N), generator=g, device="cuda", dtype=torch.int32)
        u = torch.rand(B, N, generator=g, device="cuda")
        # entropies, or log-probabilities as coarse as fp16 logits make them: with ties
        s["score"] = 8.0 * u * u if c["lowest"] else torch.log(u + 1e-6).half().float()
        s["n_reveal"] = torch.randint(1, max(2, N // 8), (B,), generator=g, device="cuda", dtype=torch.int32)
        s["window"] = None
        if c["window"]:
            lo = torch.randint(0, N - c["window"] + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s["window"] = torch.stack([lo, lo + c["window"]], 1).contiguous()
        s["ids_out"], s["n_left"] = torch.empty_like(s["ids"]), torch.empty(B, dtype=torch.int32, device="cuda")
        return s
    R, V, dt = c["rows"], c["vocab"], DTYPES[c["dtype"]]
    s = dict(case=c)
    if c["kind"] == "logprobs":
        buf = torch.empty(R, V + c["pad"], dtype=dt, device="cuda")
        if c["pad"]:
            buf[:, V:] = 1000.0
        z = buf[:, :V]
        for a, b in _chunks(R, V):
            z[a:b] = _rows_of_logits(g, b - a, V)
        if c["banned"]:
            z[:, torch.randperm(V, generator=g, device="cuda")[: c["banned"]]] = -math.inf
        s["logits"] = z
        s["row_ids"] = None
        if c["active"] < 1.0:
            s["row_ids"] = torch.where(_share(g, R, c["active"]), MASK, 1).to(torch.int32)
        s["tokens"] = torch.randint(0, V, (R, c["tokens"]), generator=g, device="cuda", dtype=torch.int32) if c["tokens"] else None
        s["token_logprobs"] = torch.zeros(R, c["tokens"], device="cuda") if c["tokens"] else None
        s["entropy"] = torch.zeros(R, device="cuda") if c["entropy"] else None
        s["top_ids"] = torch.zeros(R, c["top"], dtype=torch.int32, device="cuda") if c["top"] else None
        s["top_logprobs"] = torch.zeros(R, c["top"], device="cuda") if c["top"] else None
        return s
    k = c["top"]
    s["logits"] = torch.empty(R, V, dtype=dt, device="cuda")
    s["ids"] = torch.empty(R, k, dtype=torch.int32, device="cuda")
    s["logq"] = torch.empty(R, k, device="cuda")
    for a, b in _chunks(R, V):
        z = _rows_of_logits(g, b - a, V)
        x = z * c["scale"]
        top = torch.topk(x, k, dim=1)
        s["ids"][a:b] = top.indices
        s["logq"][a:b] = 0.0 if k == 1 else top.values - torch.logsumexp(x, 1, keepdim=True)
        s["logits"][a:b] = z + 0.7 * torch.randn(b - a, V, generator=g, device="cuda")
    if c["ragged"]:
        n = torch.randint(1, k + 1, (R, 1), generator=g, device="cuda")
        s["ids"][torch.arange(k, device="cuda")[None] >= n] = -1
    s["weight"] = (0.5 + torch.rand(R, generator=g, device="cuda")) / R
    if c["ignored"]:
        s["weight"][_share(g, R, c["ignored"])] = 0.0
    s["loss"] = torch.empty(R, device="cuda")
    s["grad"] = torch.empty(R, V, dtype=DTYPES[c["grad"]], device="cuda") if c["grad"] else None
    return s


# ---------------------------------------------------------------------------
# the operators
# ---------------------------------------------------------------------------

def _plain_logprobs(s):
    c, z = s["case"], s["logits"].float()
    V = c["vocab"]
    x = z * c["scale"]
    M = x.amax(1, keepdim=True)
    empty = M == -math.inf
    d = x - torch.where(empty, 0.0, M)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    on = torch.ones_like(empty) if s["row_ids"] is None else (s["row_ids"] == MASK)[:, None]
    out = {}

    def logprob(at):
        return torch.where(empty, -math.inf, torch.gather(d, 1, at) - torch.log(total))

    if s["tokens"] is not None:
        t = s["tokens"].long()
        v = logprob(t.clamp(0, V - 1))
        v = torch.where(t < 0, 0.0, torch.where(t >= V, math.nan, v))
        out["token_logprobs"] = torch.where(on, v, s["token_logprobs"])
    if s["entropy"] is not None:
        v = torch.log(total) - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total
        out["entropy"] = torch.where(on, torch.where(empty, 0.0, v), s["entropy"][:, None])[:, 0]
    if s["top_ids"] is not None:
        # one 64-bit key per token: its logit's order above, its index's below
        bits = (z + 0.0).view(torch.int32)
        order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
        at = torch.arange(V - 1, -1, -1, device=z.device)
        key = torch.topk((order << 32) | at, c["top"], dim=1).values
        ids = V - 1 - (key & 0xFFFFFFFF)
        out["top_ids"] = torch.where(on, ids.int(), s["top_ids"])
        out["top_logprobs"] = torch.where(on, logprob(ids), s["top_logprobs"])
    return out


def _plain_distill(s):
    c, w = s["case"], s["weight"][:, None]
    V = c["vocab"]
    x = s["logits"].float() * c["scale"]
    M = x.amax(1, keepdim=True)
    empty = M == -math.inf
    d = x - torch.where(empty, 0.0, M)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    ids, logq = s["ids"].long(), s["logq"].double()
    here = (ids >= 0) & (ids < V)
    same = torch.tril(ids[:, :, None] == ids[:, None, :], -1).any(2)
    here &= ~same
    q = torch.where(here, torch.exp(logq), 0.0)
    Q = q.sum(1, keepdim=True)
    at = torch.where(here, ids, V)
    inside = torch.zeros(x.shape[0], V + 1, dtype=torch.bool, device=x.device).scatter_(1, at, True)[:, :V]
    logp = torch.where(empty, -math.inf, torch.gather(d, 1, at.clamp(max=V - 1)).double() - torch.log(total))
    p = torch.where(empty, 0.0, e / total.float())
    if c["tail"] == "renorm":
        q = torch.where(Q > 0, q / Q, 0.0)
        logq = logq - torch.log(Q)
        loss = torch.where(q > 0, q * (logq - logp), 0.0).sum(1, keepdim=True)
        outside = p
    else:
        qt = (1.0 - Q).clamp(min=0.0)
        pt = torch.where(inside | empty, 0.0, e).sum(1, keepdim=True, dtype=torch.float64) / torch.where(empty, 1.0, total)
        loss = torch.where(q > 0, q * (logq - logp), 0.0).sum(1, keepdim=True)
        loss = loss + torch.where((qt > 0) & (pt > 0), qt * (torch.log(qt) - torch.log(pt)), 0.0)
        outside = p * torch.where(pt > 0, 1.0 - qt / pt, 1.0).float()
    out = {"loss": torch.where(w != 0, w * loss, 0.0)[:, 0].float()}
    if c["grad"]:
        target = torch.zeros(x.shape[0], V + 1, device=x.device).scatter_(1, at, q.float())[:, :V]
        none = (Q == 0).float() if c["tail"] == "renorm" else 0.0  # an empty list pulls at nothing
        grad = (torch.where(inside, p, outside) - target) * (w * c["scale"] * (1.0 - none))
        out["grad"] = torch.where(w != 0, grad, 0.0).to(DTYPES[c["grad"]])
    return out


def _plain_reveal(s):
    ids, N = s["ids"], s["ids"].shape[1]
    pos = torch.arange(N, device=ids.device)[None]
    masked = ids == MASK
    may = masked
    if s["window"] is not None:
        may = may & (pos >= s["window"][:, :1]) & (pos < s["window"][:, 1:])
    score = -s["score"] if s["case"]["lowest"] else s["score"]
    score = torch.where(torch.isnan(score), -math.inf, score) + 0.0
    bits = score.view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
    key = torch.where(may, ((order << 32) | (N - 1 - pos)), torch.iinfo(torch.int64).min)
    rank = torch.argsort(torch.argsort(key, 1, descending=True), 1)
    take = may & (rank < s["n_reveal"][:, None])
    return {"ids": torch.where(take, s["cand"], ids), "n_left": (masked & ~take).sum(1).int()}


def _own(s):
    from paper_2609_29505_gb300 import binding
    c = s["case"]
    if c["kind"] == "logprobs":
        binding.sgd_kernel_logprobs(s["logits"], tokens=s["tokens"], token_logprobs=s["token_logprobs"], entropy=s["entropy"],
                                    top_ids=s["top_ids"], top_logprobs=s["top_logprobs"], scale=c["scale"],
                                    row_ids=s["row_ids"], row_id=MASK)
        return {n: s[n] for n in ("token_logprobs", "entropy", "top_ids", "top_logprobs") if s[n] is not None}
    if c["kind"] == "distill":
        binding.sgd_kernel_distill(s["logits"], s["ids"], s["logq"], s["loss"], grad=s["grad"], row_weight=s["weight"],
                                   tail=binding.TAIL[c["tail"]], scale=c["scale"])
        return {n: s[n] for n in ("loss", "grad") if s[n] is not None}
    binding.sgd_sampler_reveal(s["ids"], s["cand"], s["score"], s["n_reveal"], s["ids_out"], MASK, lowest=c["lowest"],
                               window=s["window"], n_left=s["n_left"])
    return {"ids": s["ids_out"], "n_left": s["n_left"]}


def run(state):
    if own:
        return _own(state)
    return {"logprobs": _plain_logprobs, "distill": _plain_distill, "reveal": _plain_reveal}[state["case"]["kind"]](state)


def work(case):
    c = case
    size = {"f16": 2, "bf16": 2, "f32": 4, "": 0}
    if c["kind"] == "reveal":
        n = c["batch"] * c["tokens"]
        # ids in and out; candidate and score where the window is
        return {"bytes": 8.0 * n + 8.0 * c["batch"] * (c["window"] or c["tokens"]) + 16.0 * c["batch"], "flops": float(n)}
    R, V = c["rows"], c["vocab"]
    if c["kind"] == "logprobs":
        R = max(1, round(c["active"] * R))
        # an exponential, a subtraction, a sum (and for the entropy a product and a sum) per logit
        return {"bytes": R * (V * size[c["dtype"]] + 8.0 * c["tokens"] + 4.0 * c["entropy"] + 8.0 * c["top"]),
                "flops": R * V * (5.0 if c["entropy"] else 3.0)}
    live = R - (max(1, round(c["ignored"] * R)) if c["ignored"] else 0)
    return {"bytes": live * (V * size[c["dtype"]] + 8.0 * c["top"]) + R * (V * size[c["grad"]] + 8.0),
            "flops": live * V * (3.0 + (3.0 if c["grad"] else 0.0))}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_logprobs(s, c):
    R, V = c["rows"], c["vocab"]
    out = {n: (None if n == "top_ids" else s[n].double()) for n in ("token_logprobs", "entropy", "top_ids", "top_logprobs")
           if s[n] is not None}
    for a, b in _chunks(R, V):
        lp = torch.log_softmax(s["logits"][a:b].double() * c["scale"], 1)
        on = slice(None) if s["row_ids"] is None else s["row_ids"][a:b] == MASK
        if s["tokens"] is not None:
            out["token_logprobs"][a:b][on] = torch.take_along_dim(lp, s["tokens"][a:b].long(), 1)[on]
        if s["entropy"] is not None:
            out["entropy"][a:b][on] = -(lp.exp() * lp.clamp(min=-1e6)).sum(1)[on]
        if s["top_ids"] is not None:
            out["top_logprobs"][a:b][on] = torch.topk(lp, c["top"], 1).values[on]
    return out


def _exact_distill(s, c):
    """The loss as a sum over tokens and, where there is one, the tail; the gradient from d ln p_i / d z_j."""
    R, V = c["rows"], c["vocab"]
    loss = torch.zeros(R, dtype=torch.float64, device="cuda")
    grad = torch.zeros(R, V, dtype=torch.float64, device="cuda") if c["grad"] else None
    for a, b in _chunks(R, V):
        lp = torch.log_softmax(s["logits"][a:b].double() * c["scale"], 1)
        ids, lq, w = s["ids"][a:b].long(), s["logq"][a:b].double(), s["weight"][a:b].double()
        q = torch.zeros(b - a, V + 1, dtype=torch.float64, device="cuda")
        q.scatter_(1, torch.where(ids < 0, V, ids), lq.exp())
        q = q[:, :V]
        if c["tail"] == "renorm":
            q = q / q.sum(1, keepdim=True)
            loss[a:b] = w * (torch.xlogy(q, q) - q * lp).sum(1)
            if c["grad"]:
                grad[a:b] = (lp.exp() - q) * w[:, None] * c["scale"]
            continue
        tail = q == 0
        qt = (1 - q.sum(1)).clamp(min=0)
        lpt = torch.logsumexp(torch.where(tail, lp, -math.inf), 1)
        loss[a:b] = w * ((torch.xlogy(q, q) - q * lp).sum(1) + torch.xlogy(qt, qt) - qt * lpt)
        if c["grad"]:
            # minus each token's pull (q, or the tail's share of q_T by p_j / p_T), plus p for all the mass 1
            pull = torch.where(tail, torch.exp(lp - lpt[:, None]) * qt[:, None], q)
            grad[a:b] = (lp.exp() * (q.sum(1) + qt)[:, None] - pull) * w[:, None] * c["scale"]
    return {n: v for n, v in (("loss", loss), ("grad", grad)) if v is not None}


def exact(case, seed):
    if case["kind"] == "reveal":
        return None  # whole numbers alone
    s = prepare(case, seed)
    return (_exact_logprobs if case["kind"] == "logprobs" else _exact_distill)(s, case)
