"""The operators at the two ends of a token model, timed at the sizes a program that draws tokens from its logits, or
trains its embedding and its norms, calls them with: ``sample`` (a token per row, with temperature, top-k, min-p and
top-p, from given random numbers), ``embedding`` (rows of a table, scaled), ``embedding_grad`` (the table's gradient) and
``norm_grad`` (a norm's backward pass, with the gradients of its gain, shift and modulation).

The plain forms are the definitions in elementary torch operations, in fp32; masses that a random number or a share is
compared with, and sums over many rows, are in fp64.  Sizes are those of the synthetic models (vocabularies 1000 and
126464; widths 256, 288, 1024, 1152, 1280 and 4096), generic ones, and odd ones.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}
MASK = 0     # the id that marks a masked position here
BLOCK = 512  # tokens of a block: a token is drawn in two steps, the block and the token in it
EPS = 1e-6


def _sample(name, rows, vocab, dtype, top_k=0, top_p=1.0, min_p=0.0, scale=1.0, active=1.0, pad=0, banned=0, logprob=True):
    """`scale`: 1 / temperature; `active`: the share of rows that draws; `pad`: columns between rows; `banned`: tokens at -inf."""
    c = dict(kind="sample", rows=rows, vocab=vocab, dtype=dtype, top_k=top_k, top_p=top_p, min_p=min_p, scale=scale, active=active,
             pad=pad, banned=banned, logprob=logprob)
    return dict(c, name=name) if name else c


def _embedding(name, rows, vocab, d, dtype, out, scale=1.0, masked=0.0):
    """`out`: the type of the rows that are written; `masked`: the share of positions that hold the mask token."""
    c = dict(kind="embedding", rows=rows, vocab=vocab, d=d, dtype=dtype, out=out, scale=scale, masked=masked)
    return dict(c, name=name) if name else c


def _embedding_grad(name, rows, vocab, d, dtype, out, scale=1.0, masked=0.0, padded=0.0):
    """`dtype`: of the rows' gradients; `out`: of the table's; `padded`: the share of positions without a token."""
    c = dict(kind="embedding_grad", rows=rows, vocab=vocab, d=d, dtype=dtype, out=out, scale=scale, masked=masked, padded=padded)
    return dict(c, name=name) if name else c


def _norm_grad(name, rows, d, dtype, norm, affine, per=0, residual=True, params=True):
    """`affine`: a gain ("g"), a gain and a shift ("gb") or neither; `per`: rows of a sample with a modulation of its own (0: no
    modulation); `residual`: the gradient that comes past the branch is added; `params`: the parameters' gradients too."""
    c = dict(kind="norm_grad", rows=rows, d=d, dtype=dtype, norm=norm, affine=affine, per=per, residual=residual, params=params)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the next token of one row from the likeliest 95%, where latency is everything
        _sample("draw one row", 1, 126464, "f16", top_p=0.95, scale=1.25),
        # a denoising step of the served batch: a candidate for every position that is still masked, half of them
        _sample("draw a step", 4096, 126464, "f16", active=0.5),
        # the likeliest 90% of a broad distribution: thousands of tokens
        _sample("draw from a nucleus", 1024, 126464, "bf16", top_p=0.9),
        # every filter, another vocabulary of odd size in a padded buffer, some tokens banned
        _sample("draw with filters", 1003, 32003, "f32", top_k=50, top_p=0.9, min_p=0.02, scale=1.5, pad=13, banned=7),
        # a block of a short sample enters the model
        _embedding("look up a block", 32, 126464, 4096, "bf16", "f32"),
        # the served batch, half of it masked, scaled by sqrt(d) into the fp32 residual stream
        _embedding("look up a batch", 4096, 126464, 4096, "bf16", "f32", scale=64.0, masked=0.5),
        # a training step of a small model
        _embedding_grad("gradient of a small table", 192, 1000, 256, "f32", "f32", masked=0.3),
        # a training step of the served batch, half of it masked: one token has half of the rows
        _embedding_grad("gradient of a large table", 4096, 126464, 4096, "bf16", "bf16", scale=64.0, masked=0.5),
        # many rows for a table of odd size, with padding
        _embedding_grad("gradient of many rows", 65537, 32003, 1024, "bf16", "f32", masked=0.15, padded=0.1),
        # the final norm of the small token model
        _norm_grad("norm of a small model", 64, 256, "f32", "rms", "g", residual=False),
        # a norm of the served batch, the residual stream's gradient added
        _norm_grad("norm of a batch", 4096, 4096, "bf16", "rms", "g"),
        # a modulated norm of the image model: a shift and a scale per sample
        _norm_grad("modulated norm", 2048, 1152, "f16", "ln_plain", "", per=256),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["sample"] * 3 + ["embedding"] + ["embedding_grad"] * 2 + ["norm_grad"] * 2)
    if kind == "sample":
        vocab = rng.choice([126464, 126464, 1000, _log(rng, 1000, 126464), _log(rng, 1000, 126464)])
        dtype = rng.choice(["f16", "f16", "bf16", "f32"])
        which = rng.choice(["all", "all", "p", "p", "k", "kp", "m", "kpm", "pm"])
        rows = _log(rng, 1, 2048 if which == "all" and dtype != "f32" else 1024)
        return _sample(None, rows, vocab, dtype, top_k=rng.choice([1, 20, 50, 50, 400]) if "k" in which else 0,
                       top_p=rng.choice([0.5, 0.8, 0.9, 0.95]) if "p" in which else 1.0,
                       min_p=rng.choice([0.02, 0.05, 0.1]) if "m" in which else 0.0, scale=rng.choice([1.0, 1.0, 1.25, 2.0]),
                       active=rng.choice([1.0, 1.0, 0.5, 0.1]), pad=rng.choice([0, 0, 8, 5]), banned=rng.choice([0, 0, 1, 100]),
                       logprob=rng.random() < 0.7)
    if kind == "norm_grad":
        d = rng.choice([4096, 1152, 256, 4 * _log(rng, 16, 1024), 4 * _log(rng, 16, 1024)])
        norm = rng.choice(["rms", "rms", "ln", "ln_plain"])
        rows = _log(rng, 1, min(16384, (4096 * 4096) // d))
        return _norm_grad(None, rows, d, rng.choice(["f16", "bf16", "f32"]), norm, {"rms": "g", "ln": "gb", "ln_plain": ""}[norm],
                          per=_log(rng, 1, rows) if norm == "ln_plain" else 0, residual=rng.random() < 0.6, params=rng.random() < 0.8)
    vocab = rng.choice([126464, 1000, _log(rng, 1000, 126464), _log(rng, 1000, 126464)])
    d = rng.choice([4096, 256, _log(rng, 64, 4096), 8 * _log(rng, 8, 512)])
    dtype, masked = rng.choice(["f16", "bf16", "bf16", "f32"]), rng.choice([0.0, 0.15, 0.5, 0.9])
    scale = rng.choice([1.0, 1.0, math.sqrt(d)])
    if kind == "embedding":
        return _embedding(None, _log(rng, 1, min(65536, (4096 * 4096) // d)), vocab, d, dtype, rng.choice([dtype, "f32", "bf16"]),
                          scale=scale, masked=masked)
    out = rng.choice([dtype, "f32"])
    vocab = min(vocab, (126464 * 4096 * 2) // (d * SIZE[out]))
    return _embedding_grad(None, _log(rng, 1, min(65536, (4096 * 4096) // d)), vocab, d, dtype, out, scale=scale, masked=masked,
                           padded=rng.choice([0.0, 0.0, 0.2]))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

CHUNK = 1 << 25  # values made, or worked on, at a time


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _chunks(rows, width):
    step = max(1, CHUNK // width)
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
    """bool [n]: round(share n) of them."""
    on = torch.zeros(n, dtype=torch.bool, device="cuda")
    on[torch.randperm(n, generator=g, device="cuda")[: round(share * n)]] = True
    return on


def _tokens(g, c):
    """Ids as text has them: frequent ones and rare ones (the logarithm of the id is uniform), and the mask token."""
    u = torch.rand(c["rows"], generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(c["vocab"])).long() - 1).clamp(0, c["vocab"] - 1)
    # (the frequent ones anywhere in the table)
    ids = (ids * 48271 + 11) % c["vocab"]
    ids[_share(g, c["rows"], c["masked"])] = c["vocab"] - 1
    return ids.int()


def prepare(case, seed):
    g, c = _generator(seed), case
    s = dict(case=c)
    if c["kind"] == "sample":
        R, V = c["rows"], c["vocab"]
        buf = torch.empty(R, V + c["pad"], dtype=DTYPES[c["dtype"]], device="cuda")
        if c["pad"]:
            buf[:, V:] = 1000.0
        z = buf[:, :V]
        for a, b in _chunks(R, V):
            z[a:b] = _rows_of_logits(g, b - a, V)
        if c["banned"]:
            z[:, torch.randperm(V, generator=g, device="cuda")[: c["banned"]]] = -math.inf
        s["logits"] = z
        s["uniforms"] = torch.rand(R, 2, generator=g, device="cuda")
        s["row_ids"] = None
        if c["active"] < 1.0:
            on = _share(g, R, c["active"])
            on[0] = True
            s["row_ids"] = torch.where(on, MASK, 1).to(torch.int32)
        s["ids"] = torch.zeros(R, dtype=torch.int32, device="cuda")
        s["logprobs"] = torch.zeros(R, device="cuda") if c["logprob"] else None
        return s
    if c["kind"] == "embedding":
        s["table"] = torch.empty(c["vocab"], c["d"], dtype=DTYPES[c["dtype"]], device="cuda")
        for a, b in _chunks(c["vocab"], c["d"]):
            s["table"][a:b] = torch.randn(b - a, c["d"], generator=g, device="cuda")
        s["ids"] = _tokens(g, c)
        s["out"] = torch.empty(c["rows"], c["d"], dtype=DTYPES[c["out"]], device="cuda")
        return s
    if c["kind"] == "embedding_grad":
        s["grad"] = torch.randn(c["rows"], c["d"], generator=g, device="cuda").to(DTYPES[c["dtype"]])
        s["ids"] = _tokens(g, c)
        s["ids"][_share(g, c["rows"], c["padded"])] = -1
        s["dtable"] = torch.empty(c["vocab"], c["d"], dtype=DTYPES[c["out"]], device="cuda")
        if own:
            from paper_2609_29505_gb300 import binding
            n = binding.sgd_kernel_embedding_grad_workspace(c["rows"], c["vocab"], c["d"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        return s
    R, d = c["rows"], c["d"]
    # rows of a residual stream: an offset and a size of their own, a few channels far larger than the others
    h = torch.randn(R, d, generator=g, device="cuda") * (0.5 + torch.rand(R, 1, generator=g, device="cuda"))
    h += 0.2 * torch.randn(R, 1, generator=g, device="cuda")
    h[:, torch.randperm(d, generator=g, device="cuda")[:2]] *= 20.0
    s["h"] = h
    s["dout"] = torch.randn(R, d, generator=g, device="cuda").to(DTYPES[c["dtype"]])
    s["g"] = (1.0 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16() if "g" in c["affine"] else None
    s["b"] = (0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16() if "b" in c["affine"] else None
    n = -(-R // c["per"]) if c["per"] else 0
    s["scale"] = 0.3 * torch.randn(n, d, generator=g, device="cuda") if n else None
    s["residual"] = torch.randn(R, d, generator=g, device="cuda") if c["residual"] else None
    s["dh"] = torch.empty(R, d, device="cuda")
    s["dg"] = torch.empty(d, device="cuda") if c["params"] and "g" in c["affine"] else None
    s["db"] = torch.empty(d, device="cuda") if c["params"] and "b" in c["affine"] else None
    s["dshift"] = torch.empty(n, d, device="cuda") if c["params"] and n else None
    s["dscale"] = torch.empty(n, d, device="cuda") if c["params"] and n else None
    if own:
        from paper_2609_29505_gb300 import binding
        n = binding.sgd_kernel_norm_grad_workspace(R, d, c["per"])
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------
# the operators
# ---------------------------------------------------------------------------

def _first_above(cum, at):
    """Index of the first cumulative mass above at [n, 1]; the last one that adds anything where there is none."""
    i = (cum <= at).sum(1, keepdim=True)
    last = (cum < cum[:, -1:]).sum(1, keepdim=True)
    return torch.minimum(i, last)


def _plain_sample(s):
    c, V = s["case"], s["case"]["vocab"]
    nb = -(-V // BLOCK)
    ids, logprobs = s["ids"].clone(), None if s["logprobs"] is None else s["logprobs"].clone()
    for a, b in _chunks(c["rows"], V):
        z = s["logits"][a:b].float()
        x = z.double() * c["scale"]
        d = x - x.amax(1, keepdim=True)
        w = torch.exp(d)
        keep = torch.ones_like(w, dtype=torch.bool)
        if c["min_p"] > 0:
            keep &= w >= c["min_p"]
        if c["top_k"] or c["top_p"] < 1:
            # one 64-bit key per token: its logit's order above, its index's below
            bits = (z + 0.0).view(torch.int32)
            order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
            key = (order << 32) | torch.arange(V - 1, -1, -1, device=z.device)
            if c["top_k"]:
                key = torch.topk(key, min(c["top_k"], V), dim=1).values
            else:
                key = torch.sort(key, dim=1, descending=True).values
            at = V - 1 - (key & 0xFFFFFFFF)
            m = torch.where(torch.gather(keep, 1, at), torch.gather(w, 1, at), 0.0)
            if c["top_p"] < 1:
                before = torch.cumsum(m, 1) - m
                m = torch.where(before < c["top_p"] * m.sum(1, keepdim=True), m, 0.0)
            w = torch.zeros_like(w).scatter_(1, at, m)
        else:
            w = torch.where(keep, w, 0.0)
        w = torch.nn.functional.pad(w, (0, nb * BLOCK - V)).view(b - a, nb, BLOCK)
        u = s["uniforms"][a:b].double()
        cum = torch.cumsum(w.sum(2), 1)
        block = _first_above(cum, u[:, :1] * cum[:, -1:])
        cum = torch.cumsum(torch.gather(w, 1, block[:, :, None].expand(-1, 1, BLOCK))[:, 0], 1)
        t = block * BLOCK + _first_above(cum, u[:, 1:] * cum[:, -1:])
        on = torch.ones_like(t[:, 0], dtype=torch.bool) if s["row_ids"] is None else s["row_ids"][a:b] == MASK
        ids[a:b] = torch.where(on, t[:, 0].int(), ids[a:b])
        if logprobs is not None:
            lp = torch.gather(d, 1, t) - torch.log(torch.exp(d).sum(1, keepdim=True))
            logprobs[a:b] = torch.where(on, lp[:, 0].float(), logprobs[a:b])
    return {"ids": ids} if logprobs is None else {"ids": ids, "logprobs": logprobs}


def _plain_embedding(s):
    c = s["case"]
    return (s["table"][s["ids"].long()].float() * c["scale"]).to(DTYPES[c["out"]])


def _plain_embedding_grad(s):
    c = s["case"]
    ids = s["ids"].long()
    here = ids >= 0
    total = torch.zeros(c["vocab"], c["d"], dtype=torch.float64, device=ids.device)
    total.index_add_(0, torch.where(here, ids, 0), torch.where(here[:, None], s["grad"].double(), 0.0))
    return (total * c["scale"]).to(DTYPES[c["out"]])


def _plain_norm_grad(s):
    c, h, dout = s["case"], s["h"], s["dout"].float()
    R, d = h.shape
    x = h - h.mean(1, keepdim=True) if c["norm"] != "rms" else h
    rstd = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    xhat = x * rstd
    dn, sample = dout, None
    if s["scale"] is not None:
        sample = torch.arange(R, device=h.device) // c["per"]
        dn = dout * (1.0 + s["scale"][sample])
    dx = dn if s["g"] is None else dn * s["g"].float()
    dh = dx - xhat * (dx * xhat).mean(1, keepdim=True)
    if c["norm"] != "rms":
        dh = dh - dx.mean(1, keepdim=True)
    dh = dh * rstd
    if s["residual"] is not None:
        dh = dh + s["residual"]
    out = {"dh": dh}
    if s["dg"] is not None:
        out["dg"] = (dn * xhat).sum(0)
    if s["db"] is not None:
        out["db"] = dn.sum(0)
    if s["dscale"] is not None:
        n = xhat if s["g"] is None else xhat * s["g"].float()
        n = n if s["b"] is None else n + s["b"].float()
        def of_samples(v):
            v = torch.nn.functional.pad(v, (0, 0, 0, s["scale"].shape[0] * c["per"] - R))
            return v.view(-1, c["per"], d).sum(1)
        out["dshift"], out["dscale"] = of_samples(dout), of_samples(dout * n)
    return out


def _own(s):
    from paper_2609_29505_gb300 import binding
    c = s["case"]
    if c["kind"] == "sample":
        binding.sgd_kernel_sample(s["logits"], s["uniforms"], s["ids"], logprobs=s["logprobs"], scale=c["scale"], top_k=c["top_k"],
                                  top_p=c["top_p"], min_p=c["min_p"], row_ids=s["row_ids"], row_id=MASK)
        return {n: s[n] for n in ("ids", "logprobs") if s[n] is not None}
    if c["kind"] == "embedding":
        binding.sgd_kernel_embedding(s["table"], s["ids"], s["out"], scale=c["scale"])
        return s["out"]
    if c["kind"] == "embedding_grad":
        binding.sgd_kernel_embedding_grad(s["grad"], s["ids"], s["dtable"], scale=c["scale"], workspace=s["workspace"])
        return s["dtable"]
    binding.sgd_kernel_norm_grad(s["dout"], s["h"], binding.NORM[c["norm"]], dh=s["dh"], g=s["g"], b=s["b"], scale=s["scale"],
                                 rows_per_batch=max(c["per"], 1), eps=EPS, residual=s["residual"], dg=s["dg"], db=s["db"],
                                 dshift=s["dshift"], dscale=s["dscale"], workspace=s["workspace"])
    return {n: s[n] for n in ("dh", "dg", "db", "dshift", "dscale") if s[n] is not None}


def run(state):
    if own:
        return _own(state)
    return {"sample": _plain_sample, "embedding": _plain_embedding, "embedding_grad": _plain_embedding_grad,
            "norm_grad": _plain_norm_grad}[state["case"]["kind"]](state)


def _distinct(c, n):
    """Expected number of different tokens among n that are drawn as _tokens draws them, and the mask token."""
    t = torch.arange(1, c["vocab"], dtype=torch.float64)
    p = torch.log((t + 1) / t) / math.log(c["vocab"])
    return float((1 - (1 - p) ** n).sum()) + (1 if c["masked"] else 0)


def work(case):
    c = case
    if c["kind"] == "sample":
        R, V = c["rows"], c["vocab"]
        live = max(1, round(c["active"] * R)) if c["active"] < 1.0 else R
        # an exponential, a subtraction and a sum per logit
        return {"bytes": live * (V * SIZE[c["dtype"]] + 12.0 + 4.0 * c["logprob"]) + (4.0 * R if c["active"] < 1.0 else 0.0),
                "flops": 3.0 * live * V}
    n, d = c["rows"], c["d"]
    if c["kind"] == "embedding":
        rows = _distinct(c, n - round(c["masked"] * n))
        return {"bytes": rows * d * SIZE[c["dtype"]] + n * (d * SIZE[c["out"]] + 4.0), "flops": float(n) * d}
    if c["kind"] == "embedding_grad":
        live = n - round(c["padded"] * n)
        return {"bytes": live * d * float(SIZE[c["dtype"]]) + 4.0 * n + float(c["vocab"]) * d * SIZE[c["out"]], "flops": float(live) * d}
    b = n * d * (4.0 + SIZE[c["dtype"]] + 4.0 + (4.0 if c["residual"] else 0.0)) + 2.0 * d * len(c["affine"])
    if c["params"]:
        b += 4.0 * d * len(c["affine"])
    if c["per"]:
        b += -(-n // c["per"]) * d * (12.0 if c["params"] else 4.0)
    return {"bytes": b, "flops": n * d * (14.0 + (4.0 if c["params"] else 0.0))}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_sample(c, seed):
    """The drawn tokens are whole numbers; of theirs the log-probability, in 64 bits from the tokens that the plain form draws."""
    if not c["logprob"]:
        return None  # whole numbers alone
    s = prepare(c, seed)
    ids, out = _plain_sample(s)["ids"].long(), s["logprobs"].double()
    for a, b in _chunks(c["rows"], c["vocab"]):
        lp = torch.log_softmax(s["logits"][a:b].double() * c["scale"], 1)
        on = slice(None) if s["row_ids"] is None else s["row_ids"][a:b] == MASK
        out[a:b][on] = torch.take_along_dim(lp, ids[a:b, None], 1)[:, 0][on]
    return {"ids": None, "logprobs": out}


def _exact_embedding_grad(c, s):
    """Sums of runs of equal tokens, as differences of running sums over the rows sorted by token."""
    out = torch.zeros(c["vocab"] + 1, c["d"], dtype=torch.float64, device="cuda")
    ids, order = torch.sort(s["ids"].long(), stable=True)
    end = torch.ones_like(ids, dtype=torch.bool)
    end[:-1] = ids[1:] != ids[:-1]
    last = torch.nonzero(end)[:, 0]
    for a in range(0, c["d"], 512):
        run = torch.cumsum(s["grad"][order, a:a + 512].double(), 0)[last]
        out[ids[last], a:a + 512] = c["scale"] * torch.diff(run, dim=0, prepend=torch.zeros_like(run[:1]))
    return out[: c["vocab"]]  # (rows without a token went to the last one, index -1)


def _exact_norm_grad(c, s):
    """Through automatic differentiation of the norm in fp64."""
    h = s["h"].double().requires_grad_()
    leaves = {"dh": h}
    if c["norm"] == "rms":
        y = h / torch.sqrt(h.pow(2).mean(1, keepdim=True) + EPS)
    else:
        var, mean = torch.var_mean(h, 1, correction=0, keepdim=True)
        y = (h - mean) / torch.sqrt(var + EPS)
    for n in ("g", "b"):
        if s[n] is not None:
            leaves["d" + n] = s[n].double().requires_grad_()
            y = y * leaves["dg"] if n == "g" else y + leaves["db"]
    if s["scale"] is not None:
        leaves["dscale"] = s["scale"].double().requires_grad_()
        leaves["dshift"] = torch.zeros_like(leaves["dscale"]).requires_grad_()
        y = y * (1 + leaves["dscale"].repeat_interleave(c["per"], 0)[: c["rows"]]) \
            + leaves["dshift"].repeat_interleave(c["per"], 0)[: c["rows"]]
    grads = dict(zip(leaves, torch.autograd.grad(y, list(leaves.values()), s["dout"].double())))
    if s["residual"] is not None:
        grads["dh"] = grads["dh"] + s["residual"].double()
    return {n: grads[n] for n in ("dh", "dg", "db", "dshift", "dscale") if s[n] is not None}


def exact(case, seed):
    if case["kind"] == "sample":
        return _exact_sample(case, seed)
    s = prepare(case, seed)
    if case["kind"] == "embedding":
        return s["table"][s["ids"].long()].double() * case["scale"]
    return (_exact_embedding_grad if case["kind"] == "embedding_grad" else _exact_norm_grad)(case, s)
