"""The two ends of a token model in float64, from the definitions: a token drawn from a row of logits, rows of an embedding table
with the table's gradient, and the norms' backward pass."""
from __future__ import annotations

import numpy as np

BLOCK = 512


def weights(logits, scale=1.0):
    """e^(x - max x) of a row, x = scale z; None where the row has no distribution (NaN, +inf, or -inf alone)."""
    x = np.asarray(logits, np.float64) * np.float64(np.float32(scale))
    if np.isnan(x).any() or x.max() == np.inf or x.max() == -np.inf:
        return None
    return np.exp(x - x.max())


def order(logits):
    """Tokens by logit, descending; equal ones by index; NaN with -inf."""
    z = np.asarray(logits, np.float64)
    return np.argsort(-(np.where(np.isnan(z), -np.inf, z) + 0.0), kind="stable")


def kept(logits, scale=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(mask of the tokens that may be drawn, how near the cut by mass is to another one, relative to the mass)."""
    w, o = weights(logits, scale), order(logits)
    n = len(w)
    if 0 < top_k < n:
        n = top_k
    if min_p > 0:
        n = min(n, int((w >= min_p).sum()))
    near = np.inf
    if top_p < 1.0:
        cum = np.cumsum(w[o[:n]])
        target = top_p * cum[-1]
        near = np.abs(cum - target).min() / cum[-1]
        n = min(n, int((cum < target).sum()) + 1)
    mask = np.zeros(len(w), bool)
    mask[o[:n]] = True
    return mask, near


def _first_above(cum, target):
    """(the first cumulative mass above target, or the last that adds anything; distance to the nearest border, relative)"""
    i = min(int((cum <= target).sum()), int((cum < cum[-1]).sum()))
    inner = cum[cum < cum[-1]]  # (the last border is nowhere near: no target passes it)
    inner = inner[inner > 0]
    return i, (np.abs(inner - target).min() / cum[-1] if inner.size else np.inf)


def sample(logits, u, scale=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, ln p, how near the draw was to another token, relative to the mass compared)."""
    w = weights(logits, scale)
    if w is None:
        z = np.asarray(logits, np.float64)
        return int(order(logits)[0]), (-np.inf if (z == -np.inf).all() else np.nan), np.inf
    mask, near = kept(logits, scale, top_k, top_p, min_p)
    u = [0.0 if np.isnan(x) else min(max(float(x), 0.0), 1.0) for x in u]
    m = np.where(mask, w, 0.0)
    m = np.pad(m, (0, -len(m) % BLOCK)).reshape(-1, BLOCK)
    cum = np.cumsum(m.sum(1))
    b, near0 = _first_above(cum, u[0] * cum[-1])
    cum = np.cumsum(m[b])
    t, near1 = _first_above(cum, u[1] * cum[-1])
    t = b * BLOCK + t
    return int(t), np.log(w[t] / w.sum()), min(near, near0, near1)


def embedding(table, ids, scale=1.0):
    table, ids = np.asarray(table, np.float64), np.asarray(ids)
    here = (ids >= 0) & (ids < len(table))
    return np.where(here[:, None], table[np.where(here, ids, 0)] * float(np.float32(scale)), 0.0)


def embedding_grad(grad, ids, vocab, scale=1.0):
    """(gradient of the table, sums of magnitudes, rows of each token)"""
    grad, ids = np.asarray(grad, np.float64), np.asarray(ids)
    out, size, n = np.zeros((vocab, grad.shape[1])), np.zeros((vocab, grad.shape[1])), np.zeros(vocab, np.int64)
    here = (ids >= 0) & (ids < vocab)
    np.add.at(out, ids[here], grad[here])
    np.add.at(size, ids[here], np.abs(grad[here]))
    np.add.at(n, ids[here], 1)
    s = float(np.float32(scale))
    return out * s, size * abs(s), n


def norm(h, kind, g=None, b=None, shift=None, scale=None, rows_per_batch=1, eps=1e-6):
    """kind: rms, ln or ln_plain."""
    h = np.asarray(h, np.float64)
    x = h if kind == "rms" else h - h.mean(1, keepdims=True)
    n = x / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    n = n if g is None else n * g
    n = n if b is None else n + b
    if scale is None:
        return n
    s = np.arange(len(h)) // rows_per_batch
    return n * (1 + scale[s]) + (0.0 if shift is None else shift[s])


def norm_grad(dout, h, kind, g=None, b=None, scale=None, rows_per_batch=1, eps=1e-6, residual=None):
    """dict of dh, dg, db, dshift and dscale (those that there is a parameter for)."""
    h, dout = np.asarray(h, np.float64), np.asarray(dout, np.float64)
    rows, d = h.shape
    x = h if kind == "rms" else h - h.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    xhat = x * rstd
    s = np.arange(rows) // rows_per_batch
    dn = dout if scale is None else dout * (1 + scale[s])
    dx = dn if g is None else dn * g
    dh = dx - xhat * (dx * xhat).mean(1, keepdims=True)
    if kind != "rms":
        dh = dh - dx.mean(1, keepdims=True)
    out = dict(dh=rstd * dh + (0.0 if residual is None else residual), dg=(dn * xhat).sum(0), db=dn.sum(0))
    if scale is not None:
        n = xhat if g is None else xhat * g
        n = n if b is None else n + b
        for name, v in (("dshift", dout), ("dscale", dout * n)):
            out[name] = np.zeros((len(scale), d))
            np.add.at(out[name], s, v)
    return out
