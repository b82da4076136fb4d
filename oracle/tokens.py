"""What follows a token model's logits, in float64 from the definitions: log-probabilities with entropy
and likeliest tokens, distillation from a list of likeliest tokens, and the reveal step of the
masked-token sampler."""
from __future__ import annotations

import numpy as np


def log_softmax(logits, scale=1.0):
    """ln softmax(scale z) by rows; -inf throughout for a row of -inf alone, NaN for one with NaN or +inf."""
    x = np.asarray(logits, np.float64) * scale
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        m = x.max(axis=-1, keepdims=True)
        d = x - m
        lp = d - np.log(np.exp(d).sum(axis=-1, keepdims=True))
    lp = np.where(np.isnan(x).any(axis=-1, keepdims=True) | (m == np.inf), np.nan, lp)
    return np.where(m == -np.inf, -np.inf, lp)


def entropy(lp):
    p = np.exp(lp)
    return -np.sum(np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, lp)), axis=-1)


def top(logits, k):
    """Tokens of the k largest logits, descending, equal ones by index; NaN ranks with -inf."""
    z = np.asarray(logits, np.float64)
    z = np.where(np.isnan(z), -np.inf, z) + 0.0
    return np.argsort(-z, axis=-1, kind="stable")[:, :k]


def token_logprobs(lp, tokens):
    rows, vocab = lp.shape
    t = np.asarray(tokens)
    got = np.take_along_axis(lp, np.clip(t, 0, vocab - 1), axis=1)
    return np.where(t < 0, 0.0, np.where(t >= vocab, np.nan, got))


def distill_row(logits, ids, logq, scale=1.0, bucket=True, weight=1.0):
    """(loss, gradient) of one row; ids that are no token, or were there before, are left out."""
    z = np.asarray(logits, np.float64)
    vocab = z.size
    grad = np.zeros(vocab)
    seen = {}
    for i, lq in zip(ids, logq):
        if 0 <= i < vocab and int(i) not in seen:
            seen[int(i)] = float(lq)
    S = np.array(list(seen), np.int64)
    lq = np.array([seen[i] for i in seen], np.float64)
    if weight == 0 or S.size == 0 or (not bucket and lq.max() == -np.inf):
        return 0.0, grad
    if not bucket:
        lq = lq - lq.max()  # (only the differences count)
    q = np.exp(lq)
    Q = q.sum()
    lp = log_softmax(z[None], scale)[0]
    p = np.exp(lp)

    def term(a, la, lb):  # a (ln a - ln b), 0 where a = 0
        return 0.0 if a == 0 else a * (la - lb)

    with np.errstate(invalid="ignore", over="ignore"):
        if not bucket:
            lq, q = lq - np.log(Q), q / Q
            loss = sum(term(a, la, lp[i]) for a, la, i in zip(q, lq, S))
            grad = p.copy()
            grad[S] -= q
        else:
            qt = max(0.0, 1.0 - Q)
            out = np.ones(vocab, bool)
            out[S] = False
            loss = sum(term(a, la, lp[i]) for a, la, i in zip(q, lq, S))
            grad = p.copy()
            # the tail by itself: p_T may be below what float64 holds
            x = z * scale
            most = x[out].max(initial=-np.inf)
            if qt > 0 and most != -np.inf:
                e = np.where(out, np.exp(x - most), 0.0)
                lpt = (most - x.max()) + np.log(e.sum()) - np.log(np.exp(x - x.max()).sum())
                loss += qt * (np.log(qt) - lpt)
                grad -= qt * e / e.sum()
            # (Q + the q_T that counts: 1, but for a tail that is masked altogether.  Above 1 the list is no distribution; the
            # gradient is defined as that of Q = 1)
            grad[S] = (Q if qt > 0 and most == -np.inf else 1.0) * p[S] - q
    return weight * loss, weight * scale * grad


def reveal(ids, cand, score, n_reveal, mask_id, lowest=False, window=None):
    """(ids with the chosen positions' candidates, masked positions that remain)."""
    ids, cand = np.asarray(ids), np.asarray(cand)
    out, left = ids.copy(), np.zeros(ids.shape[0], np.int64)
    for b in range(ids.shape[0]):
        lo, hi = (0, ids.shape[1]) if window is None else (max(window[b][0], 0), min(window[b][1], ids.shape[1]))
        pos = [n for n in range(lo, hi) if ids[b, n] == mask_id]
        s = np.asarray(score[b], np.float64) * (-1.0 if lowest else 1.0)
        s = np.where(np.isnan(s), -np.inf, s)
        pos.sort(key=lambda n: (-s[n], n))
        take = pos[:max(int(n_reveal[b]), 0)]
        out[b, take] = cand[b, take]
        left[b] = int((ids[b] == mask_id).sum()) - len(take)
    return out, left
