"""fp64 definitions of the vocabulary operators: embedding lookup and its gradient, log-probabilities of given tokens
from logits (entropy, log-sum-exp, top alternatives) and their gradient, and the same from hidden states and the
head's weight.  A token below zero or at / above the vocabulary marks a row without values and without gradient."""
import numpy as np


def _live(tok, vocab):
    tok = np.asarray(tok, dtype=np.int64)
    return tok, (tok >= 0) & (tok < vocab)


def embed(table, tok, scale=1.0):
    table = np.asarray(table, dtype=np.float64)
    tok, live = _live(tok, table.shape[0])
    out = np.zeros((tok.size, table.shape[1]))
    out[live] = table[tok[live]] * scale
    return out


def embed_bwd(dout, tok, vocab, scale=1.0):
    dout = np.asarray(dout, dtype=np.float64)
    tok, live = _live(tok, vocab)
    grad = np.zeros((vocab, dout.shape[1]))
    np.add.at(grad, tok[live], dout[live] * scale)
    return grad


def row_statistics(z):
    """(lse, entropy, p, log p) of one row of scaled logits.  Nothing but -inf: lse -inf, entropy 0, p 0."""
    z = np.asarray(z, dtype=np.float64)
    if np.isnan(z).any() or np.isposinf(z).any():
        nan = np.full_like(z, np.nan)
        return np.nan, np.nan, nan, nan
    m = z.max()
    if m == -np.inf:
        return -np.inf, 0.0, np.zeros_like(z), np.full_like(z, -np.inf)
    e = np.exp(z - m)
    lse = m + np.log(e.sum())
    p = e / e.sum()
    lp = (z - m) - np.log(e.sum())                             # not z - lse: large logits would swallow the logarithm
    entropy = -np.sum(p[p > 0] * lp[p > 0])
    return lse, entropy, p, lp


def top_ids(row, k):
    """The k largest values of a row, a NaN above +inf, the lowest index first among equal ones."""
    row = np.asarray(row, dtype=np.float64)
    order = sorted(range(row.size), key=lambda i: ((0, 0.0) if np.isnan(row[i]) else (1, -row[i]), i))
    return order[:k]


def token_logp(logits, tok, temperature=1.0, top=0):
    logits = np.asarray(logits, dtype=np.float64)
    n, vocab = logits.shape
    tok, live = _live(np.zeros(n) if tok is None else tok, vocab)
    out = {"logp": np.zeros(n), "entropy": np.zeros(n), "lse": np.zeros(n),
           "top_id": np.full((n, top), -1, dtype=np.int64), "top_logp": np.zeros((n, top))}
    for i in np.nonzero(live)[0]:
        lse, ent, _, lp = row_statistics(logits[i] / temperature)
        out["logp"][i], out["entropy"][i], out["lse"][i] = lp[tok[i]], ent, lse
        out["top_id"][i] = top_ids(logits[i], top)
        out["top_logp"][i] = lp[out["top_id"][i]]
    return out


def token_logp_bwd(logits, tok, dlogp, dentropy=None, temperature=1.0):
    logits = np.asarray(logits, dtype=np.float64)
    n, vocab = logits.shape
    tok, live = _live(tok, vocab)
    grad = np.zeros((n, vocab))
    for i in np.nonzero(live)[0]:
        lse, ent, p, lp = row_statistics(logits[i] / temperature)
        if lse == -np.inf:
            continue
        h = 0.0 if dentropy is None else float(dentropy[i])
        g = -p * float(dlogp[i])
        on = p > 0
        g[on] -= h * p[on] * (lp[on] + ent)
        g[tok[i]] += float(dlogp[i])
        grad[i] = g / temperature if not np.isnan(lse) else np.nan
    return grad


def head_logp(x, w, tok, temperature=1.0):
    return token_logp(np.asarray(x, dtype=np.float64) @ np.asarray(w, dtype=np.float64).T, tok, temperature)


def head_logp_bwd(x, w, tok, dlogp, dentropy=None, temperature=1.0):
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    dz = token_logp_bwd(x @ w.T, tok, dlogp, dentropy, temperature)
    return dz @ w, dz.T @ x
