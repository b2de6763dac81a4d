"""Log-probabilities of given tokens, entropy, top alternatives and their gradient in 64 bits, written from the definition:
p = softmax(z), logprob = log p[token], entropy = -sum p log p."""
from __future__ import annotations

import numpy as np


def score(z, token=None, top=0):
    """One row: dict of logprob, entropy, max, logsum, top_token, top_logprob."""
    z = np.asarray(z, np.float64)
    if token is not None and token < 0:
        return dict(logprob=0.0, entropy=0.0, max=0.0, logsum=0.0, top_token=[-1] * top, top_logprob=[-np.inf] * top)
    order = [int(i) for i in np.argsort(-np.where(np.isnan(z), -np.inf, z), kind="stable") if z[i] > -np.inf][:top]
    place = order + [-1] * (top - len(order))
    lp = np.nan if token is None or token >= len(z) else None
    if (z == -np.inf).all():
        return dict(logprob=-np.inf if lp is None else lp, entropy=0.0, max=-np.inf, logsum=0.0, top_token=place,
                    top_logprob=[-np.inf] * top)
    if np.isnan(z).any() or (z == np.inf).any():
        m = np.nan if np.isnan(z).all() else np.nanmax(z)
        return dict(logprob=np.nan, entropy=np.nan, max=m, logsum=np.nan, top_token=place,
                    top_logprob=[np.nan if t >= 0 else -np.inf for t in place])
    m = z.max()
    d = z - m
    e = np.exp(d)
    S = e.sum()
    H = np.log(S) - (e[e > 0] * d[e > 0]).sum() / S
    logp = d - np.log(S)
    return dict(logprob=logp[token] if lp is None else lp, entropy=H, max=m, logsum=np.log(S), top_token=place,
                top_logprob=[logp[t] if t >= 0 else -np.inf for t in place])


def grad(z, token, g, gh):
    """d (g logprob + gh entropy) / dz of one row."""
    z = np.asarray(z, np.float64)
    if token is not None and token < 0 or (z == -np.inf).all() and (token is None or token < len(z)):
        return np.zeros(len(z))
    if token is not None and token >= len(z) or np.isnan(z).any() or (z == np.inf).any():
        return np.full(len(z), np.nan)
    d = z - z.max()
    S = np.exp(d).sum()
    p = np.exp(d) / S
    logp = np.where(p > 0, d - np.log(S), 0.0)
    y = -g * p - gh * p * (logp - (p * logp).sum())
    if token is not None:
        y[token] += g
    return y
