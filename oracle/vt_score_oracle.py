"""fp64 definitions of token scoring and of its gradient (numpy, no code shared with the library).

    x = h W^T      z = scale x      lse = log sum_v e^z      logprob = z[t] - lse      H = -sum_v p log p
    G = scale (gl (1[v = t] - p) - ge p (log p + H))         dh = G W               dW = G^T h

A row whose token lies outside [0, V) is not scored: zeros (ids -1), no gradient."""
from __future__ import annotations

import numpy as np


def scored_rows(tokens, M: int, V: int) -> np.ndarray:
    if tokens is None:
        return np.ones(M, bool)
    tokens = np.asarray(tokens, np.int64)
    return (tokens >= 0) & (tokens < V)


def _parts(h, W, scale):
    z = scale * (h @ W.T)
    mx = z.max(1, keepdims=True)
    rest = np.exp(z - mx)
    rest[np.arange(len(z)), z.argmax(1)] = 0.0                         # log(1 + rest) keeps what is left beside a near certain token
    log_s = np.log1p(rest.sum(1))
    lse = mx[:, 0] + log_s
    logp = (z - mx) - log_s[:, None]
    p = np.exp(logp)
    entropy = -(p * np.where(p > 0, logp, 0.0)).sum(1)
    return z, lse, logp, p, entropy


def score(h: np.ndarray, W: np.ndarray, tokens, k: int = 0, scale: float = 1.0) -> dict:
    h, W = np.asarray(h, np.float64), np.asarray(W, np.float64)
    M, V = h.shape[0], W.shape[0]
    keep = scored_rows(tokens, M, V)
    out = {"logprobs": np.zeros(M), "entropy": np.zeros(M), "lse": np.zeros(M),
           "top_ids": np.full((M, k), -1, np.int64), "top_logprobs": np.zeros((M, k))}
    if keep.any():
        z, lse, logp, _, entropy = _parts(h[keep], W, scale)
        out["lse"][keep], out["entropy"][keep] = lse, entropy
        if tokens is not None:
            out["logprobs"][keep] = logp[np.arange(len(z)), np.asarray(tokens, np.int64)[keep]]
        order = np.argsort(-z, axis=1, kind="stable")[:, :k]           # equal logits: the lower id first
        out["top_ids"][keep] = order
        out["top_logprobs"][keep] = np.take_along_axis(logp, order, 1)
    return out


def grad_logits(h, W, tokens, grad_logprobs, grad_entropy=None, scale: float = 1.0):
    """(G, A): the gradient of the logits and the sum of the magnitudes of its terms (what a relative error of p is relative to)."""
    h, W = np.asarray(h, np.float64), np.asarray(W, np.float64)
    M, V = h.shape[0], W.shape[0]
    keep = scored_rows(tokens, M, V)
    G, A = np.zeros((M, V)), np.zeros((M, V))
    if keep.any():
        _, _, logp, p, entropy = _parts(h[keep], W, scale)
        gl = np.asarray(grad_logprobs, np.float64)[keep, None]
        ge = np.zeros_like(gl) if grad_entropy is None else np.asarray(grad_entropy, np.float64)[keep, None]
        hot = np.zeros_like(p)
        hot[np.arange(len(p)), np.asarray(tokens, np.int64)[keep]] = 1.0
        G[keep] = scale * (gl * (hot - p) - ge * p * (logp + entropy[:, None]))
        A[keep] = scale * (np.abs(gl) * (hot + p) + np.abs(ge) * p * np.abs(logp + entropy[:, None]))
    return G, A


def score_backward(h, W, tokens, grad_logprobs, grad_entropy=None, scale: float = 1.0):
    h, W = np.asarray(h, np.float64), np.asarray(W, np.float64)
    G, _ = grad_logits(h, W, tokens, grad_logprobs, grad_entropy, scale)
    keep = scored_rows(tokens, h.shape[0], W.shape[0])
    return G @ W, G[keep].T @ h[keep]                                  # what a row that is not scored holds reaches nothing
