"""fp64 definitions of a draft layer's decode step: rotary positions, tree masks, attention over a paged cache, verification.

Plain loops over numpy float64 and Python floats, written from the formulas; shares no code with ``csrc/``.
"""
from __future__ import annotations

import math

import numpy as np


# ------------------------------------------------------------------------------------------ rotary positions
def rope_frequencies(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, low: float = 1.0, high: float | None = None,
                     original_len: float = 8192.0) -> np.ndarray:
    """Radians per position of each pair."""
    if high is None:
        high = 32.0 if scaling == "ramp" else 4.0
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        w = f
        if scaling == "linear":
            w = f / factor
        elif scaling == "base":
            w = (base * factor ** (rot / (rot - 2.0))) ** (-2.0 * i / rot)
        elif scaling == "wavelength":
            turns = original_len * f / (2 * math.pi)
            s = min(max((turns - low) / (high - low), 0.0), 1.0)
            w = f * s + f / factor * (1 - s)
        elif scaling == "ramp":
            def pair_that_makes(t):
                return rot * math.log(original_len / (2 * math.pi * t)) / (2 * math.log(base))
            i0, i1 = max(math.floor(pair_that_makes(high)), 0), min(math.ceil(pair_that_makes(low)), rot - 1)
            s = min(max((i - i0) / max(i1 - i0, 1e-3), 0.0), 1.0)
            w = f * (1 - s) + f / factor * s
        out.append(w)
    return np.array(out)


def rope(x: np.ndarray, positions: np.ndarray, w: np.ndarray, interleaved: bool = False, amplitude: float = 1.0, inverse: bool = False) -> np.ndarray:
    """x [N, H, D] float64, turned; w from rope_frequencies (its length says how much of the head is)."""
    y = x.copy()
    half = len(w)
    for n, pos in enumerate(positions):
        angle = float(pos) * w
        c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
        if inverse:
            s = -s
        a = np.arange(half) * 2 if interleaved else np.arange(half)
        b = a + 1 if interleaved else a + half
        y[n][:, a] = x[n][:, a] * c - x[n][:, b] * s
        y[n][:, b] = x[n][:, b] * c + x[n][:, a] * s
    return y


# ------------------------------------------------------------------------------------------ trees
def tree_mask(parents, cu, words: int):
    """(mask [N, words] int64 bit patterns, depth [N]); rows outside all requests -1 in depth."""
    N = len(parents)
    mask, depth = np.zeros((N, words), dtype=np.int64), np.full(N, -1, dtype=np.int64)
    for b in range(len(cu) - 1):
        for t in range(cu[b + 1] - cu[b]):
            at, d = t, 0
            while True:
                if at // 32 < words:
                    mask[cu[b] + t, at // 32] |= 1 << (at % 32)
                up = parents[cu[b] + at]
                if not 0 <= up < at:
                    break
                at, d = up, d + 1
            depth[cu[b] + t] = d
    return mask, depth


# ------------------------------------------------------------------------------------------ attention
def attention(q, k, v, table, lens, cu, mask, scale: float, max_tokens: int):
    """q [N, Hq, D], k and v [pages, page, heads, D] float64; mask [N, words] bit patterns or None.

    Returns out [N, Hq, D], lse [N, Hq] and absolute [N, Hq, D] = sum of weights times |v|; rows that are not computed are NaN."""
    N, Hq, D = q.shape
    pages, page, heads = k.shape[:3]
    out, absolute, lse = np.full(q.shape, np.nan), np.full(q.shape, np.nan), np.full((N, Hq), np.nan)
    room = table.shape[1] * page
    for b in range(len(lens)):
        T, L = min(int(cu[b + 1] - cu[b]), max_tokens), min(max(int(lens[b]), 0), room)
        n = min(L + T, room)
        at = np.arange(n)
        ids = table[b, at // page]
        inside = (ids >= 0) & (ids < pages)
        kb, vb = np.zeros((n, heads, D)), np.zeros((n, heads, D))
        kb[inside], vb[inside] = k[ids[inside], at[inside] % page], v[ids[inside], at[inside] % page]
        for t in range(T):
            row = int(cu[b]) + t
            sees = at < L
            for i in range(L, n):
                u = i - L
                sees[i] = u <= t if mask is None else u < 32 * mask.shape[1] and (int(mask[row, u // 32]) >> (u % 32)) & 1
            for h in range(Hq):
                kh = h // (Hq // heads)
                if not sees.any():
                    out[row, h], absolute[row, h], lse[row, h] = 0.0, 0.0, -np.inf
                    continue
                x = scale * (kb[sees, kh] @ q[row, h])
                top = x.max()
                e = np.exp(x - top)
                wgt = e / e.sum()
                lse[row, h] = top + math.log(e.sum())
                out[row, h], absolute[row, h] = wgt @ vb[sees, kh], wgt @ np.abs(vb[sees, kh])
    return out, lse, absolute


# ------------------------------------------------------------------------------------------ verification
def verify(probs, tokens, parents, cu, u_accept, u_sample, max_tokens: int, draft_probs=None, draft_ids=None, d2t=None):
    """(n_accepted [B], path [B, max_tokens], tokens [B, max_tokens]) by the rule, one request after the other."""
    B, V = len(cu) - 1, probs.shape[1]
    n_out, path, out = np.zeros(B, dtype=np.int64), np.full((B, max_tokens), -1), np.full((B, max_tokens), -1)
    for b in range(B):
        T = min(int(cu[b + 1] - cu[b]), max_tokens)
        if T == 0:
            continue
        row = int(cu[b])
        x, taken = 0, []

        def fits(c):
            if not 0 <= parents[row + c] < c or not 0 <= tokens[row + c] < V:
                return False
            return draft_probs is None or 0 <= draft_ids[row + c] < draft_probs.shape[1]

        def full(node):                 # the draft's distribution over the target's ids
            q = np.zeros(V)
            for i, p in enumerate(draft_probs[row + node]):
                to = i if d2t is None else int(d2t[i])
                if 0 <= to < V:
                    q[to] = p
            return q

        while True:
            p = np.maximum(np.nan_to_num(probs[row + x].astype(np.float64), nan=0.0), 0.0)
            q = None if draft_probs is None else np.maximum(full(x), 0.0)
            left, S, Z, step = p.copy(), 0.0, 1.0, None
            for c in range(x + 1, T):
                if not fits(c) or parents[row + c] != x:
                    continue
                y = int(tokens[row + c])
                qc = 1.0 if q is None else max(float(draft_probs[row + x][draft_ids[row + c]]), 0.0)
                if left[y] > 0 and float(u_accept[row + c]) * qc * Z < left[y]:
                    step = c
                    break
                if q is None:
                    Z -= left[y]
                    left[y] = 0.0
                else:
                    S += Z
                    left = np.maximum(p - S * q, 0.0)
                    Z = math.fsum(left)
            if step is None:
                break
            x = step
            taken.append(step)
        if not left.sum() > 0:
            left = p
        target, y, cum = max(float(u_sample[b]), 0.0) * math.fsum(left), -1, 0.0
        for w in np.nonzero(left > 0)[0]:
            cum += left[w]
            y = int(w)
            if cum > target:
                break
        n_out[b] = len(taken)
        path[b, :len(taken)] = taken
        out[b, :len(taken)] = [tokens[row + c] for c in taken]
        out[b, len(taken)] = y
    return n_out, path, out
