"""Attention weights of cached tokens, eviction by them and log probabilities (oracle, test-only), in float64.

Written from the operators' definitions in the library's header; plain loops
over sequences, rows and heads.  What an eviction rounds again it rounds in the
two float32 steps that the header names, so pages can be compared byte by byte.
"""

import numpy as np


def weigh(q, ks, there, first, scale, window):
    """(weights, their error's size) float64 [kv_heads, tokens]: what the rows q [rows, q_heads, dim] at positions
    first.. give to the tokens of a sequence with keys [tokens, kv_heads, dim].  The size is the sum of every weight
    times the largest sum |q k| * scale that its row met."""
    rows, heads, _ = q.shape
    n, kv_heads = ks.shape[:2]
    group, token = heads // kv_heads, np.arange(n)
    out, size = np.zeros((kv_heads, n)), np.zeros((kv_heads, n))
    for i in range(rows):
        seen = there & (token <= first + i)
        if window > 0:
            seen &= token > first + i - window
        if not seen.any():
            continue
        for h in range(heads):
            x = q[i, h].astype(np.float64)
            s = ks[seen, h // group] @ x * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            largest = (np.abs(ks[seen, h // group]) @ np.abs(x)).max() * abs(scale)
            out[h // group, seen] += w
            size[h // group, seen] += w * largest
    return out, size


def choose(mass, n, kept, recent):
    """The tokens that stay of a head's first n, in order (mass float32, as many places as there are)."""
    kept = min(max(kept, 0), n)
    last = min(recent, kept)
    m = np.zeros(n, np.float32)
    m[:min(n, len(mass))] = mass[:n]
    m = np.where(np.isnan(m), -np.inf, m)[:n - last]
    heavy = np.sort(np.argsort(-m.astype(np.float64), kind="stable")[:kept - last])
    return np.concatenate([heavy, np.arange(n - last, n)]).astype(np.int64)


def moved(q, scales):
    """Whole numbers [tokens, dim] of one new page from tokens of the scales [tokens] (float32): them and its scale."""
    top = np.float32(scales.max())
    ratio = np.where(top > 0, scales.astype(np.float32) / (top if top > 0 else np.float32(1)), np.float32(0)).astype(np.float32)
    return np.rint(q.astype(np.float32) * ratio[:, None]).astype(np.int8), top


def log_probs(x, temperature, tokens, top):
    """(log probabilities, entropy, spread, tokens, theirs) of one row of logits; the spread sum p (1 + |t|)^2 is what
    the entropy's error goes by."""
    x = np.asarray(x).astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    t0 = float(temperature)
    t0 = t0 if t0 > 0 else 1.0
    m = x.max()
    if m == -np.inf:
        return np.full(len(tokens), -np.inf), 0.0, 0.0, np.full(top, -1), np.full(top, -np.inf)
    with np.errstate(invalid="ignore"):
        # an infinite temperature leaves what is above -inf alike, and -inf out
        t = np.where(x == m, 0.0, np.where(x == -np.inf, -np.inf, (x - m) / t0))
    e = np.exp(t)
    log_l = np.log(e.sum())
    logs = t - log_l
    p = e / e.sum()
    live = p > 0
    entropy = float(-(p[live] * logs[live]).sum())
    spread = float((p[live] * (1 + np.abs(t[live])) ** 2).sum())
    given = np.array([logs[j] if 0 <= j < len(x) else -np.inf for j in tokens])
    order = np.argsort(-x, kind="stable")[:top]
    order = order[x[order] > -np.inf]
    pad = top - len(order)
    return given, entropy, spread, np.concatenate([order, np.full(pad, -1)]), np.concatenate([logs[order], np.full(pad, -np.inf)])
