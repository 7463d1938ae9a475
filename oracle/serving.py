"""Cache append, attention and sampling (oracle, test-only), in float64.

Written from the operators' definitions in the library's header; plain loops
over sequences, pages and heads.  Attention and rotation follow the usual
formulas of a decoder layer (Sec. 5.1 leaves them to the served model); the
sampling weights are whole numbers fixed by a sequence of float32 operations,
which numpy repeats step by step.
"""

import math

import numpy as np


def rope_f64(positions, dim, base=1e6):
    """(cos, sin) float64 [n, dim / 2] of the rotation angles."""
    angle = np.outer(np.asarray(positions, np.float64), base ** (-np.arange(0, dim, 2) / dim))
    return np.cos(angle), np.sin(angle)


def norm_and_rotate(x, weight, eps, positions, base=1e6):
    """x [n, heads, dim] -> float64, RMS norm of each head (weight or None), then rotation."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    if positions is None:
        return x
    c, s = rope_f64(positions, x.shape[-1], base)
    a, b = np.split(x, 2, -1)
    c, s = c[:, None], s[:, None]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def page_tokens_of(k, v, scales, page, which):
    """The values a page stands for, float64 [heads, page_tokens, dim]."""
    q = k[page] if which == 0 else v[page].transpose(0, 1, 3, 2).reshape(k.shape[1:])
    return q.astype(np.float64) * scales[page, :, which].astype(np.float64)[:, None, None]


def sequence(k, v, scales, pages, n):
    """float64 keys and values [n, heads, dim] of a sequence, and which tokens have a page."""
    B = k.shape[2]
    ks, vs = np.zeros((n,) + (k.shape[1], k.shape[3])), np.zeros((n,) + (k.shape[1], k.shape[3]))
    there = np.zeros(n, bool)
    for j in range(-(-n // B)):
        if j >= len(pages) or not 0 <= pages[j] < k.shape[0]:
            continue
        lo, hi = j * B, min(n, (j + 1) * B)
        ks[lo:hi] = page_tokens_of(k, v, scales, pages[j], 0).transpose(1, 0, 2)[:hi - lo]
        vs[lo:hi] = page_tokens_of(k, v, scales, pages[j], 1).transpose(1, 0, 2)[:hi - lo]
        there[lo:hi] = True
    return ks, vs, there


def attend(q, ks, vs, there, first, scale, window):
    """(out, sum of weights times |v|) float64 [rows, q_heads, dim] for rows at positions first.. of a
    sequence with keys and values [n, heads, dim]."""
    rows, heads, dim = q.shape
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    group = heads // ks.shape[1]
    token = np.arange(ks.shape[0])
    for i in range(rows):
        p = first + i
        seen = there & (token <= p)
        if window > 0:
            seen &= token > p - window
        if not seen.any():
            continue
        for h in range(heads):
            s = ks[seen, h // group] @ q[i, h].astype(np.float64) * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ vs[seen, h // group]
            size[i, h] = w @ np.abs(vs[seen, h // group])
    return out, size


def weights(x, temperature):
    """Whole sampling weights (int64) of a row of float32 logits without NaN, -inf to +inf, not all -inf."""
    f32 = np.float32
    with np.errstate(all="ignore"):
        top = x.max()
        inverse = f32(math.log2(math.e)) / f32(temperature)
        t = np.where(x == top, f32(0), (x - top) * inverse).astype(f32)
        t = np.maximum(t, f32(-64))
        whole = np.rint(t)
        f = t - whole
        p = np.full_like(f, f32(math.log(2) ** 7 / math.factorial(7)))
        for n in range(6, -1, -1):
            p = p * f + f32(math.log(2) ** n / math.factorial(n))
        assert p.dtype == f32
    return np.floor(np.ldexp(p.astype(np.float64), whole.astype(np.int64) + 40)).astype(np.int64)


def sample(x, temperature, top_k, top_p, min_p, u):
    """The token of one row of float32 logits."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float32)).astype(np.float32)
    n = len(x)
    if np.all(x == -np.inf):
        return -1
    if not temperature > 0:
        return int(np.argmax(x))
    w = weights(x, temperature)
    order = np.argsort(-x.astype(np.float64), kind="stable")
    if 0 < top_k < n:
        order = order[:top_k]
    if top_p < 1:
        total = int(w[order].sum())
        need = max(1, math.ceil(float(np.float32(top_p)) * float(total)))
        above = np.cumsum(w[order]) - w[order]
        order = order[above < need]
    keep = np.zeros(n, bool)
    keep[order] = True
    keep &= w.astype(np.float64) >= min(max(float(np.float32(min_p)), 0.0), 1.0) * 2.0 ** 40
    w = np.where(keep, w, 0)
    total = int(w.sum())
    point = min(int(math.floor(float(np.float32(u)) * float(total))), total - 1)
    return int(np.searchsorted(np.cumsum(w), point, side="right"))
