"""CPU fp64 oracle of the norms between blocks, with bounds of what fp32 arithmetic may be off by.

Written from the definitions in include/dynamicrad.h; shares no code with the GPU path.  The bounds count roundings of u = 2^-24, to first order in u: a sum over C channels
or L tokens in any tree of at most `depth` additions in a row is off by depth * u times the sum of the magnitudes.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24


def normed(t, kind, eps, e):
    """(norm(t), 1 / deviation, bound of the first, relative bound of the second) over the last axis; `e`: bound of t itself."""
    C = t.shape[-1]
    depth = 48                                             # 8 channels a lane, 6 steps in a wave, 16 waves, and the products
    mean = t.mean(-1, keepdims=True) if kind == "layer" else np.zeros_like(t[..., :1])
    d = t - mean
    ed = e + U * np.abs(d)
    if kind == "layer":
        ed = ed + e.mean(-1, keepdims=True) + depth * U * np.abs(t).mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    n = d * r
    # variance + eps: 2 sum |d| ed / C, the sum's own roundings, those of 1 / C and eps; half of it for the root, then root, division, product
    rel = 0.5 * (2.0 * (np.abs(d) * ed).mean(-1, keepdims=True) * r * r + (depth + 4) * U) + 3 * U
    return n, r, ed * r + np.abs(n) * (rel + U), rel


def _by_row(v, N, mod_tokens, empty):
    if v is None:
        return empty
    return v[:, np.arange(N) // (mod_tokens or max(N, 1))]


def forward(x, branch, vec, kind, eps, rscale, mod_tokens, branch_norm):
    """T, Y, and their bounds (without the rounding of the results)."""
    B, N, C = x.shape
    one = lambda k, v: np.full((1, 1, C), v) if vec.get(k) is None else vec[k]  # noqa: E731
    gate, scale, shift = (_by_row(vec.get(k), N, mod_tokens, np.full((1, 1, C), v)) for k, v in (("gate", 1.0), ("scale", 0.0), ("shift", 0.0)))
    t = rscale * x
    e = 2 * U * np.abs(t)
    if branch is not None:
        b, eb = branch, 0.0 * branch
        if branch_norm:
            n, _, en, _ = normed(branch, kind, eps, eb)
            b = n * one("branch_weight", 1.0)
            eb = en * np.abs(one("branch_weight", 1.0)) + U * np.abs(b)
        t = t + gate * b
        e = e + np.abs(gate) * eb + U * np.abs(t)
    n, _, en, _ = normed(t, kind, eps, e)
    mul, add = one("weight", 1.0) * (1 + scale), one("bias", 0.0) * (1 + scale) + shift
    y = n * mul + add
    bound = en * np.abs(mul) + 3 * U * np.abs(n * mul) + U * np.abs(y) + 3 * U * (np.abs(one("bias", 0.0) * (1 + scale)) + np.abs(add))
    return t, y, e, bound


def backward(t, branch, dy, dtotal, vec, kind, eps, rscale, mod_tokens, branch_norm):
    """{name: (gradient, bound)}: x, branch, gate, scale, shift, weight, bias, branch_weight."""
    B, N, C = t.shape
    depth = 48
    one = lambda k, v: np.full((1, 1, C), v) if vec.get(k) is None else vec[k]  # noqa: E731
    gate, scale = (_by_row(vec.get(k), N, mod_tokens, np.full((1, 1, C), v)) for k, v in (("gate", 1.0), ("scale", 0.0)))
    w, bias, bw = one("weight", 1.0), one("bias", 0.0), one("branch_weight", 1.0)
    step = mod_tokens or max(N, 1)
    rows = -(-N // step)

    def pull(n, r, en, rel, g, eg):
        """The gradient in front of a norm, and its bound."""
        along = (g * n).mean(-1, keepdims=True)
        ea = (eg * np.abs(n) + np.abs(g) * en).mean(-1, keepdims=True) + (depth + 2) * U * np.abs(g * n).mean(-1, keepdims=True)
        m = g.mean(-1, keepdims=True) if kind == "layer" else 0.0 * along
        em = eg.mean(-1, keepdims=True) + depth * U * np.abs(g).mean(-1, keepdims=True) if kind == "layer" else 0.0 * along
        d = r * (g - m - n * along)
        e = r * (eg + em + en * np.abs(along) + np.abs(n) * ea + 3 * U * (np.abs(g) + np.abs(m) + np.abs(n * along))) + (rel + U) * np.abs(d)
        return d, e

    def by_row(x, e):
        """Sums over the tokens of each modulation: their bound counts each token as one addition in a row."""
        s, b = np.zeros((B, rows, C)), np.zeros((B, rows, C))
        for i in range(rows):
            part = slice(i * step, min((i + 1) * step, N))
            s[:, i] = x[:, part].sum(1)
            b[:, i] = e[:, part].sum(1) + (min(step, N) + 80) * U * np.abs(x[:, part]).sum(1)
        return s, b

    def over_all(x, e):
        return x.sum((0, 1)), e.sum((0, 1)) + (B * N + 160) * U * np.abs(x).sum((0, 1))

    out = {}
    n, r, en, rel = normed(t, kind, eps, 0.0 * t)
    a = n * w + bias
    out["shift"] = by_row(dy, 0.0 * dy)
    out["scale"] = by_row(dy * a, np.abs(dy) * (en * np.abs(w) + 4 * U * (np.abs(n * w) + np.abs(bias))))
    s = 1.0 + scale
    out["weight"] = over_all(dy * s * n, np.abs(dy * s) * (en + 4 * U * np.abs(n)))
    out["bias"] = over_all(dy * s, 4 * U * np.abs(dy * s))
    g = dy * s * w
    d, e = pull(n, r, en, rel, g, 4 * U * np.abs(g))
    if dtotal is not None:
        d = d + dtotal
        e = e + U * np.abs(d)
    out["x"] = rscale * d, abs(rscale) * e + 2 * U * np.abs(rscale * d)
    if branch is not None:
        b, eb, nb = branch, 0.0 * branch, branch
        if branch_norm:
            nb, rb, enb, relb = normed(branch, kind, eps, 0.0 * branch)
            b, eb = nb * bw, enb * np.abs(bw)
        out["gate"] = by_row(d * b, e * np.abs(b) + np.abs(d) * eb + 3 * U * np.abs(d * b))
        d, e = d * gate, e * np.abs(gate) + U * np.abs(d * gate)
        if branch_norm:
            out["branch_weight"] = over_all(d * nb, e * np.abs(nb) + np.abs(d) * enb + 3 * U * np.abs(d * nb))
            d, e = pull(nb, rb, enb, relb, d * bw, e * np.abs(bw) + U * np.abs(d * bw))
        out["branch"] = d, e
    return out
