"""CPU fp64 oracle of the streaming operators: rotary positions, the paged e4m3 cache, attention over it.

Written from the definitions in include/dynamicrad.h, token by token and page by page; shares no code with the GPU path.
"""
from __future__ import annotations

import math

import numpy as np

LEAST_EXP = -100


# ---- rotary positions --------------------------------------------------------------------------------------

def frequencies(dim, axis_pairs, theta=10000.0, factor=1.0, original_len=0.0, ramp_low=1.0, ramp_high=32.0):
    """[(axis, radians per unit of position)] of the dim / 2 pairs."""
    out = []
    for a, n in enumerate(axis_pairs):
        for j in range(n):
            f = theta ** (-j / n)
            if a == 0 and factor != 1.0:
                if original_len > 0:
                    r = (original_len * f / (2 * math.pi) - ramp_low) / (ramp_high - ramp_low)
                    r = min(1.0, max(0.0, r))
                    f = f * ((1 - r) / factor + r)
                else:
                    f = f / factor
            out.append((a, f))
    assert len(out) == dim // 2
    return out


def rope(x, positions, dim, layout="half", axis_pairs=None, mscale=1.0, backward=False, **scaling):
    """x [..., N, d] float64; positions int [axes, N]."""
    y = np.array(x, dtype=np.float64)
    for i, (a, f) in enumerate(frequencies(dim, axis_pairs or [dim // 2], **scaling)):
        phi = np.asarray(positions[a], dtype=np.float64) * f
        c, s = np.cos(phi), np.sin(phi) * (-1 if backward else 1)
        p, q = (i, i + dim // 2) if layout == "half" else (2 * i, 2 * i + 1)
        y[..., p] = mscale * (x[..., p] * c - x[..., q] * s)
        y[..., q] = mscale * (x[..., q] * c + x[..., p] * s)
    return y


# ---- e4m3 --------------------------------------------------------------------------------------------------

def _table():
    v = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        x = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        v[c] = math.nan if c & 127 == 127 else (-x if s else x)
    return v


E4M3 = _table()


def decode(codes):
    return E4M3[np.asarray(codes, dtype=np.uint8)]


def encode(x):
    """Nearest code, ties to the even one; beyond +-448 saturates; NaN is 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    grid = E4M3[:127]
    a = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), 448.0)
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    dl, dh = a - grid[lo], grid[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(x), 0x7f, code | (np.signbit(x) << 7)).astype(np.uint8)


def canonical(codes):
    """Codes with both NaN codes as one."""
    c = np.array(codes, dtype=np.uint8)
    c[(c & 0x7f) == 0x7f] = 0x7f
    return c


def exponent(amax):
    """Smallest integer e >= LEAST_EXP with amax <= 448 * 2^e."""
    e = LEAST_EXP
    if amax > 0:
        e = max(LEAST_EXP, math.frexp(amax)[1] - 10)          # amax < 2^frexp: at this e, amax < 1024 * 2^e
        while amax > 448.0 * 2.0 ** e:
            e += 1
    return e


# ---- the cache ---------------------------------------------------------------------------------------------

def append(codes, scales, values, cu, lens, table, tokens_inner):
    """values [T, H, d] (what is to be stored, in the fp32 that the operator holds) into codes [pages, H, P, d], or [pages, H, d, P]
    where tokens_inner; returns new codes (NaN as 0x7f only where written) and scales."""
    codes, scales = np.array(codes, dtype=np.uint8), np.array(scales, dtype=np.float64)
    c = codes.transpose(0, 1, 3, 2) if tokens_inner else codes               # a view: [pages, H, P, d]
    pages, H, P, d = c.shape
    T = values.shape[0]
    for s in range(len(lens)):
        a, b = max(0, min(int(cu[s]), T)), max(0, min(int(cu[s + 1]), T))
        n = b - a
        places = [int(lens[s]) - n + i for i in range(max(n, 0))]
        for index in sorted({p // P for p in places if p >= 0}):
            if index >= table.shape[1] or not 0 <= table[s, index] < pages:
                continue
            page = table[s, index]
            rows = [i for i, p in enumerate(places) if p >= 0 and p // P == index]
            slots = [places[i] % P for i in rows]
            for h in range(H):
                new = np.asarray(values[[a + i for i in rows], h], dtype=np.float64)
                fine = np.abs(new[np.isfinite(new)])
                e = exponent(fine.max() if fine.size else 0.0)
                if slots[0] > 0:
                    old = int(math.log2(scales[page, h]))
                    if old > e:
                        e = old
                    elif e > old:
                        kept = c[page, h, :slots[0]]
                        c[page, h, :slots[0]] = encode(decode(kept) * 2.0 ** (old - e))
                c[page, h, slots] = encode(new / 2.0 ** e)
                scales[page, h] = 2.0 ** e
    return codes, scales


def attend(q, k, v, k_scale, v_scale, cu, lens, table, causal):
    """q [T, Hq, d] float64; codes k [pages, H, P, d], v [pages, H, d, P]; returns o [T, Hq, d], lse [Hq, T], NaN where no sequence
    has the token."""
    T, Hq, d = q.shape
    pages, H, P, _ = k.shape
    G = Hq // H
    o, lse = np.full((T, Hq, d), np.nan), np.full((Hq, T), np.nan)
    for s in range(len(lens)):
        a, b = max(0, min(int(cu[s]), T)), max(0, min(int(cu[s + 1]), T))
        n, length = b - a, int(lens[s])
        keys = [j for j in range(max(0, min(length, table.shape[1] * P))) if 0 <= table[s, j // P] < pages]
        at = np.array(keys, dtype=np.int64)
        page, slot = (table[s, at // P], at % P) if len(keys) else (at, at)
        for h in range(H):
            K = decode(k[page, h, slot]) * k_scale[page, h, None].astype(np.float64)
            V = decode(v[page, h, :, slot]) * v_scale[page, h, None].astype(np.float64)
            for i in range(max(n, 0)):
                sees = at <= length - n + i if causal else np.ones(len(keys), bool)
                for g in range(h * G, (h + 1) * G):
                    if not sees.any():
                        o[a + i, g], lse[g, a + i] = 0.0, -math.inf
                        continue
                    x = K[sees] @ q[a + i, g] / math.sqrt(d)
                    m = x.max()
                    p = np.exp(x - m)
                    o[a + i, g] = p @ V[sees] / p.sum()
                    lse[g, a + i] = m + math.log(p.sum())
    return o, lse
