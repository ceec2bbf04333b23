"""Shared plumbing of the streaming operators' tests: batches, caches filled by the oracle's rounding, tolerances."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2604_20470_amd as dr
from oracle import streaming_oracle as o

F8 = torch.float8_e4m3fn
HALF_BF16, ULP32 = 2.0 ** -8, 2.0 ** -24        # a rounding's largest relative error


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def codes(t):
    return t.detach().view(torch.uint8).cpu().numpy()


def batch_arrays(new, lens, P, pages, seed=0, spare=1, width=None):
    """cu, lens, page table (distinct pages in no order) as numpy int32."""
    rng = np.random.RandomState(seed)
    need = [-(-max(n, 0) // P) for n in lens]
    width = max(need) + spare if width is None else width
    ids, at = rng.permutation(pages), 0
    table = np.zeros((len(new), width), np.int32)
    for s, n in enumerate(need):
        n = min(n, width)
        table[s, :n] = ids[at:at + n]
        at += n
    assert at <= pages
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32), np.array(lens, np.int32), table


def on_gpu(*arrays):
    return [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


def filled_cache(pages, H, P, d, seed, spread=3):
    """Random codes without NaN, scales of 2^-spread .. 2^spread beside 1/32 (so that values are of order one)."""
    rng = np.random.RandomState(seed)
    k, v = (rng.randint(0, 256, s).astype(np.uint8) for s in ((pages, H, P, d), (pages, H, d, P)))
    for c in (k, v):
        c[(c & 0x7f) == 0x7f] = 0x38
        big = (c & 0x7f) > 0x50                 # fewer large values: most weights stay within a few orders of magnitude
        c[big] = (c[big] & 0x80) | rng.randint(0, 0x50, int(big.sum())).astype(np.uint8)
    ks, vs = (2.0 ** (-1 - rng.randint(0, spread, (pages, H))) for _ in range(2))
    return k, v, ks.astype(np.float32), vs.astype(np.float32)


def gpu_cache(k, v, ks, vs):
    k, v, ks, vs = on_gpu(k, v, ks, vs)
    return dr.PagedCache.of(k.view(F8), v.view(F8), ks, vs)


def attend_tolerance(q, k, v, ks, vs, cu, lens, table, causal, bf16):
    """(o, lse, tolerance of o, tolerance of lse) from the oracle.  With A = the largest sum |q||k| / sqrt(d) of a row, a logit's sum of
    d products is off by at most (d + 4) roundings of A, so a weight by twice that; sums of n weights by n / 8 + 32 roundings (a
    lane adds every sixteenth); bf16: one rounding of every weight and one of the result."""
    want, lse = o.attend(q, k, v, ks, vs, cu, lens, table, causal)
    weighted, _ = want, lse
    mags = np.abs(o.decode(v)) * vs.astype(np.float64)[:, :, None, None]
    d = q.shape[2]
    kmax = np.nanmax(np.sqrt(np.nansum((o.decode(k) * ks.astype(np.float64)[:, :, None, None]) ** 2, -1)))
    A = np.sqrt((q ** 2).sum(-1)) * kmax / math.sqrt(d)                          # [T, Hq], by Cauchy and Schwarz
    n = table.shape[1] * k.shape[2]
    rel = 2 * (d + 4) * ULP32 * A + (n / 8 + 32) * 2 * ULP32 + 4 * ULP32 * A
    top = np.nanmax(mags)
    tol = rel[..., None] * top * np.ones_like(want)
    if bf16:
        # the weighted mean of |v| through the same softmax
        pos = np.where(o.decode(v) < 0, v & 0x7f, v)
        absmean, _ = o.attend(q, k, pos, ks, vs, cu, lens, table, causal)
        tol = tol + HALF_BF16 * absmean + HALF_BF16 * np.abs(want)
    else:
        tol = tol + 2 * ULP32 * np.abs(want)
    ltol = (rel + 4 * ULP32 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0)).T)).T
    return want, lse, tol, ltol


def assert_close(got, want, tol, what):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    same = (np.isnan(got) & np.isnan(want)) | (np.isinf(want) & (got == want))
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - want) <= tol))
    if bad.any():
        i = np.unravel_index(np.argmax(bad), bad.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} off, first at {i}: {got[i]!r} for {want[i]!r}, tolerance {np.broadcast_to(tol, want.shape)[i]!r}")
