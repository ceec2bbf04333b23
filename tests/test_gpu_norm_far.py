"""Norms of fp32 rows far from 0: what a mean costs.  The rows hold exact values, so an error is the kernels' own.

Bound of norm(t), with u = 2^-24, dev the deviation and D = max |t - mean|.  The first mean m is off by q |mean| u at most, q = 50 for the longest chain of sums (16 values a lane, 6 steps in a wave,
16 waves, the products).  Distances to m are exact where t and m lie within a factor of two of each other, as here; o, their sum over C, is known to 50 u times their mean size, which is
below dev + q |mean| u.  The result is rounded a few times (distance, move, root, product): 6 u D / dev, and the root's own bound of 30 u.  So
    error <= u (60 (1 + q |mean| u / dev) + 6 D / dev + 30 D / dev),
and with the mean at 10^5 and dev = 1, q |mean| u = 0.3.  Without o the error is |mean| u itself and more: 6e-3 there.
"""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import layer_oracle as o

from stream_helpers import HALF_BF16, f64

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def bound(t):
    mean, dev = t.mean(-1, keepdims=True), t.std(-1, keepdims=True)
    D = np.abs(t - mean).max(-1, keepdims=True) / dev
    return U * (60 * (1 + 50 * np.abs(mean) * U / dev) + 36 * D)


@pytest.mark.parametrize("C", [5, 64, 128, 200, 256, 512, 513, 640, 1030, 2048, 5120, 8192])
@pytest.mark.parametrize("mean", [-300.0, 1e4, 1e5])
def test_forward_and_gradients(C, mean):
    g = torch.Generator().manual_seed(C)
    x, dy = mean + torch.randn(1, 37, C, generator=g), torch.randn(1, 37, C, generator=g)
    br = mean + torch.randn(1, 37, C, generator=g)
    ctx, X, Y, DX = dr.Context(0), x.cuda(), torch.empty(1, 37, C, device="cuda"), torch.empty(1, 37, C, device="cuda")
    norm = dr.NormParams(eps=0.0)
    t, tb = f64(x), f64(br)
    n = (t - t.mean(-1, keepdims=True)) / t.std(-1, keepdims=True)
    b = bound(t)
    dr.dr_norm_fwd(ctx, norm, X, Y)
    assert (np.abs(f64(Y) - n) <= b).all(), np.abs(f64(Y) - n).max()
    # the branch's norm, alone: T = norm(branch)
    T = torch.empty_like(Y)
    dr.dr_norm_fwd(ctx, dr.NormParams(eps=0.0, branch_norm=True, residual_scale=0.0), X, Y, branch=br.cuda(), total=T)
    nb = (tb - tb.mean(-1, keepdims=True)) / tb.std(-1, keepdims=True)
    assert (np.abs(f64(T) - nb) <= bound(tb) + U).all(), np.abs(f64(T) - nb).max()
    # gradients: a sum of dY n is off by the tokens' bounds and its own roundings; dX by what n is off, twice (n along, and 1 / dev), and some 60 roundings
    dw = torch.empty(C, device="cuda")
    dr.dr_norm_bwd(ctx, norm, X, dy.cuda(), DX, grads=dr.NormVectors(weight=dw))
    d, dev = f64(dy), t.std(-1, keepdims=True)
    want = (d * n).sum((0, 1))
    assert (np.abs(f64(dw) - want) <= (np.abs(d) * (b + 60 * U * np.abs(n))).sum((0, 1))).all()
    along = (d * n).mean(-1, keepdims=True)
    dx = (d - d.mean(-1, keepdims=True) - n * along) / dev
    size = (np.abs(d) + np.abs(d).mean(-1, keepdims=True) + np.abs(n * along)) / dev
    err = (b * np.abs(along) + np.abs(n) * ((np.abs(d) * b).mean(-1, keepdims=True) + 50 * U * np.abs(d * n).mean(-1, keepdims=True))) / dev + 96 * U * size
    assert (np.abs(f64(DX) - dx) <= err).all(), np.abs(f64(DX) - dx).max()


@pytest.mark.parametrize("C", [64, 512, 5120])
def test_bf16_rows_keep_to_their_rounding(C):
    """Values that bf16 tells apart lie 2^-8 of the mean or more from each other; the mean without o is off by 50 u |mean| at most."""
    x = (300.0 + 4.0 * torch.randn(1, 37, C, generator=torch.Generator().manual_seed(C))).bfloat16()
    Y = torch.empty(1, 37, C, dtype=torch.bfloat16, device="cuda")
    dr.dr_norm_fwd(dr.Context(0), dr.NormParams(eps=0.0), x.cuda(), Y)
    t = f64(x)
    mean, dev = t.mean(-1, keepdims=True), t.std(-1, keepdims=True)
    n = (t - mean) / dev
    e = bound(t) + 50 * U * np.abs(mean) / dev
    assert (np.abs(f64(Y) - n) <= e + HALF_BF16 * (np.abs(n) + e)).all()


def test_values_far_apart_in_a_row():
    """Parts of a row at different heights: means of the waves' parts far from each other."""
    g = torch.Generator().manual_seed(0)
    x = torch.randn(1, 9, 5120, generator=g)
    x[..., :512] += 1e5
    x[..., 4096:] -= 3e3
    X, Y = x.cuda(), torch.empty(1, 9, 5120, device="cuda")
    dr.dr_norm_fwd(dr.Context(0), dr.NormParams(eps=0.0), X, Y)
    _, y, _, e = o.forward(f64(x), None, {}, "layer", 0.0, 1.0, 0, False)
    assert (np.abs(f64(Y) - y) <= e).all()
