"""Gradients of the norms' vectors, whichever are asked for, on inputs whose sums are exact: rows of +-1 (their root mean square is 1), gradients that are small whole numbers,
vectors in halves.  Every token counts once, so each result is one number, to the last bit.  And the scratch of sums does not grow with the tokens."""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr

from stream_helpers import f64

pytestmark = pytest.mark.gpu

# no modulation: one run in one piece, in several; a modulation: runs in pieces, whole runs, many of them to a unit, side by side in a wave
RUNS = {"few": (1, 3, 0), "one": (3, 2003, 0), "pieces": (2, 1500, 700), "whole": (2, 900, 7), "many": (1, 9001, 1), "sides": (3, 1500, 2)}
WANTED = [("weight",), ("bias",), ("scale",), ("shift",), ("weight", "bias"), ("scale", "weight"), ("shift", "bias"), ("scale", "bias"), ("shift", "weight"),
          ("scale", "shift", "weight", "bias")]


def halves(rng, shape, values):
    return torch.from_numpy(rng.choice(values, shape).astype(np.float32))


def spread(v, N, mod_tokens):
    """Rows of a modulation [B, rows, C] (or None: 0) for each token."""
    return v if v is None else v[:, np.arange(N) // (mod_tokens or N)]


def fold(x, mod_tokens):
    """Sums over the tokens of each modulation."""
    N = x.shape[1]
    return np.add.reduceat(x, np.arange(0, N, mod_tokens or N), axis=1)


def ones_stay(C):
    return np.float32(C) * (np.float32(1.0) / np.float32(C)) == np.float32(1.0)


def setup(runs, C, dtype, given, seed):
    B, N, mod_tokens = RUNS[runs]
    assert ones_stay(C)
    rng = np.random.RandomState(seed)
    rows = -(-N // mod_tokens) if mod_tokens else 1
    sign = lambda: halves(rng, (B, N, C), [-1.0, 1.0]).to(dtype)  # noqa: E731
    t, br, dy, dt = sign(), sign(), halves(rng, (B, N, C), [-2, -1, 0, 1, 2]).to(dtype), halves(rng, (B, N, C), [-2, -1, 0, 1, 2]).to(dtype)
    vec = {k: halves(rng, (B, rows, C) if k in ("gate", "scale", "shift") else (C,), [-0.5, 0.5, 1.0, 2.0]) for k in given}
    return (B, N, mod_tokens, rows), (t, br, dy, dt), vec


def new_grads(wanted, B, rows, C):
    return {k: torch.full((B, rows, C) if k in ("gate", "scale", "shift") else (C,), 7.0, device="cuda") for k in wanted}


@pytest.mark.parametrize("runs", list(RUNS))
@pytest.mark.parametrize("C", [5, 64, 128, 640, 1032])
def test_any_of_those_behind_the_norm(runs, C):
    ctx = dr.Context(0)
    for i, (given, dtype) in enumerate(((("scale", "shift", "weight", "bias"), torch.float32), (("scale", "weight", "bias"), torch.bfloat16), (("weight", "bias"), torch.bfloat16), ((), torch.float32))):
        (B, N, mod_tokens, rows), (t, br, dy, dt), vec = setup(runs, C, dtype, given, 10 * i + C)
        norm = dr.NormParams(dr.NORM_RMS, eps=0.0, mod_tokens=mod_tokens)
        v = {k: f64(x) for k, x in vec.items()}
        n, g = f64(t), f64(dy)
        w, b = v.get("weight", np.ones(C)), v.get("bias", np.zeros(C))
        s = 1.0 + (spread(v["scale"], N, mod_tokens) if "scale" in v else 0.0)
        want = dict(shift=fold(g, mod_tokens), scale=fold(g * (n * w + b), mod_tokens), weight=(g * s * n).sum((0, 1)), bias=(g * s).sum((0, 1)))
        held, T, DY = dr.NormVectors(**{k: x.cuda() for k, x in vec.items()}), t.cuda(), dy.cuda()
        dx = first = None
        for wanted in WANTED:
            grads = new_grads(wanted, B, rows, C)
            dx = torch.empty_like(T)
            dr.dr_norm_bwd(ctx, norm, T, DY, dx, vectors=held, grads=dr.NormVectors(**grads))
            for k, got in grads.items():
                assert np.array_equal(f64(got), want[k]), (given, wanted, k)
            first = dx if first is None else first
            if "scale" in given:                                # (else what is asked for decides whether there are modulations)
                assert torch.equal(dx, first)


@pytest.mark.parametrize("runs", list(RUNS))
@pytest.mark.parametrize("C", [5, 64, 128, 640, 1032])
def test_any_of_those_in_front_of_it(runs, C):
    """With dY = 0 the sum's gradient is dtotal: gate, branch_weight, and the branch as it is or normalised."""
    ctx = dr.Context(0)
    for i, (given, branch_norm, dtype) in enumerate(((("gate", "branch_weight"), True, torch.float32), (("gate",), False, torch.bfloat16), (("branch_weight", "scale"), True, torch.bfloat16), ((), True, torch.float32))):
        (B, N, mod_tokens, rows), (t, br, dy, dt), vec = setup(runs, C, dtype, given, 10 * i + C)
        norm = dr.NormParams(dr.NORM_RMS, eps=0.0, mod_tokens=mod_tokens, branch_norm=branch_norm)
        v = {k: f64(x) for k, x in vec.items()}
        d, nb, bw = f64(dt), f64(br), v.get("branch_weight", np.ones(C))
        gate = spread(v["gate"], N, mod_tokens) if "gate" in v else 1.0
        want = dict(gate=fold(d * nb * bw, mod_tokens), branch_weight=(d * gate * nb).sum((0, 1)), bias=np.zeros(C), weight=np.zeros(C))
        held, T, DY, BR, DT = dr.NormVectors(**{k: x.cuda() for k, x in vec.items()}), t.cuda(), torch.zeros_like(dy).cuda(), br.cuda(), dt.cuda()
        for wanted in (("gate",), ("branch_weight",), ("gate", "branch_weight"), ("gate", "bias"), ("branch_weight", "weight")):
            if "branch_weight" in wanted and not branch_norm:
                continue
            grads = new_grads(wanted, B, rows, C)
            dx = torch.empty_like(T)
            dr.dr_norm_bwd(ctx, norm, T, DY, dx, branch=BR, dtotal=DT, vectors=held, grads=dr.NormVectors(**grads))
            for k, got in grads.items():
                assert np.array_equal(f64(got), want[k]), (given, wanted, k)
            assert torch.equal(dx, DT)


@pytest.mark.parametrize("C", [64, 640])
def test_x_in_the_place_of_the_sum(C):
    g = torch.Generator().manual_seed(C)
    t, dy, dt = (torch.randn(2, 300, C, generator=g).bfloat16().cuda() for _ in range(3))
    w = torch.randn(C, generator=g).cuda()
    ctx, norm, vec = dr.Context(0), dr.NormParams(mod_tokens=50), dr.NormVectors(weight=w)
    for dtotal in (None, dt):
        dx, dw, dw2 = torch.empty_like(t), torch.empty_like(w), torch.empty_like(w)
        dr.dr_norm_bwd(ctx, norm, t, dy, dx, dtotal=dtotal, vectors=vec, grads=dr.NormVectors(weight=dw))
        again = t.clone()
        dr.dr_norm_bwd(ctx, norm, again, dy, again, dtotal=dtotal, vectors=vec, grads=dr.NormVectors(weight=dw2))
        assert torch.equal(again, dx) and torch.equal(dw, dw2)


@pytest.mark.parametrize("N,C,mod_tokens", [(60000, 1024, 1), (400000, 64, 1)])
def test_scratch_does_not_grow_with_the_tokens(N, C, mod_tokens):
    """A row of sums (12 C bytes) for each modulation would be 737 and 307 MB; a unit, or a side of a wave, has one, four units for each that the device holds: 101 MB at most."""
    ctx, norm = dr.Context(0), dr.NormParams(dr.NORM_RMS, eps=0.0, mod_tokens=mod_tokens)
    t, dy = torch.ones(1, N, C, dtype=torch.bfloat16, device="cuda"), torch.ones(1, N, C, dtype=torch.bfloat16, device="cuda")
    dx, scale, dw = torch.empty_like(t), torch.zeros(1, N // mod_tokens, C, device="cuda"), torch.empty(C, device="cuda")
    vec, grads = dr.NormVectors(scale=scale), dr.NormVectors(weight=dw)
    dr.dr_norm_bwd(ctx, norm, t[:, :2], dy[:, :2], dx[:, :2], vectors=dr.NormVectors(scale=scale[:, :2 // mod_tokens]), grads=grads)
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    dr.dr_norm_bwd(ctx, norm, t, dy, dx, vectors=vec, grads=grads)
    torch.cuda.synchronize()
    assert before - torch.cuda.mem_get_info()[0] <= 2 ** 27 + 2 ** 21
    assert (dw == N).all()
