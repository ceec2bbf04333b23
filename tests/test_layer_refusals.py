"""What the binding of the norms and of the other views of the cache refuses before the library is called (no GPU needed), and the oracle's norm against plain loops."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import layer_oracle as o


class _Ctx:
    """Stands for a context of device 0; any call that gets through the binding's checks fails the test."""
    device, _h = 0, C.c_void_p(1)

    def __init__(self):
        self._lib = type("L", (), {n: staticmethod(lambda *a: pytest.fail("the library was called")) for n in
                                   ("dr_norm_fwd", "dr_norm_bwd", "dr_cache_read", "dr_cache_attn_window_fwd", "dr_cache_attn_shared_fwd")})()


def test_vectors_must_fit_together():
    m, w = torch.ones(2, 3, 8), torch.ones(8)
    dr.NormVectors(gate=m, weight=w)
    for bad in (dict(gate=m, weight=w.bfloat16()), dict(gate=w), dict(weight=m), dict(scale=m.transpose(1, 2)), dict(bias=torch.ones(16)[::2]), dict(shift=m.half()),
                dict(weight=w.double()), dict(gate=m, scale=m[:, :1]), dict(weight=w, bias=w[:4])):
        with pytest.raises(dr.DRError):
            dr.NormVectors(**bad)


def test_tensors_of_another_form_are_refused():
    ctx, x, w = _Ctx(), torch.zeros(2, 4, 8), torch.ones(8)
    norm = dr.NormParams(mod_tokens=2)
    V = dr.NormVectors
    for bad in (lambda: dr.dr_norm_fwd(ctx, norm, x, x), lambda: dr.dr_norm_fwd(ctx, norm, x, x[:, :2]), lambda: dr.dr_norm_fwd(ctx, norm, x, x.bfloat16()),
                lambda: dr.dr_norm_fwd(ctx, norm, x[0], x[0]), lambda: dr.dr_norm_fwd(ctx, norm, x.half(), x.half()),
                lambda: dr.dr_norm_fwd(ctx, norm, x, x, vectors=V(weight=w[:4])), lambda: dr.dr_norm_fwd(ctx, norm, x, x, vectors=V(scale=torch.ones(2, 1, 8))),
                lambda: dr.dr_norm_fwd(ctx, norm, x, x.transpose(1, 2).contiguous().transpose(1, 2)), lambda: dr.dr_norm_bwd(ctx, norm, x, x, x, branch=x[:1]),
                lambda: dr.dr_norm_bwd(ctx, norm, x, x, x, grads=V(weight=w.bfloat16()))):
        with pytest.raises(dr.DRError):
            bad()


def test_views_of_the_cache_refuse_what_does_not_fit():
    ctx, i32 = _Ctx(), lambda *s: torch.zeros(s, dtype=torch.int32)
    cache, batch = dr.PagedCache(2, 2, 32, 64, device="cpu"), dr.CacheBatch(i32(2), i32(1), i32(1, 1), 3)
    q = torch.zeros(3, 4, 64)
    for bad in (lambda: dr.dr_cache_read(ctx, cache, batch, q[:, :2], q[:, :2].clone()), lambda: dr.dr_cache_read(ctx, cache, batch, q[:2, :2]),
                lambda: dr.dr_cache_attn_window_fwd(ctx, cache, batch, q, q.clone(), 5), lambda: dr.dr_cache_attn_window_fwd(ctx, cache, batch, q, q[:2], 5),
                lambda: dr.dr_cache_attn_shared_fwd(ctx, cache, batch, batch, q, q.clone()), lambda: dr.dr_cache_attn_shared_fwd(ctx, cache, batch, batch, q.half(), q.half())):
        with pytest.raises(dr.DRError):
            bad()
    dr.dr_cache_read(ctx, cache, batch)             # nothing is wanted


def test_struct_layouts_match_the_header():
    from paper_2604_20470_amd import binding as bd
    assert C.sizeof(bd._Window) == 16 and C.sizeof(dr.NormParams) == 32 and C.sizeof(bd._Rows) == 24 and C.sizeof(bd._NormVectors) == 96
    assert bd._NormCall.data0.offset == 24 and bd._NormCall.data5.offset == 24 + 5 * 24 and C.sizeof(bd._NormCall) == 168


def test_numbers_beyond_32_bits_do_not_wrap():
    """A window or a run of tokens longer than everything, however it is written."""
    assert dr.NormParams(mod_tokens=2 ** 32 + 1).mod_tokens == 2 ** 31 - 1
    seen = []

    class Ctx(_Ctx):
        def __init__(self):
            self._lib = type("L", (), {"dr_cache_attn_window_fwd": staticmethod(lambda *a: seen.append(a[5]._obj) or 0)})()

        def check(self, st):
            assert st == 0

    class Cuda(torch.Tensor):
        def get_device(self):
            return 0

    gpu = lambda t: t.as_subclass(Cuda)  # noqa: E731
    cache, batch = dr.PagedCache(2, 2, 32, 64, device="cpu"), dr.CacheBatch(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32), 3)
    cache.k, batch.cu = gpu(cache.k), gpu(batch.cu)
    q = gpu(torch.zeros(3, 4, 64))
    dr.dr_cache_attn_window_fwd(Ctx(), cache, batch, q, gpu(torch.zeros(3, 4, 64)), 2 ** 32 + 5, sinks=2 ** 40, frame_tokens=2 ** 33, stream=0)
    assert (seen[0].frame_tokens, seen[0].window, seen[0].sinks) == (2 ** 31 - 1,) * 3
    dr.dr_cache_attn_window_fwd(Ctx(), cache, batch, q, gpu(torch.zeros(3, 4, 64)), -2 ** 32 + 5, stream=0)
    assert seen[1].window == -1


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_oracle_norm_by_loops(kind):
    rng = np.random.RandomState(0)
    x, br = rng.randn(2, 3, 5), rng.randn(2, 3, 5)
    vec = dict(gate=rng.randn(2, 2, 5), scale=rng.randn(2, 2, 5), shift=rng.randn(2, 2, 5), weight=rng.randn(5), bias=rng.randn(5))
    t, y, _, _ = o.forward(x, br, vec, kind, 0.1, 0.5, 2, False)
    for b in range(2):
        for n in range(3):
            row = [0.5 * x[b, n, c] + vec["gate"][b, n // 2, c] * br[b, n, c] for c in range(5)]
            mean = sum(row) / 5 if kind == "layer" else 0.0
            var = sum((z - mean) ** 2 for z in row) / 5
            for c in range(5):
                want = ((row[c] - mean) / (var + 0.1) ** 0.5 * vec["weight"][c] + vec["bias"][c]) * (1 + vec["scale"][b, n // 2, c]) + vec["shift"][b, n // 2, c]
                assert abs(t[b, n, c] - row[c]) < 1e-12 and abs(y[b, n, c] - want) < 1e-12


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("branch_norm", [False, True])
def test_oracle_gradients_by_differences(kind, branch_norm):
    rng = np.random.RandomState(1)
    x, br, dy, dt = (rng.randn(2, 5, 7) for _ in range(4))
    vec = dict(gate=rng.randn(2, 3, 7), scale=rng.randn(2, 3, 7), shift=rng.randn(2, 3, 7), weight=rng.randn(7), bias=rng.randn(7))
    if branch_norm:
        vec["branch_weight"] = rng.randn(7)

    def loss(x, b, v):
        t, y, _, _ = o.forward(x, b, v, kind, 0.1, 0.5, 2, branch_norm)
        return (y * dy).sum() + (t * dt).sum()

    t = o.forward(x, br, vec, kind, 0.1, 0.5, 2, branch_norm)[0]
    got = o.backward(t, br, dy, dt, vec, kind, 0.1, 0.5, 2, branch_norm)
    for k, (grad, _) in got.items():
        if k == "branch_weight" and not branch_norm:
            continue
        way = rng.randn(*grad.shape)
        at = lambda s: loss(x + (s * way if k == "x" else 0), br + (s * way if k == "branch" else 0), {n: a + (s * way if n == k else 0) for n, a in vec.items()})  # noqa: E731
        slope = (at(1e-5) - at(-1e-5)) / 2e-5
        assert abs((grad * way).sum() - slope) < 1e-6 * (1 + np.abs(grad * way).sum()), k
