"""One layer of a streaming video model between its weights' products: norm and modulation, norms of the heads, rotary positions, append, attention over the last
frames and the first one, the gated residual; its cache read back for the sparse attention; samples that go on from it; its training step; on other streams and devices."""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import layer_oracle as lo
from oracle import streaming_oracle as so
from stream_helpers import HALF_BF16, assert_close, f64
from test_gpu_cache_views import positive, tolerance

pytestmark = pytest.mark.gpu
EPS = 1e-6


def arrays_of(cache):
    return (cache.k.view(torch.uint8).cpu().numpy(), cache.v.view(torch.uint8).cpu().numpy(), cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy())


class Layer:
    """Weights, modulations and the rolling cache of one stream: pages behind the window go back to the pool and come again."""

    def __init__(self, dtype, Hq=4, H=2, d=64, P=32, frame=50, window=3, sinks=1, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.Hq, self.H, self.d, self.frame, self.window, self.sinks, self.P = dtype, Hq, H, d, frame, window, sinks, P
        self.C = Hq * d
        rnd = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()  # noqa: E731
        self.wq, self.wk, self.wv, self.wo = (rnd(self.C, n) / self.C ** 0.5 for n in (self.C, H * d, H * d, self.C))
        self.head_weight = (1 + 0.1 * torch.randn(d, generator=g)).cuda()
        self.mods = (0.3 * torch.randn(1, 1, 3, self.C, generator=g)).cuda()
        self.ctx = dr.Context(0)
        self.cache = dr.PagedCache(12, H, P, d)
        self.free, self.pages = list(range(12)), {}
        self.rope = dr.RopeParams(d, axis_pairs=[d // 2 - 2 * (d // 6), d // 6, d // 6])
        self.pre = dr.NormParams(dr.NORM_LAYER, eps=EPS)
        self.heads = dr.NormParams(dr.NORM_RMS, eps=EPS)
        self.first = dr.NormVectors(shift=self.mods[:, :, 0], scale=self.mods[:, :, 1])
        self.second = dr.NormVectors(gate=self.mods[:, :, 2], shift=self.mods[:, :, 0], scale=self.mods[:, :, 1])
        self.hw = dr.NormVectors(weight=self.head_weight)

    def pages_for(self, held, new):
        """The page table for frames up to held + new: pages that no new token sees are given back first."""
        lo = max(0, (held // self.frame + 1 - self.window) * self.frame)
        for i in [i for i in self.pages if i * self.P >= self.sinks * self.frame and (i + 1) * self.P <= lo]:
            self.free.append(self.pages.pop(i))
        for i in range(held // self.P, -(-(held + new) // self.P)):
            self.pages.setdefault(i, self.free.pop(0) if i not in self.pages else None)
        width = max(self.pages) + 1
        return np.array([[self.pages.get(i, -1) for i in range(width)]], np.int32)

    def run(self, x, batch, positions, out):
        """x [1, T, C] -> (its normed form, attention's q and o and lse, the residual, the next block's input)."""
        T, Hq, H, d = x.shape[1], self.Hq, self.H, self.d
        y = torch.empty_like(x)
        dr.dr_norm_fwd(self.ctx, self.pre, x, y, vectors=self.first)
        q, k, v = (y[0] @ w for w in (self.wq, self.wk, self.wv))
        q, k = (t.view(T, -1, d) for t in (q, k))
        qn, kn = torch.empty_like(q), torch.empty_like(k)
        dr.dr_norm_fwd(self.ctx, self.heads, q, qn, vectors=self.hw)
        dr.dr_norm_fwd(self.ctx, self.heads, k, kn, vectors=self.hw)
        turned = torch.empty_like(qn)
        dr.dr_rope_fwd(self.ctx, self.rope, qn.transpose(0, 1)[None], positions, turned.transpose(0, 1)[None])
        dr.dr_cache_append(self.ctx, self.cache, batch, kn, v.view(T, H, d), rope=self.rope, positions=positions)
        o, lse = torch.empty_like(turned), torch.empty(Hq, T, device="cuda")
        dr.dr_cache_attn_window_fwd(self.ctx, self.cache, batch, turned, o, self.window, sinks=self.sinks, frame_tokens=self.frame, lse=lse)
        branch = (o.view(T, -1) @ self.wo)[None]
        total, after = torch.empty_like(x), torch.empty_like(x)
        dr.dr_norm_fwd(self.ctx, self.pre, x, after, branch=branch, total=total, vectors=self.second)
        out.update(y=y, q=q, qn=qn, turned=turned, o=o, lse=lse, branch=branch, total=total, after=after)
        return after


def positions_of(first, T, frame):
    p = torch.arange(first, first + T)
    return torch.stack([p // frame, p % frame // 10, p % 10]).to(torch.int32).cuda()


def batch_of(table, length, T):
    return dr.CacheBatch(torch.tensor([0, T], dtype=torch.int32, device="cuda"), torch.tensor([length], dtype=torch.int32, device="cuda"), torch.from_numpy(table).cuda(), T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_frame_after_frame_with_a_rolling_cache(dtype):
    """Every operator of every step against the oracle on what it was given."""
    layer, held, bf16 = Layer(dtype), 0, dtype == torch.bfloat16
    mods = {k: f64(layer.mods[:, :, i]) for i, k in enumerate(("shift", "scale", "gate"))}
    round_ = lambda x, e: e + (HALF_BF16 * (np.abs(x) + e) if bf16 else 0.0)  # noqa: E731
    for new in (50, 50, 150, 7, 43, 50, 1, 99):
        table = layer.pages_for(held, new)
        x = torch.randn(1, new, layer.C, generator=torch.Generator().manual_seed(held), dtype=torch.float32).to(dtype).cuda()
        r = {}
        layer.run(x, batch_of(table, held + new, new), positions_of(held, new, layer.frame), r)
        _, y, _, e = lo.forward(f64(x), None, {k: mods[k] for k in ("shift", "scale")}, "layer", EPS, 1.0, 0, False)
        assert_close(f64(r["y"]), y, round_(y, e), "norm")
        _, y, _, e = lo.forward(f64(r["q"]), None, {"weight": f64(layer.head_weight)}, "rms", EPS, 1.0, 0, False)
        assert_close(f64(r["qn"]), y, round_(y, e), "norm of the heads")
        arrays, cu, lens = arrays_of(layer.cache), np.array([0, new]), np.array([held + new])
        args = (cu, lens, table, layer.frame, layer.window, layer.sinks)
        want, wlse = so.attend_window(f64(r["turned"]), *arrays, *args)
        mean = so.attend_window(f64(r["turned"]), arrays[0], positive(arrays[1]), *arrays[2:], *args)[0]
        tol, ltol = tolerance(f64(r["turned"]), arrays, want, wlse, mean, table.size * layer.P, bf16)
        assert_close(f64(r["o"]), want, tol, "attention")
        assert_close(f64(r["lse"]), wlse, ltol, "lse")
        t, y, et, e = lo.forward(f64(x), f64(r["branch"]), mods, "layer", EPS, 1.0, 0, False)
        assert_close(f64(r["total"]), t, round_(t, et), "residual")
        assert_close(f64(r["after"]), y, round_(y, e), "next block's input")
        held += new
    assert held > layer.frame * (layer.window + layer.sinks + 1) and len(layer.free) >= 1


def test_a_step_on_another_stream_captured_and_replayed():
    layer, new = Layer(torch.bfloat16), 50
    table = layer.pages_for(0, new)
    batch, pos = batch_of(table, new, new), positions_of(0, new, layer.frame)
    x, r = torch.randn(1, new, layer.C, device="cuda").bfloat16(), {}
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.run(x, batch, pos, r)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            layer.run(x, batch, pos, r)
    torch.cuda.synchronize()
    held = dict(r)
    for i in range(3):
        x.copy_(torch.randn(x.shape, device="cuda"))
        eager = {}
        layer.run(x, batch, pos, eager)
        want = {k: v.clone() for k, v in eager.items()}
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(held[k], want[k]) for k in want)


def test_the_cache_read_back_feeds_the_sparse_attention():
    """[1, H, N, d] out of the pages, all blocks kept, against the attention over the cache itself."""
    H, d, P, N = 2, 128, 64, 8 * 64
    ctx, cache = dr.Context(0), dr.PagedCache(9, H, P, d)
    g = torch.Generator().manual_seed(1)
    k, v, q = (torch.randn(N, H, d, generator=g).bfloat16().cuda() for _ in range(3))
    batch = batch_of(np.array([[3, 1, 4, 0, 5, 8, 2, 6]], np.int32), N, N)
    dr.dr_cache_append(ctx, cache, batch, k, v)
    Q = q.transpose(0, 1)[None].contiguous()
    K, V, O = (torch.empty_like(Q) for _ in range(3))
    dr.dr_cache_read(ctx, cache, batch, K[0].transpose(0, 1), V[0].transpose(0, 1))
    shape = dr.shape_of(Q, 8, 8, 8, 64)
    Sb = N // 64
    rowptr = (torch.arange(Sb + 1, dtype=torch.int32, device="cuda") * Sb)[None, None].contiguous()
    colidx = torch.arange(Sb, dtype=torch.int32, device="cuda").repeat(Sb)[None, None].contiguous()
    dr.dr_sparse_attn_fwd(ctx, shape, Q, K, V, rowptr, colidx, 1, Sb * Sb, O)
    out = torch.empty_like(q)
    dr.dr_cache_attn_fwd(ctx, cache, batch, q, out, causal=False)
    # each has rounded its probabilities and its result once
    w = torch.softmax(Q.float() @ K.float().transpose(2, 3).contiguous() / d ** 0.5, -1)
    mean = (w @ V.float().abs())[0].transpose(0, 1)
    off = (O[0].transpose(0, 1).float() - out.float()).abs()
    assert bool((off <= 2.2 * HALF_BF16 * (mean + out.float().abs()) + 1e-5).all())
    assert torch.equal(K[0].transpose(0, 1).float(), k.to(torch.float8_e4m3fn).float()) or float((K[0].transpose(0, 1) - k).abs().max()) <= 2.0 ** -4 * float(k.abs().max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_samples_that_go_on_from_one_past(dtype):
    """A prefix of whole pages: the same as each sample's own table with those pages in front."""
    H, d, P, past, n = 2, 64, 32, 20 * 32, 5
    ctx, cache = dr.Context(0), dr.PagedCache(40, H, P, d)
    g = torch.Generator().manual_seed(2)
    whole = batch_of(np.arange(20, dtype=np.int32)[None], past, past)
    dr.dr_cache_append(ctx, cache, whole, *(torch.randn(past, H, d, generator=g).to(dtype).cuda() for _ in range(2)))
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    own_pages = [[20 + 3 * s, 21 + 3 * s, 22 + 3 * s] for s in range(n)]
    for step, new in ((0, 30), (1, 1), (2, 40)):
        held = (0, 30, 31)[step]
        T = n * new
        cu, lens = i32([new * s for s in range(n + 1)]), i32([held + new] * n)
        own = dr.CacheBatch(cu, lens, i32(own_pages), T)
        k, v, q = (torch.randn(T, h, d, generator=g).to(dtype).cuda() for h in (H, H, 4))
        dr.dr_cache_append(ctx, cache, own, k, v)
        prefix = dr.CacheBatch(i32([0, T]), i32([past]), i32([list(range(20))]), T)
        full = dr.CacheBatch(cu, lens + past, i32([list(range(20)) + p for p in own_pages]), T)
        a, b = torch.empty_like(q), torch.empty_like(q)
        la, lb = (torch.empty(4, T, device="cuda") for _ in range(2))
        dr.dr_cache_attn_shared_fwd(ctx, cache, prefix, own, q, a, lse=la)
        dr.dr_cache_attn_fwd(ctx, cache, full, q, b, lse=lb)
        size = float(cache.values().abs().max())
        assert float((a.float() - b.float()).abs().max()) <= (4 * HALF_BF16 if dtype == torch.bfloat16 else 2e-5) * size
        assert float((la - lb).abs().max()) <= 1e-4


def test_a_training_step_captured_while_eager_ones_go_on():
    """Forward and all gradients of two norms around a product, one leaf used by both; the same graph replayed between eager steps of the same tensors."""
    B, N, C = 2, 300, 256
    ctx, g = dr.Context(0), torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    x, dy, w, m = rnd(B, N, C), rnd(B, N, C), rnd(C, C) / 16, 0.3 * rnd(B, 3, 3, C)
    norm = dr.NormParams(eps=EPS, mod_tokens=100)
    first, second = dr.NormVectors(scale=m[:, :, 1], shift=m[:, :, 0]), dr.NormVectors(gate=m[:, :, 2], scale=m[:, :, 1], shift=m[:, :, 0])
    out = {}

    def step():
        y, total, after = (torch.empty_like(x) for _ in range(3))
        dr.dr_norm_fwd(ctx, norm, x, y, vectors=first)
        branch = y @ w
        dr.dr_norm_fwd(ctx, norm, x, after, branch=branch, total=total, vectors=second)
        dx, db, dx2 = (torch.empty_like(x) for _ in range(3))
        grads = [{k: torch.empty(B, 3, C, device="cuda") for k in names} for names in (("gate", "scale", "shift"), ("scale", "shift"))]
        dr.dr_norm_bwd(ctx, norm, total, dy, dx, branch=branch, dbranch=db, vectors=second, grads=dr.NormVectors(**grads[0]))
        dr.dr_norm_bwd(ctx, norm, x, db @ w.t().contiguous(), dx2, dtotal=dx, vectors=first, grads=dr.NormVectors(**grads[1]))
        out.update(after=after, dx=dx2, gate=grads[0]["gate"], scale=grads[0]["scale"] + grads[1]["scale"], shift=grads[0]["shift"] + grads[1]["shift"])

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    held = dict(out)
    for i in range(3):
        x.copy_(torch.randn(x.shape, device="cuda"))
        step()
        want = {k: v.clone() for k, v in out.items()}
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(held[k], want[k]) for k in want)
    # the whole step against autograd in fp64
    X, M = x.double().cpu().requires_grad_(), m.double().cpu().requires_grad_()
    mods = [M[:, :, i].repeat_interleave(100, 1) for i in range(3)]
    ln = lambda t: (t - t.mean(-1, keepdim=True)) / torch.sqrt(t.var(-1, unbiased=False, keepdim=True) + EPS)  # noqa: E731
    y = ln(X) * (1 + mods[1]) + mods[0]
    total = X + mods[2] * (y @ w.double().cpu())
    ((ln(total) * (1 + mods[1]) + mods[0]) * dy.double().cpu()).sum().backward()
    for got, wanted in ((out["dx"], X.grad), (out["shift"], M.grad[:, :, 0]), (out["scale"], M.grad[:, :, 1]), (out["gate"], M.grad[:, :, 2])):
        # fp32 throughout: products of 256 terms and sums of 100, some 400 roundings of 2^-24 of the largest
        assert float((got.double().cpu() - wanted).abs().max()) <= 400 * 2.0 ** -24 * float(wanted.abs().max()) * 4


def test_two_contexts_at_once_on_two_streams():
    """The same calls, each context its scratch, overlapping in time."""
    layers = [Layer(torch.bfloat16, seed=7) for _ in range(2)]
    new = 150
    table = [l.pages_for(0, new) for l in layers][0]
    batch, pos = batch_of(table, new, new), positions_of(0, new, 50)
    x = torch.randn(1, new, layers[0].C, device="cuda").bfloat16()
    streams, got = [torch.cuda.Stream() for _ in layers], [{}, {}]
    torch.cuda.synchronize()
    for _ in range(5):
        for l, s, r in zip(layers, streams, got):
            with torch.cuda.stream(s):
                l.run(x, batch, pos, r)
    torch.cuda.synchronize()
    assert all(torch.equal(got[0][k], got[1][k]) for k in got[0])
