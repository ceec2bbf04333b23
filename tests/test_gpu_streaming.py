"""The streaming operators as a model uses them: queries rotated, keys and values appended, attention, chunk after chunk; captured, on other
streams, with contexts that share nothing or graphs that share one."""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import streaming_oracle as o
from stream_helpers import assert_close, attend_tolerance, batch_arrays, codes, f64, filled_cache, gpu_cache, on_gpu

pytestmark = pytest.mark.gpu


class Stream:
    """A layer's state: its cache, its batch arrays (whose values change from step to step), and its contexts."""

    def __init__(self, S, Hq, H, d, P, pages, width, dtype, ctx=None):
        self.ctx = ctx or dr.Context(0)
        self.cache = dr.PagedCache(pages, H, P, d)
        self.rope = dr.RopeParams(d, layout=dr.ROPE_INTERLEAVED, axis_pairs=[d // 2 - 2 * (d // 6), d // 6, d // 6])
        self.cu, self.lens = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (S + 1, S))
        ids = torch.randperm(pages, generator=torch.Generator().manual_seed(S)).to(torch.int32)
        self.table = ids[:S * width].view(S, width).contiguous().cuda()
        self.shape = (Hq, H, d, dtype)

    def step(self, q, k, v, positions, causal, out, lse):
        T = q.shape[0]
        batch = dr.CacheBatch(self.cu, self.lens, self.table, T)
        turned = torch.empty_like(q)
        dr.dr_rope_fwd(self.ctx, self.rope, q.transpose(0, 1)[None], positions, turned.transpose(0, 1)[None])
        dr.dr_cache_append(self.ctx, self.cache, batch, k, v, rope=self.rope, positions=positions)
        dr.dr_cache_attn_fwd(self.ctx, self.cache, batch, turned, out, causal=causal, lse=lse)
        return turned

    def grow(self, new):
        self.cu.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)))
        self.lens += torch.tensor(new, dtype=torch.int32, device="cuda")


def _chunk(rng, T, Hq, H, d, dtype):
    q, k, v = (torch.from_numpy(rng.randn(T, h, d).astype(np.float32)).to(dtype).cuda() for h in (Hq, H, H))
    return q, k, v, torch.from_numpy(rng.randint(0, 400, (3, T)).astype(np.int32)).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "both"])
def test_chunk_after_chunk(causal, dtype):
    S, Hq, H, d, P = 2, 4, 2, 64, 32
    st, rng = Stream(S, Hq, H, d, P, 20, 9, dtype), np.random.RandomState(5)
    exact = [[], []]                                     # the rotated keys and the values of each sequence, not quantised
    for new in ([30, 45], [1, 1], [64, 0], [1, 1], [17, 80]):
        T = sum(new)
        q, k, v, pos = _chunk(rng, T, Hq, H, d, dtype)
        st.grow(new)
        out, lse = torch.empty_like(q), torch.empty(Hq, T, device="cuda")
        turned = st.step(q, k, v, pos, causal, out, lse)
        cu, lens, table = (t.cpu().numpy() for t in (st.cu, st.lens, st.table))
        arrays = (codes(st.cache.k), codes(st.cache.v), st.cache.k_scale.cpu().numpy(), st.cache.v_scale.cpu().numpy())
        want, wlse, tol, ltol = attend_tolerance(f64(turned), *arrays, cu, lens, table, causal, dtype == torch.bfloat16)
        assert_close(f64(out), want, tol, "o")
        assert_close(f64(lse), wlse, ltol, "lse")
        # and against attention without the 8 bits
        p = pos.cpu().numpy()
        pairs = [st.rope.axis_pairs[i] for i in range(3)]
        rk = o.rope(f64(k).transpose(1, 0, 2), p, d, "interleaved", pairs).transpose(1, 0, 2)
        rq = o.rope(f64(q).transpose(1, 0, 2), p, d, "interleaved", pairs).transpose(1, 0, 2)
        at = 0
        for s, n in enumerate(new):
            exact[s].append((rk[at:at + n], f64(v)[at:at + n]))
            K, V = (np.concatenate([c[i] for c in exact[s]]) for i in (0, 1))
            for i in range(n):
                upto = len(K) - n + i + 1 if causal else len(K)
                for h in range(Hq):
                    x = K[:upto, h // 2] @ rq[at + i, h] / 8
                    w = np.exp(x - x.max())
                    w /= w.sum()
                    plain = w @ V[:upto, h // 2]
                    # a code is off by 2^-4 of its value at most, at random: a logit by some 2^-4 |q||k| / 8 / sqrt(64) * 2, a value by 2^-4
                    err = 2.0 ** -4 * np.linalg.norm(rq[at + i, h]) * np.abs(K[:upto, h // 2]).max() / 8
                    assert np.abs(f64(out)[at + i, h] - plain).max() <= (2 * err + 2.0 ** -4 + 2.0 ** -6) * np.abs(V[:upto, h // 2]).max()
            at += n


def _capture(call):
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            call()
    torch.cuda.synchronize()
    return graph


def test_a_captured_step_follows_lengths_tables_and_inputs():
    S, Hq, H, d, P, dtype = 3, 6, 2, 128, 64, torch.bfloat16
    st, eager = (Stream(S, Hq, H, d, P, 60, 18, dtype) for _ in range(2))
    rng, new = np.random.RandomState(6), [1, 1, 1]
    q, k, v, pos = _chunk(rng, 3, Hq, H, d, dtype)
    out, lse = torch.empty_like(q), torch.empty(Hq, 3, device="cuda")
    eo, el = torch.empty_like(q), torch.empty(Hq, 3, device="cuda")
    for s in (st, eager):
        s.grow([700, 3, 65])                             # a history of whatever lies in the pages
        for t in (s.cache.k, s.cache.v):
            t.view(torch.uint8).copy_(torch.randint(0, 0x48, t.shape, generator=torch.Generator().manual_seed(1), dtype=torch.uint8))
        s.grow(new)
    graph = _capture(lambda: st.step(q, k, v, pos, True, out, lse))
    for c in ("k", "v", "k_scale", "v_scale"):           # the capture's own eager step wrote here
        getattr(st.cache, c).view(torch.uint8).copy_(getattr(eager.cache, c).view(torch.uint8))
    for rep in range(4):
        for t, x in zip((q, k, v, pos), _chunk(rng, 3, Hq, H, d, dtype)):
            t.copy_(x)
        out.fill_(9), lse.fill_(9)
        torch.cuda.synchronize()
        graph.replay()
        eager.step(q, k, v, pos, True, eo, el)
        torch.cuda.synchronize()
        assert torch.equal(out, eo) and torch.equal(lse, el), rep
        for c in ("k", "v"):
            assert torch.equal(getattr(st.cache, c).view(torch.uint8), getattr(eager.cache, c).view(torch.uint8))
        for s in (st, eager):
            s.lens += torch.tensor([1, 30, 1], dtype=torch.int32, device="cuda")
            s.table.copy_(s.table.roll(1, 0) if rep == 1 else s.table)


def test_graphs_that_share_a_context_and_scratch_that_grows_behind_them():
    ctx, P, H, d = dr.Context(0), 32, 2, 64
    rng, jobs = np.random.RandomState(7), []
    for lens, new in (([3000], [1]), ([9000, 500], [1, 1]), ([40000] * 3, [2, 1, 1])):        # each needs more scratch than the last
        pages = sum(-(-n // P) for n in lens)
        cu, lens, table = batch_arrays(new, lens, P, pages, spare=0)
        cache = gpu_cache(*filled_cache(pages, H, P, d, seed=len(new)))
        batch = dr.CacheBatch(*on_gpu(cu, lens, table), int(cu[-1]))
        q = torch.from_numpy(rng.randn(int(cu[-1]), 4, d).astype(np.float32)).cuda()
        out = torch.empty_like(q)
        call = lambda c=cache, b=batch, q=q, out=out, x=ctx: dr.dr_cache_attn_fwd(x, c, b, q, out)
        jobs.append((_capture(call), call, q, out, cache, batch))
    for rep in range(3):
        for graph, call, q, out, cache, batch in jobs + jobs[::-1]:
            q.copy_(torch.randn_like(q))
            out.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            dr.dr_cache_attn_fwd(dr.Context(0), cache, batch, q, out)
            torch.cuda.synchronize()
            assert torch.equal(got, out)


def test_a_capture_without_scratch_is_refused_and_goes_on():
    P, H, d, n = 32, 1, 64, 20000
    pages = n // P
    cu, lens, table = batch_arrays([1], [n], P, pages, spare=0)
    cache, batch = gpu_cache(*filled_cache(pages, H, P, d, seed=1)), dr.CacheBatch(*on_gpu(cu, lens, table), 1)
    q = torch.randn(1, 2, d, device="cuda")
    out, other, ctx = torch.zeros_like(q), torch.zeros(8, device="cuda"), dr.Context(0)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            other += 1
            with pytest.raises(dr.DRError) as e:
                dr.dr_cache_attn_fwd(ctx, cache, batch, q, out)
    assert e.value.status_name == "DR_ERR_NOMEM"
    graph.replay()
    torch.cuda.synchronize()
    assert (other == 1).all() and (out == 0).all()
    dr.dr_cache_attn_fwd(ctx, cache, batch, q, out)
    assert torch.isfinite(out).all() and (out != 0).any()


def test_streams_of_two_contexts_at_once():
    """Two layers on two streams, each behind the work that makes its inputs: the results are those of one after the other."""
    dtype, args = torch.bfloat16, (2, 4, 2, 128, 64, 90, 40)
    rng = np.random.RandomState(9)
    chunks = [[_chunk(rng, 400, 4, 2, 128, dtype) for _ in range(3)] for _ in range(2)]

    def run(apart):
        outs, streams = [], [torch.cuda.Stream() for _ in range(2)]
        states = [Stream(*args, dtype) for _ in range(2)]
        torch.cuda.synchronize()
        for i in range(3):
            for layer in range(2):
                with torch.cuda.stream(streams[layer] if apart else torch.cuda.current_stream()):
                    q, k, v, pos = (t.clone() for t in chunks[layer][i])
                    states[layer].grow([250, 150])
                    out, lse = torch.empty_like(q), torch.empty(4, 400, device="cuda")
                    states[layer].step(q, k, v, pos, True, out, lse)
                    outs += [out, lse]
        torch.cuda.synchronize()
        return outs

    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b)


def test_stream_argument_and_repeated_calls_give_the_same_bits():
    st, rng = Stream(1, 4, 2, 128, 128, 30, 28, torch.bfloat16), np.random.RandomState(10)
    q, k, v, pos = _chunk(rng, 500, 4, 2, 128, torch.bfloat16)
    st.grow([500])
    out, lse = torch.empty_like(q), torch.empty(4, 500, device="cuda")
    turned = st.step(q, k, v, pos, True, out, lse)
    batch, side = dr.CacheBatch(st.cu, st.lens, st.table, 500), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        again = torch.empty_like(out)
        side.wait_stream(torch.cuda.current_stream())
        dr.dr_cache_attn_fwd(st.ctx, st.cache, batch, turned, again, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(again, out)
