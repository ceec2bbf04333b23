"""The streaming operators where their kernels change shape: heads that share angles, batches of many sequences, groups larger than a tile,
results larger than the caches."""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import streaming_oracle as o
from stream_helpers import ULP32, assert_close, attend_tolerance, batch_arrays, codes, f64, filled_cache, gpu_cache, on_gpu

pytestmark = pytest.mark.gpu


def _batch(cu, lens, table, tokens):
    return dr.CacheBatch(*on_gpu(cu, lens, table), tokens)


@pytest.mark.parametrize("layout,dtype,d,P,H,new,held", [
    ("half", torch.bfloat16, 128, 128, 40, [1500], [300]),
    ("interleaved", torch.bfloat16, 128, 128, 40, [900, 500], [0, 77]),
    ("half", torch.float32, 64, 32, 24, [2000, 40], [3, 90]),
    ("interleaved", torch.float32, 128, 64, 9, [16, 3, 11], [20, 63, 100]),
], ids=lambda x: str(x).replace("torch.", "") if not isinstance(x, list) else f"new{max(x)}")
def test_keys_take_the_nearest_code(layout, dtype, d, P, H, new, held):
    """Several heads to a workgroup (and few tokens, where nothing is kept): a key's code is that of the exact rotation rounded to fp32."""
    lens = [a + b for a, b in zip(new, held)]
    pages = sum(-(-n // P) for n in lens) + 2
    cu, lens, table = batch_arrays(new, lens, P, pages, seed=H)
    T = int(cu[-1])
    rng = np.random.RandomState(T)
    K, V = (torch.from_numpy(rng.randn(T, H, d).astype(np.float32)).to(dtype).cuda() for _ in range(2))
    params = dr.RopeParams(d, layout=dr.ROPE_HALF if layout == "half" else dr.ROPE_INTERLEAVED, mscale=1.0986)
    k, v, ks, vs = filled_cache(pages, H, P, d, seed=2)
    cache = gpu_cache(k, v, ks, vs)
    dr.dr_cache_append(dr.Context(0), cache, _batch(cu, lens, table, T), K, V, rope=params)
    where = np.concatenate([np.arange(b, a + b) for a, b in zip(new, held)])[None]
    x = f64(K).transpose(1, 0, 2)
    turned = o.rope(x, where, d, layout, [d // 2], mscale=1.0986).transpose(1, 0, 2)
    wk, wks = o.append(k, ks, turned.astype(np.float32), cu, lens, table, False)
    wv, wvs = o.append(v, vs, f64(V), cu, lens, table, True)
    assert np.array_equal(f64(cache.k_scale), wks) and np.array_equal(f64(cache.v_scale), wvs) and np.array_equal(codes(cache.v), wv)
    got = codes(cache.k)
    # Polynomials to 1e-15, products to 2^-53, and angles of up to 1800 that either side forms from a frequency of 53 bits (2e-13): the rounding to fp32
    # differs for 2e-13 / 2^-24 of the values, and one fp32 number in 2^20 borders on two codes: 3e-12 of the codes, of 8e6 at most here.
    assert np.array_equal(got, wk)


@pytest.mark.parametrize("d,P,H,T,held", [(128, 128, 40, 700, 60), (64, 32, 24, 2000, 45), (128, 64, 3, 200, 17), (64, 128, 2, 14, 100)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_infinities_in_some_heads(d, P, H, T, held, dtype):
    """They saturate and leave the scale to the finite values, in a page that is new and in one that held tokens; other heads do not notice."""
    pages = -(-(T + held) // P) + 1
    cu, lens, table = batch_arrays([T], [T + held], P, pages, seed=4)
    rng = np.random.RandomState(T)
    K, V = (torch.from_numpy((rng.randn(T, H, d) * 4.0 ** rng.randint(-2, 3, (T, H, 1))).astype(np.float32)).to(dtype).cuda() for _ in range(2))
    for n, x in enumerate((K, V)):
        x[3 + n, 1, 5], x[T - 1, 1, 6], x[T - 2, 0, 7] = float("inf"), float("-inf"), float("nan")
        if dtype == torch.float32:
            x[T // 2, 0] = 3.4e38
    k, v, ks, vs = filled_cache(pages, H, P, d, seed=6)
    cache = gpu_cache(k, v, ks, vs)
    dr.dr_cache_append(dr.Context(0), cache, _batch(cu, lens, table, T), K, V)
    for got, scale, was, ws, new, inner in ((cache.k, cache.k_scale, k, ks, K, False), (cache.v, cache.v_scale, v, vs, V, True)):
        want, wscale = o.append(was, ws, f64(new), cu, lens, table, inner)
        assert np.array_equal(f64(scale), wscale)
        assert np.array_equal(o.canonical(codes(got)), o.canonical(want))


def _attend(arrays, cu, lens, table, q, causal):
    cache = gpu_cache(*arrays)
    T, Hq = q.shape[:2]
    out, lse = torch.full_like(q, 7.0), torch.full((Hq, T), 7.0, device="cuda")
    dr.dr_cache_attn_fwd(dr.Context(0), cache, _batch(cu, lens, table, T), q, out, causal=causal, lse=lse)
    want, wlse, tol, ltol = attend_tolerance(f64(q), *arrays, cu, lens, table, causal, q.dtype == torch.bfloat16)
    nobody = np.isnan(want).all(-1)
    assert (f64(out)[nobody] == 7.0).all() and (f64(lse)[nobody.T] == 7.0).all()
    assert_close(f64(out)[~nobody], want[~nobody], tol[~nobody], "o")
    assert_close(f64(lse)[~nobody.T], wlse[~nobody.T], ltol[~nobody.T], "lse")


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "both"])
@pytest.mark.parametrize("d,P,group", [(64, 32, 1), (128, 64, 1), (64, 128, 3)])
def test_unequal_sequences_of_many_rows(d, P, group, causal):
    """An empty one, one token, one shorter than its new tokens (rows that see nothing), a page that is missing, rows of no sequence at either end."""
    new, lens = [400, 0, 1, 450, 220], [400 + 130, 9, 700, 110, 220]
    H = 2
    pages = sum(-(-n // P) for n in lens) + 2
    cu, lens, table = batch_arrays(new, lens, P, pages, seed=8)
    cu = cu + 3
    table[0, 1] = pages + 5
    arrays = filled_cache(pages, H, P, d, seed=d)
    q = torch.from_numpy(np.random.RandomState(1).randn(int(cu[-1]) + 4, H * group, d).astype(np.float32)).bfloat16().cuda()
    _attend(arrays, cu, lens, table, q, causal)


@pytest.mark.parametrize("S", [2, 64, 65])
def test_many_sequences_of_many_rows(S):
    rng = np.random.RandomState(S)
    new = list(rng.randint(150, 330, S))
    held = list(rng.randint(0, 200, S))
    new[0], new[S - 1] = 330, 250
    d, P, H = 64, 64, 1
    lens = [a + b for a, b in zip(new, held)]
    pages = sum(-(-n // P) for n in lens)
    cu, lens, table = batch_arrays(new, lens, P, pages, seed=S)
    arrays = filled_cache(pages, H, P, d, seed=S)
    q = torch.from_numpy(rng.randn(int(cu[-1]), H, d).astype(np.float32)).bfloat16().cuda()
    _attend(arrays, cu, lens, table, q, True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("heads", [256, 257, 700])
def test_a_group_as_large_as_a_tile_and_larger(heads, dtype):
    d, P = 64, 32
    cu, lens, table = batch_arrays([2, 1], [400, 130], P, 20, seed=heads)
    arrays = filled_cache(20, 1, P, d, seed=5)
    q = torch.from_numpy(np.random.RandomState(heads).randn(3, heads, d).astype(np.float32)).to(dtype).cuda()
    for causal in (True, False):
        _attend(arrays, cu, lens, table, q, causal)


@pytest.mark.parametrize("where", ["everywhere", "late"])
@pytest.mark.parametrize("growth", [4.0, 30.0, 60.0])
@pytest.mark.parametrize("d,P", [(64, 32), (128, 128)])
def test_values_near_the_largest_number(d, P, growth, where):
    """Logits that grow along the keys, by less and by more than a reference is left behind, over values of 2^118: their sums stay in range only if
    no probability is far above 1."""
    cu, lens, table = batch_arrays([300], [900], P, 32)
    k, v, ks, vs = filled_cache(32, 1, P, d, seed=12)
    v[(v & 0x7f) > 0x40] = 0x40                             # at most 2
    vs[:] = 2.0 ** 116
    if where == "late":
        vs[table[0, :700 // P]] = 1.0
    k[:, :, :, 0] = 0x38                                    # 1 in channel 0, times a scale that grows by steps
    order = table[0, :-(-900 // P)]
    q = torch.from_numpy(np.random.RandomState(3).randn(300, 1, d).astype(np.float32)).bfloat16().cuda()
    q[:, :, 1:] *= 0.01
    q[:, :, 0] = float(growth * np.sqrt(d) / 4)             # logits of channel 0: growth / 4 * scale
    ks[order] = (2.0 ** -np.arange(len(order))[::-1] * 4).clip(2.0 ** -6)[:, None]
    _attend((k, v, ks, vs), cu, lens, table, q, False)


@pytest.mark.parametrize("layout", [dr.ROPE_HALF, dr.ROPE_INTERLEAVED], ids=["half", "interleaved"])
def test_a_result_larger_than_the_caches(layout):
    """269 MB of bf16: the same bits as calls on parts of it, forward, backward and in place."""
    H, N, d = 40, 26300, 128
    ctx, rope = dr.Context(0), dr.RopeParams(96, layout=layout, axis_pairs=[16, 16, 16])
    X = torch.randn(1, H, N, d, device="cuda").bfloat16()
    pos = torch.randint(0, 400, (3, N), dtype=torch.int32, device="cuda")
    for call in (dr.dr_rope_fwd, dr.dr_rope_bwd):
        Y = torch.empty_like(X)
        call(ctx, rope, X, pos, Y)
        for a, b in ((0, 700), (N - 900, N)):
            part = torch.empty(1, H, b - a, d, dtype=X.dtype, device="cuda")
            call(ctx, rope, X[:, :, a:b], pos[:, a:b], part)
            assert torch.equal(Y[:, :, a:b], part)
        Z = X.clone()
        call(ctx, rope, Z, pos, Z)
        assert torch.equal(Z, Y)
