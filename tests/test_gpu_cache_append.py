"""dr_cache_append against the fp64 oracle: ragged batches, pages that fill in steps, scales that grow, values that are no numbers."""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import streaming_oracle as o
from stream_helpers import F8, ULP32, batch_arrays, codes, f64, filled_cache, gpu_cache, on_gpu

pytestmark = pytest.mark.gpu


def _batch(cu, lens, table, tokens):
    return dr.CacheBatch(*on_gpu(cu, lens, table), tokens)


def _check_exact(cache, k, ks, v, vs):
    for name, got, scale, want, wscale in (("k", cache.k, cache.k_scale, k, ks), ("v", cache.v, cache.v_scale, v, vs)):
        assert np.array_equal(f64(scale), wscale), name
        assert np.array_equal(o.canonical(codes(got)), o.canonical(want)), name


SHAPES = [  # d, P, heads, new, held
    (64, 32, 2, [1], [0]),
    (128, 128, 3, [1, 1, 1], [0, 127, 500]),
    (128, 64, 2, [70, 0, 1, 129, 3], [0, 9, 63, 64, 61]),
    (64, 128, 1, [300], [77]),
    (64, 32, 5, [33, 31, 32], [31, 1, 0]),
    (128, 32, 2, [95, 2], [18, 14]),
    (64, 64, 3, [2] * 70, [i % 90 for i in range(70)]),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"d{s[0]}-P{s[1]}-H{s[2]}-S{len(s[3])}")
def test_against_the_oracle_bit_for_bit(shape, dtype):
    d, P, H, new, held = shape
    lens = [a + b for a, b in zip(new, held)]
    pages = sum(-(-n // P) for n in lens) + 3
    cu, lens, table = batch_arrays(new, lens, P, pages, seed=d + P)
    T = int(cu[-1])
    k, v, ks, vs = filled_cache(pages, H, P, d, seed=P)
    rng = np.random.RandomState(T)
    K, V = (torch.from_numpy((rng.randn(T, H, d) * 4.0 ** rng.randint(-2, 3, (T, H, 1))).astype(np.float32)).to(dtype).cuda() for _ in range(2))
    cache = gpu_cache(k, v, ks, vs)
    dr.dr_cache_append(dr.Context(0), cache, _batch(cu, lens, table, T), K, V)
    wk, wks = o.append(k, ks, f64(K), cu, lens, table, False)
    wv, wvs = o.append(v, vs, f64(V), cu, lens, table, True)
    _check_exact(cache, wk, wks, wv, wvs)
    # again: the same slots, nothing else moves
    dr.dr_cache_append(dr.Context(0), cache, _batch(cu, lens, table, T), K, V)
    wk, wks = o.append(wk, wks, f64(K), cu, lens, table, False)
    wv, wvs = o.append(wv, wvs, f64(V), cu, lens, table, True)
    _check_exact(cache, wk, wks, wv, wvs)


ROPES = [("half", 1.0, 1), ("interleaved", 1.0, 3), ("half", 0.5, 3), ("interleaved", 0.75, 1), ("half", 38 / 64, 1)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("d,P", [(64, 32), (128, 128)])
@pytest.mark.parametrize("rope", ROPES, ids=lambda r: "-".join(map(str, r)))
def test_rotated_keys(rope, d, P, dtype):
    layout, part, axes = rope
    dim = int(d * part) // 2 * 2
    pairs = [dim // 2] if axes == 1 else [dim // 2 - 2 * (dim // 6), dim // 6, dim // 6]
    new, held, H = [150, 1, 40], [20, 63, 0], 2
    lens = [a + b for a, b in zip(new, held)]
    pages = sum(-(-n // P) for n in lens) + 1
    cu, lens, table = batch_arrays(new, lens, P, pages, seed=3)
    T = int(cu[-1])
    rng = np.random.RandomState(dim)
    K, V = (torch.from_numpy(rng.randn(T, H, d).astype(np.float32)).to(dtype).cuda() for _ in range(2))
    params = dr.RopeParams(dim, layout=dr.ROPE_HALF if layout == "half" else dr.ROPE_INTERLEAVED, axis_pairs=pairs, factor=2.0, mscale=1.25)
    pos = None
    if axes == 3:
        pos = rng.randint(0, 5000, (3, T)).astype(np.int32)
    where = np.concatenate([np.arange(b, a + b) for a, b in zip(new, held)])[None] if pos is None else pos
    k, v, ks, vs = filled_cache(pages, H, P, d, seed=1)
    cache = gpu_cache(k, v, ks, vs)
    dr.dr_cache_append(dr.Context(0), cache, _batch(cu, lens, table, T), K, V, rope=params, positions=None if pos is None else on_gpu(pos)[0])
    x = f64(K).transpose(1, 0, 2)
    turned = o.rope(x, where, dim, layout, pairs, mscale=1.25, factor=2.0).transpose(1, 0, 2)
    wk, wks = o.append(k, ks, turned.astype(np.float32), cu, lens, table, False)
    wv, wvs = o.append(v, vs, f64(V), cu, lens, table, True)
    assert np.array_equal(f64(cache.k_scale), wks) and np.array_equal(codes(cache.v), wv) and np.array_equal(f64(cache.v_scale), wvs)
    got = codes(cache.k)
    # a code differs only where the rotation's 8 roundings reach over a border between two codes: one code, and seldom
    off = got != wk
    assert off.mean() < 1e-4
    step = np.abs(o.decode(got) - o.decode(wk))[off]
    near = np.maximum(np.abs(o.decode(got)), np.abs(o.decode(wk)))[off]
    assert (step <= np.maximum(near / 8, 2.0 ** -9)).all()
    # and every stored key is within half a step of the exact one
    for s in range(3):
        for i in range(new[s]):
            p = int(lens[s]) - new[s] + i
            page, slot, t = table[s, p // P], p % P, cu[s] + i
            val, want = o.decode(got[page, :, slot]) * wks[page][:, None], turned[t]
            sums = np.abs(x[:, t]).max() * 2 * 1.25
            assert (np.abs(val - want) <= np.maximum(np.abs(want) * 2.0 ** -4, 2.0 ** -10 * wks[page][:, None]) * (1 + 1e-6) + 8 * ULP32 * sums).all()


def test_token_by_token_equals_the_oracle_and_scales_only_grow():
    """A page that fills one token at a time, each larger than the last: every append rescales what is there."""
    d, P, H = 64, 32, 2
    ctx, cache = dr.Context(0), dr.PagedCache(2, H, P, d)
    k, ks = codes(cache.k), f64(cache.k_scale)
    v, vs = codes(cache.v), f64(cache.v_scale)
    rng = np.random.RandomState(8)
    table = np.array([[1, 0]], np.int32)
    for i in range(40):
        K, V = (torch.from_numpy((rng.randn(1, H, d) * 1.35 ** (i if i < 20 else 40 - i)).astype(np.float32)).cuda() for _ in range(2))
        cu, lens = np.array([0, 1], np.int32), np.array([i + 1], np.int32)
        dr.dr_cache_append(ctx, cache, _batch(cu, lens, table, 1), K, V)
        k, ks = o.append(k, ks, f64(K), cu, lens, table, False)
        v, vs = o.append(v, vs, f64(V), cu, lens, table, True)
        _check_exact(cache, k, ks, v, vs)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_values_that_are_no_numbers(dtype):
    d, P, H, T = 64, 32, 2, 40
    K, V = torch.randn(T, H, d, device="cuda").to(dtype), torch.randn(T, H, d, device="cuda").to(dtype)
    for x in (K, V):
        x[3, 0, 5], x[3, 0, 6], x[4, 1, 7] = float("inf"), float("-inf"), float("nan")
        x[33:, 1] = float("nan")                      # a page and head without a number
        x[:, 0, 9] = 0.0
        x[35, 0] = 3e38 if dtype == torch.float32 else 1e38
        x[36, 0] = 1e-39                              # below the fp32 normals
    cu, lens, table = batch_arrays([T], [T], P, 3)
    cache = dr.PagedCache(3, H, P, d)
    k, v = codes(cache.k), codes(cache.v)
    dr.dr_cache_append(dr.Context(0), cache, _batch(cu, lens, table, T), K, V)
    wk, wks = o.append(k, np.ones((3, H)), f64(K), cu, lens, table, False)
    wv, wvs = o.append(v, np.ones((3, H)), f64(V), cu, lens, table, True)
    _check_exact(cache, wk, wks, wv, wvs)


def test_bad_pages_and_lengths_store_nothing_and_touch_nothing():
    """Page numbers outside the pool, tokens at negative places, places beyond the table, offsets beyond the tensors."""
    d, P, H, pages = 64, 32, 2, 6
    k, v, ks, vs = filled_cache(pages, H, P, d, seed=4)
    cu = np.array([0, 40, 50, 80, 1000], np.int32)     # the last sequence ends behind the 100 rows
    lens = np.array([40, 7, 64 + 15, 20], np.int32)    # the second: three of its ten tokens at negative places
    table = np.array([[0, 99], [1, 5], [-7, 2], [3, 3]], np.int32)
    K, V = torch.randn(100, H, d, device="cuda"), torch.randn(100, H, d, device="cuda")
    cache = gpu_cache(k, v, ks, vs)
    dr.dr_cache_append(dr.Context(0), cache, _batch(cu, lens, table, 100), K, V)
    wk, wks = o.append(k, ks, f64(K), cu, lens, table, False)
    wv, wvs = o.append(v, vs, f64(V), cu, lens, table, True)
    _check_exact(cache, wk, wks, wv, wvs)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_strides_and_alignment(dtype):
    d, P, H, T = 128, 64, 3, 90
    cu, lens, table = batch_arrays([50, 40], [77, 40], P, 5)
    k, v, ks, vs = filled_cache(5, H, P, d, seed=5)
    buf = torch.randn(T, 3, H, d, device="cuda").to(dtype)
    flat = torch.zeros(T * (H * d + 5) + 1, device="cuda", dtype=dtype)
    odd = flat[1:].view(T, H * d + 5)[:, :H * d].unflatten(1, (H, d))
    odd.copy_(buf[:, 1])
    params = dr.RopeParams(96, axis_pairs=[48])
    got = []
    for K in (buf[:, 1], odd):
        cache = gpu_cache(k, v, ks, vs)
        dr.dr_cache_append(dr.Context(0), cache, _batch(cu, lens, table, T), K, buf[:, 2], rope=params)
        got.append(cache)
    assert torch.equal(got[0].v.view(torch.uint8), got[1].v.view(torch.uint8)) and torch.equal(got[0].k_scale, got[1].k_scale)
    a, b = codes(got[0].k), codes(got[1].k)
    assert (a != b).mean() < 1e-4                     # sums contracted differently: borders between codes only
    wv, wvs = o.append(v, vs, f64(buf[:, 2]), cu, lens, table, True)
    assert np.array_equal(codes(got[0].v), wv) and np.array_equal(f64(got[0].v_scale), wvs)
    # heads that are one tensor (stride 0)
    cache = gpu_cache(k, v, ks, vs)
    one = buf[:, :1, 0].contiguous()
    dr.dr_cache_append(dr.Context(0), cache, _batch(cu, lens, table, T), one.expand(T, H, d), one.expand(T, H, d))
    wk, _ = o.append(k, ks, np.repeat(f64(one), H, 1), cu, lens, table, False)
    assert np.array_equal(codes(cache.k), wk)


def test_pages_behind_four_gibibytes():
    """Codes of the last pages lie past 2^32 bytes of the pool."""
    d, P, H = 128, 128, 64
    pages = (1 << 32) // (H * P * d) + 3
    cache = dr.PagedCache(pages, H, P, d)
    K, V = torch.randn(130, H, d, device="cuda").bfloat16(), torch.randn(130, H, d, device="cuda").bfloat16()
    cu, lens = np.array([0, 130], np.int32), np.array([130], np.int32)
    small = dr.PagedCache(2, H, P, d)
    dr.dr_cache_append(dr.Context(0), cache, _batch(cu, lens, np.array([[pages - 1, pages - 2]], np.int32), 130), K, V)
    dr.dr_cache_append(dr.Context(0), small, _batch(cu, lens, np.array([[1, 0]], np.int32), 130), K, V)
    for a, b in ((cache.k, small.k), (cache.v, small.v)):
        assert torch.equal(a[-2:].view(torch.uint8), b.view(torch.uint8))
        assert int(a[:2].view(torch.uint8).max()) == 0
    assert torch.equal(cache.k_scale[-2:], small.k_scale) and torch.equal(cache.v_scale[-2:], small.v_scale)
    Q = torch.randn(130, H, d, device="cuda").bfloat16()
    out = [torch.empty_like(Q) for _ in range(2)]
    for c, t, y in ((cache, [[pages - 1, pages - 2]], out[0]), (small, [[1, 0]], out[1])):
        dr.dr_cache_attn_fwd(dr.Context(0), c, _batch(cu, lens, np.array(t, np.int32), 130), Q, y)
    assert torch.equal(*out)
