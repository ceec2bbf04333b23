"""dr_cache_attn_fwd against the fp64 oracle: lengths from one token on, ragged batches, grouped heads, both maskings, rows that see
nothing, values that are no numbers in places that cannot be seen."""
import math

import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import streaming_oracle as o
from stream_helpers import assert_close, attend_tolerance, batch_arrays, f64, filled_cache, gpu_cache, on_gpu

pytestmark = pytest.mark.gpu


def _run(cache_arrays, cu, lens, table, q, causal, ctx=None, sentinel=7.0):
    """(o, lse) of a call, in tensors that held a sentinel."""
    cache = gpu_cache(*cache_arrays)
    T, Hq = q.shape[:2]
    out, lse = torch.full_like(q, sentinel), torch.full((Hq, T), sentinel, device="cuda")
    dr.dr_cache_attn_fwd(ctx or dr.Context(0), cache, dr.CacheBatch(*on_gpu(cu, lens, table), T), q, out, causal=causal, lse=lse)
    torch.cuda.synchronize()
    return out, lse


def _compare(cache_arrays, cu, lens, table, q, causal):
    out, lse = _run(cache_arrays, cu, lens, table, q, causal)
    want, wlse, tol, ltol = attend_tolerance(f64(q), *cache_arrays, cu, lens, table, causal, q.dtype == torch.bfloat16)
    nobody = np.isnan(want).all(-1)                   # rows of no sequence keep what they held
    assert (f64(out)[nobody] == 7.0).all() and (f64(lse)[nobody.T] == 7.0).all()
    assert_close(f64(out)[~nobody], want[~nobody], tol[~nobody], "o")
    assert_close(f64(lse)[~nobody.T], wlse[~nobody.T], ltol[~nobody.T], "lse")


SHAPES = [  # d, P, heads, cached heads, new, held
    (64, 32, 1, 1, [1], [0]),
    (128, 128, 4, 2, [1, 1, 1, 1], [0, 127, 128, 700]),
    (128, 64, 3, 1, [1, 0, 5], [900, 40, 64]),
    (64, 128, 5, 5, [2, 17], [31, 0]),
    (64, 64, 8, 1, [3, 1], [2000, 63]),
    (128, 32, 6, 3, [16, 7, 1], [33, 300, 2500]),
    (128, 128, 2, 1, [70], [200]),
    (64, 32, 2, 2, [130], [61]),
    (64, 64, 1, 1, [1] * 67, [i * 3 for i in range(67)]),
    (128, 64, 10, 2, [33, 65, 31], [0, 1, 63]),
    # many rows over many keys
    (128, 128, 1, 1, [256], [500]),
    (128, 64, 2, 1, [150, 131], [300, 900]),
    (128, 32, 2, 2, [300], [701]),
    (64, 128, 3, 1, [120], [640]),
    (64, 64, 1, 1, [257], [450]),
    (64, 32, 2, 1, [200], [333]),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "both"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"d{s[0]}-P{s[1]}-{s[2]}of{s[3]}-new{max(s[4])}x{len(s[4])}")
def test_against_the_oracle(shape, causal, dtype):
    d, P, Hq, H, new, held = shape
    lens = [a + b for a, b in zip(new, held)]
    pages = sum(-(-n // P) for n in lens) + 2
    cu, lens, table = batch_arrays(new, lens, P, pages, seed=Hq)
    arrays = filled_cache(pages, H, P, d, seed=P + d)
    q = torch.from_numpy(np.random.RandomState(d).randn(int(cu[-1]), Hq, d).astype(np.float32)).to(dtype).cuda()
    _compare(arrays, cu, lens, table, q, causal)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("P", [32, 128])
def test_rows_that_see_nothing_bad_pages_and_rows_of_no_sequence(P, dtype):
    """A sequence shorter than its new tokens, an empty one, page numbers outside the pool, a table that is too narrow, tokens in front of the
    first and behind the last sequence."""
    d, H, pages = 64, 2, 9
    arrays = filled_cache(pages, H, P, d, seed=6)
    cu = np.array([3, 43, 53, 60, 70, 90], np.int32)
    lens = np.array([12, 0, 4 * P + 9, 2 * P + 3, -5], np.int32)
    table = np.array([[1, 2, 3], [4, 5, 6], [7, 100, 8], [0, -1, -2147483648], [1, 1, 1]], np.int32)
    q = torch.randn(100, 4, d, device="cuda").to(dtype)
    for causal in (True, False):
        _compare(arrays, cu, lens, table, q, causal)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("d,P,new", [(64, 32, 20), (128, 64, 90), (128, 128, 300)])
def test_what_cannot_be_seen_has_no_influence(d, P, new, dtype):
    """NaN codes behind the end of a sequence and in tokens that are masked; the rows that do see one get NaN in its channel."""
    H, held = 2, 70
    n = new + held
    pages = -(-n // P) + 1
    cu, lens, table = batch_arrays([new], [n], P, pages)
    k, v, ks, vs = filled_cache(pages, H, P, d, seed=2)
    q = torch.randn(new, H, d, device="cuda").to(dtype)
    clean, clse = _run((k, v, ks, vs), cu, lens, table, q, True)
    last, spare = table[0, (n - 1) // P], n % P
    if spare:
        k[last, :, spare:] = 0x7f
        v[last, :, :, spare:] = 0xff
    at = held + new // 2                              # a cached token that only the later half may see
    page, slot = table[0, at // P], at % P
    v[page, 0, 3, slot] = 0x7f
    k[page, 1, slot, 5] = 0xff
    out, lse = _run((k, v, ks, vs), cu, lens, table, q, True)
    assert torch.equal(out[:new // 2], clean[:new // 2]) and torch.equal(lse[:, :new // 2], clse[:, :new // 2])
    assert torch.isnan(out[new // 2:, 0, 3]).all() and torch.isnan(out[new // 2:, 1]).all() and torch.isnan(lse[1, new // 2:]).all()
    assert torch.equal(lse[0], clse[0])
    rest = [c for c in range(d) if c != 3]
    assert torch.equal(out[:, 0][:, rest], clean[:, 0][:, rest])


def test_queries_that_are_no_numbers_stay_in_their_rows():
    d, P, H = 128, 64, 2
    cu, lens, table = batch_arrays([40], [300], P, 6)
    arrays = filled_cache(6, H, P, d, seed=9)
    q = torch.randn(40, 4, d, device="cuda").bfloat16()
    clean, _ = _run(arrays, cu, lens, table, q, True)
    bad = q.clone()
    bad[7, 1, 3], bad[9, 2, 0] = float("nan"), float("inf")
    out, _ = _run(arrays, cu, lens, table, bad, True)
    keep = torch.ones(40, 4, dtype=torch.bool, device="cuda")
    keep[7, 1] = keep[9, 2] = False
    assert torch.equal(out[keep], clean[keep]) and torch.isnan(out[7, 1]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_large_logits(dtype):
    """Logits of some thousands, increasing along the keys: every chunk moves the running maximum."""
    d, P, H = 64, 64, 1
    cu, lens, table = batch_arrays([3], [640], P, 10, spare=0)
    k, v, ks, vs = filled_cache(10, H, P, d, seed=3)
    k[:] = o.encode(np.random.RandomState(1).rand(*k.shape) + 0.5)
    ks[:] = 1.0
    for i, p in enumerate(table[0]):
        ks[p] = 2.0 ** (i // 2)
    q = torch.ones(3, 1, d, device="cuda") * torch.tensor([4.0, -4.0, 0.25], device="cuda")[:, None, None]
    _compare((k, v, ks, vs), cu, lens, table, q.to(dtype), False)


def test_long_caches_are_cut_into_pieces_with_the_same_result():
    """One row over 20 000 tokens, whole tables and tables far wider than the sequence (more and smaller pieces)."""
    d, P, H, n = 64, 32, 1, 20011
    pages = -(-n // P)
    cu, lens, table = batch_arrays([1], [n], P, pages, spare=0)
    arrays = filled_cache(pages, H, P, d, seed=11)
    q = torch.randn(1, 2, d, device="cuda")
    _compare(arrays, cu, lens, table, q, True)
    wide = np.concatenate([table, np.full((1, 40000), -1, np.int32)], 1)
    _compare(arrays, cu, lens, wide, q, True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_strided_queries_and_outputs(dtype):
    d, P, H = 128, 32, 2
    cu, lens, table = batch_arrays([19, 30], [60, 30], P, 4)
    arrays = filled_cache(4, H, P, d, seed=12)
    buf = torch.randn(49, 3, 4, d, device="cuda").to(dtype)
    want, _ = _run(arrays, cu, lens, table, buf[:, 0].contiguous(), True)
    out = torch.zeros(4, 49, d + 16, device="cuda", dtype=dtype)
    view = out.permute(1, 0, 2)[..., :d]
    dr.dr_cache_attn_fwd(dr.Context(0), gpu_cache(*arrays), dr.CacheBatch(*on_gpu(cu, lens, table), 49), buf[:, 0], view)
    assert torch.equal(view, want) and (out[..., d:] == 0).all()


def test_any_choice_of_pages_without_causality():
    """Attending to some of a sequence's blocks is attending over a table of those."""
    d, P, H = 64, 64, 2
    arrays = filled_cache(12, H, P, d, seed=13)
    keep = np.array([[9, 2, 5]], np.int32)
    cu, lens = np.array([0, 25], np.int32), np.array([2 * P + 11], np.int32)
    q = torch.randn(25, 2, d, device="cuda").bfloat16()
    _compare(arrays, cu, lens, keep, q, False)
    k, v, ks, vs = arrays
    # the same through the block-sparse call on what the codes stand for
    K = torch.from_numpy((o.decode(k[keep[0]]) * ks[keep[0]][:, :, None, None]).transpose(1, 0, 2, 3).reshape(1, H, -1, d)[:, :, :lens[0]].astype(np.float32)).cuda()
    V = torch.from_numpy((o.decode(v[keep[0]]) * vs[keep[0]][:, :, None, None]).transpose(1, 0, 3, 2).reshape(1, H, -1, d)[:, :, :lens[0]].astype(np.float32)).cuda()
    N = int(lens[0])
    Q = torch.zeros(1, H, N, d, device="cuda")
    Q[0, :, :25] = q.transpose(0, 1)
    ref, ref_lse = torch.empty_like(Q), torch.empty(1, H, N, device="cuda")
    Sb = -(-N // 64)
    rowptr = (torch.arange(Sb + 1, dtype=torch.int32, device="cuda") * Sb)[None, None].contiguous()
    colidx = torch.arange(Sb, dtype=torch.int32, device="cuda").repeat(Sb)[None, None].contiguous()
    ctx = dr.Context(0)
    dr.dr_sparse_attn_fwd(ctx, dr.shape_of(Q, 1, 1, N, 64), Q, K, V, rowptr, colidx, 1, Sb * Sb, ref, ref_lse)
    out, lse = _run(arrays, cu, lens, keep, q, False)
    # bf16 probabilities and result on one side: two roundings of values up to the largest |V|
    assert float((out.float() - ref[0, :, :25].transpose(0, 1)).abs().max()) <= 2 * 2.0 ** -8 * float(V.abs().max())
    assert float((lse - ref_lse[0, :, :25]).abs().max()) <= 1e-4


@pytest.mark.parametrize("d,P", [(128, 128), (128, 32), (64, 64)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "both"])
def test_many_rows_with_a_page_that_is_missing(d, P, causal):
    """The first page, one in the middle, the last one: the keys on it do not count."""
    n, new = 900, 250
    for hole in (0, (n // 2) // P, (n - 1) // P):
        cu, lens, table = batch_arrays([new], [n], P, -(-n // P))
        table[0, hole] = 10 ** 6
        arrays = filled_cache(table.shape[1], 1, P, d, seed=hole)
        q = torch.from_numpy(np.random.RandomState(P).randn(new, 1, d).astype(np.float32)).bfloat16().cuda()
        _compare(arrays, cu, lens, table, q, causal)


@pytest.mark.parametrize("d,P", [(128, 64), (64, 32)])
def test_many_rows_whose_logits_outgrow_those_of_the_first_keys(d, P):
    """Logits up to 2^11 behind a first chunk of ordinary ones, and the reverse: no power of two leaves its range."""
    n, new = 1000, 200
    cu, lens, table = batch_arrays([new], [n], P, -(-n // P), spare=0)
    for order in (1, -1):
        k, v, ks, vs = filled_cache(table.shape[1], 1, P, d, seed=5)
        k[:] = o.encode(np.random.RandomState(1).rand(*k.shape) + 0.5)
        for i, p in enumerate(table[0][::order]):
            ks[p] = 2.0 ** (9 * i // table.shape[1] - 2)
        q = torch.linspace(-4, 4, new, device="cuda").bfloat16()[:, None, None].expand(new, 1, d).contiguous()
        _compare((k, v, ks, vs), cu, lens, table, q, False)


def test_many_rows_that_see_a_token_without_a_number():
    d, P, n, new = 128, 64, 1000, 200
    cu, lens, table = batch_arrays([new], [n], P, -(-n // P))
    k, v, ks, vs = filled_cache(table.shape[1] + 1, 2, P, d, seed=5)
    q = torch.randn(new, 2, d, device="cuda").bfloat16()
    clean, clse = _run((k, v, ks, vs), cu, lens, table, q, True)
    page, slot = table[0, 300 // P], 300 % P
    v[page, 0, 77, slot] = 0xff
    k[page, 1, slot, 9] = 0x7f
    out, lse = _run((k, v, ks, vs), cu, lens, table, q, True)
    assert torch.isnan(out[:, 0, 77]).all() and torch.isnan(out[:, 1]).all() and torch.isnan(lse[1]).all()
    rest = [c for c in range(d) if c != 77]
    assert torch.equal(out[:, 0][:, rest], clean[:, 0][:, rest]) and torch.equal(lse[0], clse[0])
