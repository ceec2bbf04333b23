"""Reading the cache back, attention over a window of it and over a shared prefix, against the fp64 oracle and against the attention over all of it."""
import math

import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import streaming_oracle as o
from stream_helpers import HALF_BF16, ULP32, assert_close, batch_arrays, f64, filled_cache, gpu_cache, on_gpu

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])


def tolerance(q, arrays, want, lse, mean, keys, bf16):
    """Of o and of lse.  As in stream_helpers: with A the largest sum |q||k| / sqrt(d) of a row, a logit is off by (d + 4) roundings of A, a weight by twice that, sums of n
    weights by n / 8 + 32 roundings, and joining pieces by a few more; bf16: one rounding of every weight (`mean`: the weighted mean of |v|) and one of the result."""
    k, v, ks, vs = arrays
    d = q.shape[2]
    kmax = np.nanmax(np.sqrt(np.nansum((o.decode(k) * ks.astype(np.float64)[:, :, None, None]) ** 2, -1)))
    A = np.sqrt((q ** 2).sum(-1)) * kmax / math.sqrt(d)
    rel = 2 * (d + 4) * ULP32 * A + (keys / 8 + 48) * 2 * ULP32 + 4 * ULP32 * A
    top = np.nanmax(np.abs(o.decode(v)) * vs.astype(np.float64)[:, :, None, None])
    tol = rel[..., None] * top + (HALF_BF16 * (mean + np.abs(want)) if bf16 else 2 * ULP32 * np.abs(want))
    return tol, (rel + 4 * ULP32 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0)).T)).T


def positive(v):
    return np.where(o.decode(v) < 0, v & 0x7f, v)


def window(arrays, cu, lens, table, q, frame, win, sinks, ctx=None):
    T, Hq = q.shape[:2]
    out, lse = torch.full_like(q, 7.0), torch.full((Hq, T), 7.0, device="cuda")
    dr.dr_cache_attn_window_fwd(ctx or dr.Context(0), gpu_cache(*arrays), dr.CacheBatch(*on_gpu(cu, lens, table), T), q, out, win, sinks=sinks, frame_tokens=frame, lse=lse)
    torch.cuda.synchronize()
    return out, lse


def compare_window(arrays, cu, lens, table, q, frame, win, sinks):
    out, lse = window(arrays, cu, lens, table, q, frame, win, sinks)
    k, v, ks, vs = arrays
    args = (cu, lens, table, frame, win, sinks)
    want, wlse = o.attend_window(f64(q), *arrays, *args)
    mean = o.attend_window(f64(q), k, positive(v), ks, vs, *args)[0]
    tol, ltol = tolerance(f64(q), arrays, want, wlse, mean, table.shape[1] * k.shape[2], q.dtype == torch.bfloat16)
    nobody = np.isnan(want).all(-1)
    assert (f64(out)[nobody] == 7.0).all() and (f64(lse)[nobody.T] == 7.0).all()
    assert_close(f64(out)[~nobody], want[~nobody], tol[~nobody], "o")
    assert_close(f64(lse)[~nobody.T], wlse[~nobody.T], ltol[~nobody.T], "lse")


def forget(table, lens, new, P, frame, win, sinks):
    """The page table without the pages that no new token sees."""
    table = table.copy()
    for s, (n, length) in enumerate(zip(new, lens)):
        lo = max(0, ((length - n) // frame + 1 - win) * frame)
        for i in range(table.shape[1]):
            if i * P >= sinks * frame and (i + 1) * P <= lo:
                table[s, i] = (-1, 1 << 30)[i & 1]
    return table


WINDOWS = [  # d, P, heads, cached heads, new, held, frame, window, sinks
    (64, 32, 1, 1, [1], [0], 1, 1, 0),
    (128, 128, 4, 2, [1, 1, 1, 1], [0, 127, 128, 700], 1, 64, 4),
    (128, 64, 3, 1, [1, 0, 5], [900, 40, 64], 1, 100, 1),
    (64, 128, 5, 5, [2, 17], [31, 0], 7, 2, 1),
    (64, 64, 8, 1, [3, 1], [2000, 63], 1, 513, 70),
    (128, 32, 6, 3, [16, 7, 1], [33, 300, 2500], 33, 5, 2),
    (128, 128, 2, 1, [70], [200], 1, 30, 0),
    (64, 64, 1, 1, [1] * 67, [i * 9 for i in range(67)], 1, 50, 3),
    (128, 64, 10, 2, [33, 65, 31], [0, 1, 63], 16, 3, 0),
    # many rows over many keys: both ends inside tiles, whole frames, sinks of many chunks, sinks that meet the window
    (128, 128, 1, 1, [256], [500], 1, 200, 4),
    (128, 64, 2, 1, [150, 131], [300, 1900], 1, 640, 130),
    (128, 32, 2, 2, [300], [701], 100, 4, 2),
    (64, 128, 3, 1, [120], [1640], 360, 2, 1),
    (64, 64, 1, 1, [257], [1450], 200, 3, 2),
    (64, 32, 2, 1, [200, 300, 0, 1], [333, 1100, 5, 900], 1, 1000, 1),
    (128, 128, 2, 2, [700], [900], 350, 2, 2),
    # few tiles of many rows, cut into pieces; sequences without new tokens between them; more sequences than lanes
    (64, 32, 8, 2, [40, 0, 100, 1, 0, 64], [2000, 700, 1900, 30, 0, 2500], 1, 1500, 5),
    (128, 128, 5, 1, [52, 52, 52], [2900, 3000, 3100], 1, 2500, 0),
    (64, 64, 4, 1, [50] * 70, [1000 + 7 * i for i in range(70)], 1, 1200, 3),
]


@TYPES
@pytest.mark.parametrize("gone", [False, True], ids=["kept", "gone"])
@pytest.mark.parametrize("shape", WINDOWS, ids=lambda s: f"d{s[0]}-P{s[1]}-{s[2]}of{s[3]}-new{max(s[4])}x{len(s[4])}-{s[6]}.{s[7]}.{s[8]}")
def test_window_against_the_oracle(shape, gone, dtype):
    d, P, Hq, H, new, held, frame, win, sinks = shape
    lens = [a + b for a, b in zip(new, held)]
    pages = sum(-(-n // P) for n in lens) + 2
    cu, lens, table = batch_arrays(new, lens, P, pages, seed=Hq)
    if gone:
        table = forget(table, lens, new, P, frame, win, sinks)
    arrays = filled_cache(pages, H, P, d, seed=P + d)
    q = torch.from_numpy(np.random.RandomState(d).randn(int(cu[-1]), Hq, d).astype(np.float32)).to(dtype).cuda()
    compare_window(arrays, cu, lens, table, q, frame, win, sinks)


@TYPES
@pytest.mark.parametrize("P", [32, 128])
def test_window_rows_that_see_nothing_bad_pages_and_rows_of_no_sequence(P, dtype):
    d, H, pages = 64, 2, 9
    arrays = filled_cache(pages, H, P, d, seed=6)
    cu = np.array([3, 43, 53, 60, 70, 90], np.int32)
    lens = np.array([12, 0, 4 * P + 9, 2 * P + 3, -5], np.int32)
    table = np.array([[1, 2, 3], [4, 5, 6], [7, 100, 8], [0, -1, -2147483648], [1, 1, 1]], np.int32)
    q = torch.randn(100, 4, d, device="cuda").to(dtype)
    for frame, win, sinks in ((1, 5, 0), (1, 2147483647, 2147483647), (7, 2, 1), (2147483647, 1, 0), (1, 1, P + 3)):
        compare_window(arrays, cu, lens, table, q, frame, win, sinks)


@TYPES
@pytest.mark.parametrize("d,P,new,held", [(64, 32, 20, 170), (128, 64, 90, 400), (128, 128, 300, 900), (64, 128, 300, 700)])
def test_what_is_outside_the_window_has_no_influence(d, P, new, held, dtype):
    """NaN codes, infinite scales and values at the window's edges; rows that do see one get NaN in its channel."""
    H, win, sinks = 2, 60, 3
    n = new + held
    cu, lens, table = batch_arrays([new], [n], P, -(-n // P) + 1)
    k, v, ks, vs = filled_cache(-(-n // P) + 1, H, P, d, seed=2)
    q = torch.randn(new, H, d, device="cuda").to(dtype)
    clean, clse = window((k, v, ks, vs), cu, lens, table, q, 1, win, sinks)
    for at in (sinks, held - win, n - 1):                       # seen by nobody, by nobody, by the last row only
        page, slot = table[0, at // P], at % P
        k[page, 0, slot, 1] = v[page, 0, 2, slot] = 0x7f
    whole = [i for i in range(len(table[0])) if i * P >= sinks and (i + 1) * P <= held + 1 - win]
    for i in whole:
        k[table[0, i]], v[table[0, i]] = 0xff, 0x7f
        ks[table[0, i]] = vs[table[0, i]] = np.inf
    spare = n % P
    if spare:
        k[table[0, n // P], :, spare:] = v[table[0, n // P], :, :, spare:] = 0x7f
    out, lse = window((k, v, ks, vs), cu, lens, table, q, 1, win, sinks)
    assert torch.equal(out[:-1], clean[:-1]) and torch.equal(lse[:, :-1], clse[:, :-1])
    assert torch.equal(out[-1, 1], clean[-1, 1]) and torch.isnan(out[-1, 0]).all() and torch.isnan(lse[0, -1])
    at = held + new // 2                                        # a new token that only the rows behind it see
    page, slot = table[0, at // P], at % P
    v[page, 1, 3, slot] = 0xff
    out, lse = window((k, v, ks, vs), cu, lens, table, q, 1, win, sinks)
    rest = [c for c in range(d) if c != 3]
    sees = torch.zeros(new, dtype=torch.bool, device="cuda")
    sees[new // 2:min(new, new // 2 + win)] = True
    assert torch.isnan(out[sees, 1, 3]).all() and torch.equal(out[~sees][:, 1, 3], clean[~sees][:, 1, 3])
    assert torch.equal(out[:, 1][:, rest], clean[:, 1][:, rest]) and torch.equal(lse[1], clse[1])


@TYPES
@pytest.mark.parametrize("new,held", [([1, 1, 1], [5, 900, 64]), ([300, 17], [650, 0])])
def test_window_that_reaches_everything_is_the_causal_attention(new, held, dtype):
    d, P, H = 128, 64, 2
    lens = [a + b for a, b in zip(new, held)]
    cu, lens, table = batch_arrays(new, lens, P, 40)
    arrays = filled_cache(40, H, P, d, seed=4)
    q = torch.randn(int(cu[-1]), 4, d, device="cuda").to(dtype)
    out, lse = window(arrays, cu, lens, table, q, 1, 1 << 20, 0)
    want, wlse = torch.empty_like(q), torch.empty(4, q.shape[0], device="cuda")
    dr.dr_cache_attn_fwd(dr.Context(0), gpu_cache(*arrays), dr.CacheBatch(*on_gpu(cu, lens, table), q.shape[0]), q, want, lse=wlse)
    # (pieces may be cut elsewhere: two results, each off by its own rounding and by that of its weights)
    size = float(want.float().abs().max())
    assert float((out.float() - want.float()).abs().max()) <= (3 * HALF_BF16 if dtype == torch.bfloat16 else 1e-5) * max(size, 1.0)
    assert float((lse - wlse).abs().max()) <= 1e-4


def test_window_of_many_tiles_the_last_of_them_in_pieces():
    """288 tiles at once, and the same heads in calls of their own, which are cut elsewhere."""
    d, P, H, new, win = 64, 128, 36, 2048, 2500
    cu, lens, table = batch_arrays([new], [new + 3000], P, 41)
    k, v, ks, vs = filled_cache(41, H, P, d, seed=4)
    q = torch.randn(new, H, d, device="cuda").to(torch.bfloat16)
    out, lse = window((k, v, ks, vs), cu, lens, table, q, 1, win, 2)
    for h in range(0, H, 9):
        some = [np.ascontiguousarray(x[:, h:h + 9]) for x in (k, v, ks, vs)]
        want, wlse = window(some, cu, lens, table, q[:, h:h + 9].contiguous(), 1, win, 2)
        # (two results, each off by its own rounding and by that of its weights)
        size = float(want.float().abs().max())
        assert float((out[:, h:h + 9].float() - want.float()).abs().max()) <= 3 * HALF_BF16 * max(size, 1.0)
        assert float((lse[h:h + 9] - wlse).abs().max()) <= 1e-4


# ---- the shared prefix ------------------------------------------------------------------------------------

def shared(arrays, prefix, own, q, causal, ctx=None):
    T, Hq = q.shape[:2]
    out, lse = torch.full_like(q, 7.0), torch.full((Hq, T), 7.0, device="cuda")
    dr.dr_cache_attn_shared_fwd(ctx or dr.Context(0), gpu_cache(*arrays), dr.CacheBatch(*on_gpu(*prefix), T), dr.CacheBatch(*on_gpu(*own), T), q, out, causal=causal, lse=lse)
    torch.cuda.synchronize()
    return out, lse


def compare_shared(arrays, prefix, own, q, causal):
    out, lse = shared(arrays, prefix, own, q, causal)
    k, v, ks, vs = arrays
    want, wlse = o.attend_shared(f64(q), *arrays, prefix, own, causal)
    mean = o.attend_shared(f64(q), k, positive(v), ks, vs, prefix, own, causal)[0]
    tol, ltol = tolerance(f64(q), arrays, want, wlse, mean, (prefix[2].shape[1] + own[2].shape[1]) * k.shape[2], q.dtype == torch.bfloat16)
    nobody = np.isnan(want).all(-1)
    assert (f64(out)[nobody] == 7.0).all() and (f64(lse)[nobody.T] == 7.0).all()
    assert_close(f64(out)[~nobody], want[~nobody], tol[~nobody], "o")
    assert_close(f64(lse)[~nobody.T], wlse[~nobody.T], ltol[~nobody.T], "lse")


SHARED = [  # d, P, heads, cached heads, prefixes, sequences of each group, new, held
    (64, 32, 1, 1, [1], [1], [1], [0]),
    (128, 128, 4, 2, [700], [4], [1, 1, 1, 1], [0, 5, 128, 300]),
    (128, 64, 3, 1, [33, 64], [2, 1], [1, 0, 5], [90, 40, 0]),
    (64, 128, 5, 5, [1000, 0, 129], [1, 1, 1], [2, 17, 3], [31, 0, 200]),
    (64, 64, 8, 1, [2000], [40], [1] * 40, list(range(40))),
    (128, 32, 6, 3, [300, 1], [2, 1], [16, 7, 1], [33, 300, 500]),
    (128, 128, 2, 1, [1500], [3], [70, 90, 120], [200, 0, 64]),
    (64, 32, 2, 1, [900, 400], [1, 1], [200, 150], [61, 700]),
    (128, 64, 5, 1, [700], [60], [1] * 60, [3 * i for i in range(60)]),
    (64, 32, 8, 2, [1300, 2100], [4, 2], [40, 0, 100, 1, 0, 64], [0, 70, 1200, 30, 0, 500]),
    (64, 64, 4, 1, [1100], [70], [50] * 70, [5 * i for i in range(70)]),
]


def shared_batches(shape):
    d, P, Hq, H, prefixes, each, new, held = shape
    lens = [a + b for a, b in zip(new, held)]
    pages = sum(-(-n // P) for n in lens + prefixes) + 3
    cu, both, table = batch_arrays(new + [0] * len(prefixes), lens + prefixes, P, pages, seed=Hq)
    S = len(new)
    own = cu[:S + 1], both[:S], np.ascontiguousarray(table[:S])
    ends = np.cumsum([0] + each)
    return (cu[ends].astype(np.int32), both[S:], np.ascontiguousarray(table[S:])), own, filled_cache(pages, H, P, d, seed=P + d)


@TYPES
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "both"])
@pytest.mark.parametrize("shape", SHARED, ids=lambda s: f"d{s[0]}-P{s[1]}-{s[2]}of{s[3]}-{max(s[4])}x{len(s[4])}-new{max(s[6])}x{len(s[6])}")
def test_shared_against_the_oracle(shape, causal, dtype):
    prefix, own, arrays = shared_batches(shape)
    q = torch.from_numpy(np.random.RandomState(shape[0]).randn(int(own[0][-1]), shape[2], shape[0]).astype(np.float32)).to(dtype).cuda()
    compare_shared(arrays, prefix, own, q, causal)


@TYPES
def test_shared_with_tokens_outside_groups_and_sequences_and_bad_pages(dtype):
    """Groups that do not end where sequences do, tokens of no group, tokens of no sequence, prefixes and sequences of which nothing is stored."""
    P, d, H, pages = 32, 64, 2, 12
    arrays = filled_cache(pages, H, P, d, seed=8)
    own = np.array([3, 10, 10, 30, 41], np.int32), np.array([9, 0, 50, -4], np.int32), np.array([[1, 2], [3, 3], [4, 99], [5, 6]], np.int32)
    prefix = np.array([5, 20, 30, 36], np.int32), np.array([70, 33, 20], np.int32), np.array([[7, -1, 8], [9, 10, 0], [-3, 0, 0]], np.int32)
    q = torch.randn(50, 4, d, device="cuda").to(dtype)
    for causal in (True, False):
        compare_shared(arrays, prefix, own, q, causal)
    empty = np.array([0], np.int32), np.zeros(0, np.int32), np.zeros((0, 1), np.int32)
    compare_shared(arrays, empty, own, q, True)


@TYPES
def test_what_another_group_has_has_no_influence(dtype):
    prefix, own, (k, v, ks, vs) = shared_batches((128, 64, 4, 2, [700, 300], [3, 2], [1, 1, 1, 1, 1], [10, 20, 30, 40, 50]))
    q = torch.randn(5, 4, 128, device="cuda").to(dtype)
    clean, clse = shared((k, v, ks, vs), prefix, own, q, True)
    for page in prefix[2][0][:11]:
        k[page], v[page] = 0x7f, 0xff
    last = prefix[2][1][300 // 64]
    k[last, :, 300 % 64:] = v[last, :, :, 300 % 64:] = 0x7f
    out, lse = shared((k, v, ks, vs), prefix, own, q, True)
    assert torch.equal(out[3:], clean[3:]) and torch.equal(lse[:, 3:], clse[:, 3:])
    assert torch.isnan(out[:3]).all() and torch.isnan(lse[:, :3]).all()


# ---- reading back -----------------------------------------------------------------------------------------

@TYPES
@pytest.mark.parametrize("planes", [False, True])
@pytest.mark.parametrize("d,P,H,new,held", [(64, 32, 1, [1], [0]), (128, 128, 5, [1, 300, 0, 17], [127, 40, 9, 128]), (64, 64, 9, [64, 65, 63], [0, 64, 1]),
                                              (128, 32, 4, [200], [33]), (64, 128, 3, [1] * 70, list(range(70)))])
def test_read_is_exact(d, P, H, new, held, planes, dtype):
    lens = [a + b for a, b in zip(new, held)]
    pages = sum(-(-n // P) for n in lens) + 2
    cu, lens, table = batch_arrays(new, lens, P, pages, seed=1)
    rng = np.random.RandomState(3)
    k, v = rng.randint(0, 256, (pages, H, P, d)).astype(np.uint8), rng.randint(0, 256, (pages, H, d, P)).astype(np.uint8)       # NaN codes among them
    ks, vs = (2.0 ** rng.randint(-100, 118, (pages, H))).astype(np.float32), (2.0 ** rng.randint(-3, 3, (pages, H))).astype(np.float32)
    T = int(cu[-1]) + 2
    K, V = (torch.full((H, T, d), 7.0, device="cuda", dtype=dtype).transpose(0, 1) if planes else torch.full((T, H, d), 7.0, device="cuda", dtype=dtype) for _ in range(2))
    cache, batch = gpu_cache(k, v, ks, vs), dr.CacheBatch(*on_gpu(cu, lens, table), T)
    dr.dr_cache_read(dr.Context(0), cache, batch, K, V)
    for got, want in zip((K, V), o.read(k, v, ks, vs, cu, lens, table, T)):
        assert np.array_equal(f64(got), np.where(want == -1e300, 7.0, want), equal_nan=True)
    only = torch.zeros_like(V)
    dr.dr_cache_read(dr.Context(0), cache, batch, V=only)
    assert torch.equal(torch.nan_to_num(only[:-2].float(), nan=3.0), torch.nan_to_num(V[:-2].float(), nan=3.0))


@TYPES
def test_read_of_what_is_not_stored_and_largest_scales(dtype):
    P, d, H, pages = 32, 64, 2, 9
    k, v, ks, vs = filled_cache(pages, H, P, d, seed=6)
    ks[7], vs[8] = 2.0 ** 120, 2.0 ** 120
    k[7, 0, 3, :4] = (0x7e, 0x78, 0x77, 0xfe)                   # 448, 256: infinities there; 240: the largest below
    ks[1] = 1.5 * 2.0 ** -4                                     # no power of two: the next lower one
    cu = np.array([3, 43, 53, 60, 70, 90], np.int32)
    lens = np.array([12, 0, 4 * P + 9, 2 * P + 3, -5], np.int32)
    table = np.array([[1, 2, 3], [4, 5, 6], [7, 100, 8], [0, -1, -2147483648], [1, 1, 1]], np.int32)
    lens[2] = 7
    K, V = (torch.full((100, H, d), 7.0, device="cuda", dtype=dtype) for _ in range(2))
    dr.dr_cache_read(dr.Context(0), gpu_cache(k, v, ks, vs), dr.CacheBatch(*on_gpu(cu, lens, table), 100), K, V)
    down = np.exp2(np.floor(np.log2(ks.astype(np.float64)))), vs
    for got, want in zip((K, V), o.read(k, v, down[0], down[1], cu, lens, table, 100)):
        want = np.where(want == -1e300, 7.0, np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want))
        assert np.array_equal(f64(got), want, equal_nan=True)


@pytest.mark.parametrize("off", [1, 2])
def test_read_into_rows_that_are_not_aligned(off):
    P, d, H = 64, 64, 2
    k, v, ks, vs = filled_cache(4, H, P, d, seed=6)
    cu, lens, table = batch_arrays([90], [150], P, 4)
    K, V = torch.zeros(90, H, d + off, device="cuda")[:, :, off:], torch.zeros(90, H, d + off, device="cuda", dtype=torch.float32)[:, :, :d]
    dr.dr_cache_read(dr.Context(0), gpu_cache(k, v, ks, vs), dr.CacheBatch(*on_gpu(cu, lens, table), 90), K, V)
    wk, wv = o.read(k, v, ks, vs, cu, lens, table, 90)
    assert np.array_equal(f64(K), wk) and np.array_equal(f64(V), wv)


# ---- together ---------------------------------------------------------------------------------------------

def test_refusals_of_the_library():
    ctx = dr.Context(0)
    arrays = filled_cache(4, 2, 32, 64, seed=1)
    cache = gpu_cache(*arrays)
    batch = dr.CacheBatch(*on_gpu(np.array([0, 3], np.int32), np.array([9], np.int32), np.array([[1]], np.int32)), 3)
    other = dr.CacheBatch(*on_gpu(np.array([0, 3], np.int32), np.array([9], np.int32), np.array([[1]], np.int32)), 4)
    q, out = torch.zeros(3, 4, 64, device="cuda"), torch.zeros(3, 4, 64, device="cuda")
    kv = torch.zeros(3, 2, 64, device="cuda")
    for bad in (lambda: dr.dr_cache_attn_window_fwd(ctx, cache, batch, q, out, 0), lambda: dr.dr_cache_attn_window_fwd(ctx, cache, batch, q, out, 3, sinks=-1),
                lambda: dr.dr_cache_attn_window_fwd(ctx, cache, batch, q, out, 3, frame_tokens=0), lambda: dr.dr_cache_attn_window_fwd(ctx, cache, batch, q, q, 3),
                lambda: dr.dr_cache_attn_window_fwd(ctx, cache, batch, q[:, :3], out[:, :3], 3), lambda: dr.dr_cache_attn_shared_fwd(ctx, cache, other, batch, q, out),
                lambda: dr.dr_cache_attn_shared_fwd(ctx, cache, batch, batch, q, q), lambda: dr.dr_cache_read(ctx, cache, batch, kv, kv), lambda: dr.dr_cache_read(ctx, cache, batch, q, out),
                lambda: dr.dr_cache_read(ctx, cache, batch, kv[:1].expand(3, 2, 64), kv)):
        with pytest.raises(dr.DRError):
            bad()


def test_captured_and_replayed_with_other_lengths():
    """One graph of all three; the batch's arrays change between replays, and eager calls of another size lie between them."""
    d, P, H, T = 128, 64, 2, 6
    rng = np.random.RandomState(0)
    prefix, own, arrays = shared_batches((d, P, 4, H, [700, 300], [4, 2], [1] * T, [300, 20, 700, 40, 50, 0]))
    ctx, cache = dr.Context(0), gpu_cache(*arrays)
    pb, ob = dr.CacheBatch(*on_gpu(*prefix), T), dr.CacheBatch(*on_gpu(*own), T)
    q = torch.randn(T, 4, d, device="cuda").bfloat16()
    a, b, c, e = torch.empty_like(q), torch.empty_like(q), torch.empty(T, H, d, device="cuda"), torch.empty(T, H, d, device="cuda")

    def step():
        dr.dr_cache_attn_shared_fwd(ctx, cache, pb, ob, q, a)
        dr.dr_cache_attn_window_fwd(ctx, cache, ob, q, b, 100, sinks=2)
        dr.dr_cache_read(ctx, cache, ob, c, e)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        ob.lens.copy_(torch.from_numpy(np.minimum(own[1], rng.randint(1, 700, T)).astype(np.int32)))
        pb.lens.copy_(torch.from_numpy(np.array([rng.randint(1, 700), rng.randint(1, 300)], np.int32)))
        q.copy_(torch.randn(q.shape, device="cuda"))
        step()
        want = [t.clone() for t in (a, b, c, e)]
        for t in (a, b, c, e):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(want, (a, b, c, e)))


def test_without_a_call_before_a_capture_scratch_is_refused():
    prefix, own, arrays = shared_batches((128, 64, 4, 2, [700], [2], [1, 1], [300, 20]))
    ctx, cache = dr.Context(0), gpu_cache(*arrays)
    pb, ob = dr.CacheBatch(*on_gpu(*prefix), 2), dr.CacheBatch(*on_gpu(*own), 2)
    q = torch.randn(2, 4, 128, device="cuda").bfloat16()
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q.add_(0.0)
        with pytest.raises(dr.DRError):
            dr.dr_cache_attn_shared_fwd(ctx, cache, pb, ob, q, out)
