"""The sums of dr_cache_attn_fwd: what divides a row is the sum of the same rounded probabilities that multiply its values, so a row with one dominant key
returns that key's value; and the sum behind the log-sum-exp keeps small probabilities beside a large one."""
import math

import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import streaming_oracle as o
from stream_helpers import HALF_BF16, ULP32, assert_close, attend_tolerance, batch_arrays, f64, filled_cache, gpu_cache, on_gpu

pytestmark = pytest.mark.gpu


def _attend(arrays, cu, lens, table, q, causal=False):
    T, Hq = q.shape[:2]
    out, lse = torch.full_like(q, 7.0), torch.full((Hq, T), 7.0, device="cuda")
    dr.dr_cache_attn_fwd(dr.Context(0), gpu_cache(*arrays), dr.CacheBatch(*on_gpu(cu, lens, table), T), q, out, causal=causal, lse=lse)
    return f64(out), f64(lse)


def _flat(arrays, table, n):
    """Keys and values [n, d] of the only head of one sequence."""
    k, v, ks, vs = arrays
    at = np.arange(n)
    P = k.shape[2]
    page, slot = table[0, at // P], at % P
    return o.decode(k[page, 0, slot]) * ks[page, 0, None], o.decode(v[page, 0, :, slot]) * vs[page, 0, None]


@pytest.mark.parametrize("where", ["first", "early", "middle", "last"])
@pytest.mark.parametrize("new", [3, 40, 300])
@pytest.mark.parametrize("d,P", [(64, 32), (128, 64), (128, 128)])
def test_rows_with_one_dominant_key(d, P, new, where):
    """Every row has a key whose weight is 1 but for 2^-18, under a probability of any mantissa (the reference is the first keys' maximum)."""
    n = 1500
    cu, lens, table = batch_arrays([new], [n], P, -(-n // P), spare=0)
    arrays = filled_cache(table.shape[1], 1, P, d, seed=P + new)
    k, v, ks, vs = arrays
    at = {"first": 5, "early": 100, "middle": 700, "last": n - 2}[where]
    k[:, :, :, 0] = 0
    ks[:] = 2.0 ** -5
    k[table[0, at // P], 0, at % P] = 0
    k[table[0, at // P], 0, at % P, 0] = o.encode(64.0)[()]            # 2 in channel 0, 0 in the others
    rng = np.random.RandomState(new)
    x = rng.randn(new, 1, d) * 0.02
    x[:, 0, 0] = rng.uniform(11.0, 15.0, new) * math.sqrt(d)            # its logit: 22 to 30
    q = torch.from_numpy(x.astype(np.float32)).bfloat16().cuda()
    out, lse = _attend(arrays, cu, lens, table, q)
    K, V = _flat(arrays, table, n)
    s = f64(q)[:, 0] @ K.T / math.sqrt(d)
    w = np.exp(s - s.max(1, keepdims=True))
    total = w.sum(1, keepdims=True)
    w /= total
    assert (w[:, at] > 1 - 2.0 ** -18).all()
    want = w @ V
    # A rounding of a probability moves the row towards that value or away from it, so it counts by the distance to it: 2^-8 of the mean distance; the
    # same holds for errors of logits, (d + 4) roundings of 30.  Then 8 roundings of fp32 and the one to bf16.
    away = np.stack([w[i] @ np.abs(V - want[i]) for i in range(new)])
    tol = (HALF_BF16 + 2 * (d + 4) * ULP32 * 30) * 1.01 * away + (HALF_BF16 + 8 * ULP32) * np.abs(want)
    assert_close(out[:, 0], want, tol, "o")
    ref = s.max(1) + np.log(total[:, 0])
    assert_close(lse[0], ref, 2 * (d + 4) * ULP32 * 30 + 8 * ULP32 * np.abs(ref), "lse")


@pytest.mark.parametrize("dtype,new,heads,plain", [(torch.bfloat16, 256, 256, False), (torch.bfloat16, 256, 256, True), (torch.bfloat16, 5, 2, False), (torch.float32, 20, 3, False)],
                         ids=["bf16-256", "bf16-256-large-values", "bf16-5", "f32-20"])
@pytest.mark.parametrize("where", [3, 40, 30000])
def test_small_probabilities_beside_a_large_one(where, dtype, new, heads, plain):
    """60 000 keys with a probability of some 2^-25 each beside one of 1: together they are 0.0017 of the sum, one by one less than half of its last bit."""
    d, P, n = 64, 128, 60000
    cu, lens, table = batch_arrays([new], [n], P, -(-n // P), spare=0)
    pages = table.shape[1]
    k, v = np.zeros((pages, 1, P, d), np.uint8), np.zeros((pages, 1, d, P), np.uint8)
    ks, vs = np.ones((pages, 1), np.float32), np.ones((pages, 1), np.float32)
    k[table[0, where // P], 0, where % P, 0] = o.encode(8.0)[()]
    if plain:
        vs[table[0, 7]] = 2.0 ** 60
    q = torch.zeros(new, heads, d, device="cuda")                        # (256 tiles of 256 rows: nothing is cut into pieces)
    q[:, :, 0] = torch.linspace(17.25, 17.5, new, device="cuda")[:, None]
    q = q.to(dtype)
    _, lse = _attend((k, v, ks, vs), cu, lens, table, q)
    large = f64(q)[:, :, 0].T                                             # its logit; those of the others are 0, both exactly
    want = large + np.log1p((n - 1) * np.exp(-large))
    # The exponent of 2: four roundings of 25.3.  The sum: a lane adds the partial sum of every 256 keys (of every 32 where large values keep the running
    # maximum's loop), each addition off by 2^-24 of a sum of 1, and 128 more in all for the partial sums and the joins.
    tol = 4 * ULP32 * 25.3 + (n / (32 if plain else 256) + 128) * ULP32 + 4 * ULP32 * want
    assert (0.0015 < (n - 1) * np.exp(-large)).all() and (tol < 1.4e-4).all()
    assert_close(lse, want, tol, "lse")


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "both"])
@pytest.mark.parametrize("d,P,new,group", [(128, 128, 1, 5), (128, 32, 1, 1), (64, 64, 3, 5), (128, 64, 5, 3), (64, 32, 16, 1)])
def test_few_rows_keep_sixteen_bits_of_their_probabilities(d, P, new, group, causal):
    """bf16, up to 16 rows of a cached head: next to the result's own rounding nothing is left of the probabilities'.  Few keys whose weights are alike, so that
    values cancel; logits of order one, so that their own roundings count little."""
    H, lens = 2, [new + 2, 20, 90]
    cu, lens, table = batch_arrays([new] * 3, lens, P, sum(-(-n // P) for n in lens))
    arrays = filled_cache(int(table.max()) + 1, H, P, d, seed=P)
    arrays[2][:] = 2.0 ** -6
    q = torch.from_numpy(np.random.RandomState(new).randn(3 * new, H * group, d).astype(np.float32)).bfloat16().cuda()
    out, _ = _attend(arrays, cu, lens, table, q, causal)
    want, _, tol, _ = attend_tolerance(f64(q), *arrays, cu, lens, table, causal, False)
    k, v, ks, vs = arrays
    absmean, _ = o.attend(f64(q), k, v & 0x7f, ks, vs, cu, lens, table, causal)
    # two parts of a probability: what the second is rounded by, 2^-8 of 2^-8
    assert_close(out, want, tol + HALF_BF16 ** 2 * absmean + HALF_BF16 * np.abs(want), "o")
