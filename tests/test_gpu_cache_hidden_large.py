"""Values beside the largest number, whose code times scale is 2^128: rows that may not see such a token are not touched by it (a probability of 0 times an
infinite value would be no number)."""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from stream_helpers import assert_close, attend_tolerance, batch_arrays, codes, f64, on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,new", [(torch.float32, 70), (torch.bfloat16, 70), (torch.bfloat16, 400)], ids=["f32", "bf16", "bf16-400"])
@pytest.mark.parametrize("d,P", [(64, 32), (128, 64), (64, 128)])
def test_hidden_values_near_the_largest_number(d, P, new, dtype):
    H, held = 2, 3 * P - 40
    n = held + new
    pages = -(-n // P)
    cu, lens, table = batch_arrays([new], [n], P, pages, spare=0)
    rng = np.random.RandomState(P)
    K, V, Q = (torch.from_numpy(rng.randn(T, H, d).astype(np.float32)).to(dtype).cuda() for T in (n, n, new))
    ctx, batch = dr.Context(0), dr.CacheBatch(*on_gpu(cu, lens, table), new)
    fill = dr.CacheBatch(*on_gpu(np.array([0, n], np.int32), lens, table), n)
    at = n - 3                                                        # a token of the last page; rows in front of its page see nothing of that
    first = at // P * P
    rows = first - held
    assert 0 < rows < new
    out, cache = [], None
    for large in (False, True):
        v = V.clone()
        if large:
            v[at, :, 7], v[at, :, 9] = torch.finfo(dtype).max, torch.finfo(dtype).min
        cache = dr.PagedCache(pages, H, P, d)
        dr.dr_cache_append(ctx, cache, fill, K, v)
        if not large:
            clean = codes(cache.k), codes(cache.v), cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy()
        o, lse = torch.empty_like(Q), torch.empty(H, new, device="cuda")
        dr.dr_cache_attn_fwd(ctx, cache, batch, Q, o, causal=True, lse=lse)
        out.append((o, lse))
    assert float(cache.v_scale.max()) == 2.0 ** 120 and torch.isinf(cache.values()).any()
    want, wlse, tol, ltol = attend_tolerance(f64(Q), *clean, cu, lens, table, True, dtype == torch.bfloat16)
    for o, lse in out:
        assert_close(f64(o)[:rows], want[:rows], tol[:rows], "o")
        assert_close(f64(lse), wlse, ltol, "lse")
    rest = [c for c in range(d) if c not in (7, 9)]
    assert torch.isfinite(out[1][0][rows:][..., rest]).all()
