"""Pages that are missing have no influence on attention, whatever the pool holds where a page number of 0 would lead: neither the codes of page 0
nor its scales, which no append may have set yet."""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from stream_helpers import assert_close, attend_tolerance, batch_arrays, f64, filled_cache, gpu_cache, on_gpu

pytestmark = pytest.mark.gpu

SCALES = {"nan": float("nan"), "inf": float("inf"), "-inf": float("-inf"), "largest": 2.0 ** 127, "zero": 0.0}


def _attend(arrays, cu, lens, table, q, causal):
    T, Hq = q.shape[:2]
    out, lse = torch.full_like(q, 7.0), torch.full((Hq, T), 7.0, device="cuda")
    dr.dr_cache_attn_fwd(dr.Context(0), gpu_cache(*arrays), dr.CacheBatch(*on_gpu(cu, lens, table), T), q, out, causal=causal, lse=lse)
    return out, lse


@pytest.mark.parametrize("scale", SCALES, ids=str)
@pytest.mark.parametrize("dtype,new", [(torch.float32, 3), (torch.bfloat16, 3), (torch.bfloat16, 40), (torch.bfloat16, 300)], ids=["f32", "bf16", "bf16-40", "bf16-300"])
@pytest.mark.parametrize("P", [32, 64, 128])
def test_scales_of_a_page_that_nobody_has(P, dtype, new, scale):
    """Page 0 belongs to no sequence; pages are missing at the start, in the middle and at the end of the table."""
    d, H, n = 64, 2, 700
    pages = -(-n // P) + 2
    cu, lens, table = batch_arrays([new], [n], P, pages - 1)
    table += 1                                            # page 0 stays out
    for hole in (0, (n // 2) // P, (n - 1) // P):
        table[0, hole] = -1
    k, v, ks, vs = filled_cache(pages, H, P, d, seed=P)
    q = torch.from_numpy(np.random.RandomState(new).randn(new, 2 * H, d).astype(np.float32)).to(dtype).cuda()
    for causal in (True, False):
        clean, clse = _attend((k, v, ks, vs), cu, lens, table, q, causal)
        want, wlse, tol, ltol = attend_tolerance(f64(q), k, v, ks, vs, cu, lens, table, causal, dtype == torch.bfloat16)
        assert_close(f64(clean), want, tol, "o")
        assert_close(f64(clse), wlse, ltol, "lse")
        kb, vb, ksb, vsb = k.copy(), v.copy(), ks.copy(), vs.copy()
        kb[0], vb[0], ksb[0], vsb[0] = 0x7f, 0x7f, SCALES[scale], SCALES[scale]
        out, lse = _attend((kb, vb, ksb, vsb), cu, lens, table, q, causal)
        assert torch.equal(out, clean) and torch.equal(lse, clse)
