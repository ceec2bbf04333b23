"""Scales that are no power of two count as the next lower one: what a PagedCache reads back is what attention reads, and what an append goes on from."""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import streaming_oracle as o
from stream_helpers import assert_close, attend_tolerance, batch_arrays, codes, f64, filled_cache, gpu_cache, on_gpu

ODD = [(3.0, 2.0), (1.0, 1.0), (1.9999999, 1.0), (0.7, 0.5), (2.0 ** -100 * 1.5, 2.0 ** -100), (3e38, 2.0 ** 127)]


@pytest.mark.parametrize("scale,power", ODD)
def test_keys_and_values_read_the_next_lower_power(scale, power):
    cache = dr.PagedCache(2, 1, 32, 64, device="cpu")
    cache.k.view(torch.uint8)[1, 0, 3, 5] = 0x38
    cache.v.view(torch.uint8)[1, 0, 5, 3] = 0xb8
    cache.k_scale[1], cache.v_scale[1] = scale, scale
    assert float(cache.keys()[1, 0, 3, 5]) == power and float(cache.values()[1, 0, 3, 5]) == -power


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,new", [(torch.float32, 4), (torch.bfloat16, 4), (torch.bfloat16, 250)], ids=["f32", "bf16", "bf16-250"])
def test_attention_reads_what_the_cache_reads_back(dtype, new):
    d, P, H, n = 64, 64, 2, 500
    cu, lens, table = batch_arrays([new], [n], P, 8)
    k, v, ks, vs = filled_cache(8, H, P, d, seed=1)
    rng = np.random.RandomState(2)
    odd = [(s * rng.uniform(1.0, 1.999, s.shape)).astype(np.float32) for s in (ks, vs)]
    q = torch.from_numpy(rng.randn(new, H, d).astype(np.float32)).to(dtype).cuda()
    cache, batch = gpu_cache(k, v, *odd), dr.CacheBatch(*on_gpu(cu, lens, table), new)
    out = torch.empty_like(q)
    dr.dr_cache_attn_fwd(dr.Context(0), cache, batch, q, out, causal=False)
    want, _, tol, _ = attend_tolerance(f64(q), k, v, ks, vs, cu, lens, table, False, dtype == torch.bfloat16)
    assert_close(f64(out), want, tol, "o")
    assert np.array_equal(f64(cache.keys()), o.decode(k) * ks[:, :, None, None])
    assert np.array_equal(f64(cache.values()), (o.decode(v) * vs[:, :, None, None]).transpose(0, 1, 3, 2))


@pytest.mark.gpu
def test_an_append_goes_on_from_the_next_lower_power():
    d, P, H = 64, 32, 2
    cu, lens, table = batch_arrays([3], [10], P, 2)
    k, v, ks, vs = filled_cache(2, H, P, d, seed=3)
    K, V = (torch.from_numpy(np.random.RandomState(i).randn(3, H, d).astype(np.float32)).cuda() for i in (1, 2))
    cache = gpu_cache(k, v, ks * np.float32(1.75), vs * np.float32(1.25))
    dr.dr_cache_append(dr.Context(0), cache, dr.CacheBatch(*on_gpu(cu, lens, table), 3), K, V)
    page = table[0, 0]
    wk, wks = o.append(k, ks, f64(K), cu, lens, table, False)
    wv, wvs = o.append(v, vs, f64(V), cu, lens, table, True)
    assert np.array_equal(codes(cache.k), wk) and np.array_equal(codes(cache.v), wv)
    assert np.array_equal(f64(cache.k_scale)[page], wks[page]) and np.array_equal(f64(cache.v_scale)[page], wvs[page])
