"""dr_cache_append with positions that the caller gives, on one, two and three axes, where only a part of a head is rotated: codes and scales equal
the oracle's, for many tokens a sequence and for few."""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import streaming_oracle as o
from stream_helpers import batch_arrays, codes, f64, filled_cache, gpu_cache, on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("axes", [1, 2, 3])
@pytest.mark.parametrize("d,P,dim", [(128, 128, 64), (128, 32, 96), (64, 64, 16), (64, 128, 64), (64, 32, 38)])
def test_given_positions(d, P, dim, axes, layout, dtype):
    # Codes are compared exactly: either side forms angles up to 5000 from a frequency of 53 bits (6e-13), which moves the rounding to fp32 of 6e-13 / 2^-24
    # of the keys, and one fp32 number in 2^20 borders on two codes: 1e-11 of the codes, of 8e4 at most here.
    H = 3
    pairs = {1: [dim // 2], 2: [dim // 2 - dim // 6, dim // 6], 3: [dim // 2 - 2 * (dim // 6), dim // 6, dim // 6]}[axes]
    for new, held in (([150, 1, 40], [20, 63, 0]), ([3, 1, 16], [20, 63, 0])):
        lens = [a + b for a, b in zip(new, held)]
        pages = sum(-(-n // P) for n in lens) + 1
        cu, lens, table = batch_arrays(new, lens, P, pages, seed=axes)
        T = int(cu[-1])
        rng = np.random.RandomState(dim + axes)
        K, V = (torch.from_numpy(rng.randn(T, H, d).astype(np.float32)).to(dtype).cuda() for _ in range(2))
        pos = rng.randint(0, 5000, (axes, T)).astype(np.int32)
        params = dr.RopeParams(dim, layout=dr.ROPE_HALF if layout == "half" else dr.ROPE_INTERLEAVED, axis_pairs=pairs, mscale=1.25)
        k, v, ks, vs = filled_cache(pages, H, P, d, seed=1)
        cache = gpu_cache(k, v, ks, vs)
        dr.dr_cache_append(dr.Context(0), cache, dr.CacheBatch(*on_gpu(cu, lens, table), T), K, V, rope=params, positions=on_gpu(pos)[0])
        turned = o.rope(f64(K).transpose(1, 0, 2), pos, dim, layout, pairs, mscale=1.25).transpose(1, 0, 2)
        wk, wks = o.append(k, ks, turned.astype(np.float32), cu, lens, table, False)
        wv, wvs = o.append(v, vs, f64(V), cu, lens, table, True)
        assert np.array_equal(f64(cache.k_scale), wks) and np.array_equal(f64(cache.v_scale), wvs)
        assert np.array_equal(codes(cache.v), wv) and np.array_equal(codes(cache.k), wk)
