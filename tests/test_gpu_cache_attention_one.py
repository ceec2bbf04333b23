"""dr_cache_attn_fwd of one token, or one head, whose tensors carry any stride along that dimension: nobody reads it."""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from stream_helpers import batch_arrays, filled_cache, gpu_cache, on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_strides_of_a_dimension_of_one(dtype):
    d, P = 64, 32
    for tokens, heads in ((1, 4), (5, 1)):
        cu, lens, table = batch_arrays([tokens], [90], P, 4)
        cache, batch = gpu_cache(*filled_cache(4, 1, P, d, seed=1)), dr.CacheBatch(*on_gpu(cu, lens, table), tokens)
        q = torch.from_numpy(np.random.RandomState(3).randn(tokens, heads, d).astype(np.float32)).to(dtype).cuda()
        want, got = torch.empty_like(q), torch.empty_like(q)
        dr.dr_cache_attn_fwd(dr.Context(0), cache, batch, q, want)
        for stride in (0, 1, 7, d + 3):
            strides = (stride, d, 1) if tokens == 1 else (d, stride, 1)
            got.fill_(7.0)
            dr.dr_cache_attn_fwd(dr.Context(0), cache, batch, q.as_strided(q.shape, strides), got.as_strided(q.shape, strides))
            assert torch.equal(got, want), (tokens, stride)
    # where there is more than one, a row that is not aligned is refused
    q = torch.zeros(2, 4, d, device="cuda", dtype=dtype)
    cu, lens, table = batch_arrays([2], [90], P, 4)
    with pytest.raises(dr.DRError, match="aligned"):
        dr.dr_cache_attn_fwd(dr.Context(0), cache, dr.CacheBatch(*on_gpu(cu, lens, table), 2), q[:, :1].as_strided((2, 1, d), (d + 1, 7, 1)), torch.empty(2, 1, d, device="cuda", dtype=dtype))
