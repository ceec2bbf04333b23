"""dr_rope_fwd / dr_rope_bwd over more work items than one launch holds (2^32 threads along an axis)."""
import pytest
import torch

import paper_2604_20470_amd as dr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", [dr.ROPE_HALF, dr.ROPE_INTERLEAVED], ids=["half", "interleaved"])
def test_more_work_items_than_a_launch_holds(layout):
    """One pair and 254 copied channels, one by one: 255 items for each of 16.85 million tokens, which all have the same input row."""
    d, N, ctx, rope = 256, (1 << 24) + 70000, dr.Context(0), dr.RopeParams(2, layout=layout)
    x = torch.randn(d, device="cuda").bfloat16()
    X, Y = x.expand(1, 1, N, d), torch.full((1, 1, N, d), 7.0, device="cuda", dtype=torch.bfloat16)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")[None]
    assert 255 * N > 1 << 32
    for call, sign in ((dr.dr_rope_fwd, 1.0), (dr.dr_rope_bwd, -1.0)):
        Y.fill_(7.0)
        call(ctx, rope, X, pos, Y)
        for a in range(0, N, 1 << 21):
            y = Y[0, 0, a:a + (1 << 21)]
            assert (y[:, 2:] == x[2:]).all(), a
            phi, (p, q) = pos[0, a:a + (1 << 21)].double(), x[:2].double()
            c, s = torch.cos(phi), sign * torch.sin(phi)
            # 8 roundings of fp32, as elsewhere, and the result's own
            for got, want in ((y[:, 0], p * c - q * s), (y[:, 1], q * c + p * s)):
                assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 8 * 2.0 ** -24 * (p.abs() + q.abs())).all(), a
