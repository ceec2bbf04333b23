"""dr_rope_fwd / dr_rope_bwd against the fp64 oracle, by differences, and in the forms in which callers have their tensors."""
import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr
from oracle import streaming_oracle as o
from stream_helpers import HALF_BF16, ULP32, assert_close, f64

pytestmark = pytest.mark.gpu
KINDS = {"half": dr.ROPE_HALF, "interleaved": dr.ROPE_INTERLEAVED}


def _args(dim, layout, pairs, **more):
    return dr.RopeParams(dim, layout=KINDS[layout], axis_pairs=pairs, **more), dict(dim=dim, layout=layout, axis_pairs=pairs, **more)


def _partner_sum(x, dim, layout):
    """|x0| + |x1| of every channel's pair."""
    a = np.abs(x)
    s = a.copy()
    if layout == "half":
        t = a[..., :dim // 2] + a[..., dim // 2:dim]
        s[..., :dim // 2] = t
        s[..., dim // 2:dim] = t
    else:
        t = a[..., 0:dim:2] + a[..., 1:dim:2]
        s[..., 0:dim:2] = t
        s[..., 1:dim:2] = t
    return s


def _check(got, x, positions, args, backward, bf16):
    # cosine and sine within 4 roundings (argument, polynomial, mscale), a product and a sum: 8 roundings of |x0| + |x1| at most
    want = np.stack([o.rope(x[b], positions if positions.ndim == 2 else positions[b], backward=backward, **args) for b in range(x.shape[0])])
    tol = 8 * ULP32 * abs(args.get("mscale", 1.0)) * _partner_sum(x, args["dim"], args["layout"]) + (HALF_BF16 if bf16 else ULP32) * np.abs(want)
    assert_close(f64(got), want, tol, "rope")


CASES = [  # B, H, N, d, dim, layout, pairs, far
    (1, 1, 1, 64, 64, "half", [32], 1),
    (2, 3, 37, 128, 128, "half", [64], 4000000),
    (1, 9, 130, 128, 128, "interleaved", [22, 21, 21], 60),
    (1, 40, 5, 128, 96, "half", [16, 16, 16], 500),
    (3, 2, 61, 64, 32, "interleaved", [16], 75600),
    (1, 2, 33, 70, 38, "half", [7, 6, 6], 90),           # no whole vectors
    (2, 2, 19, 64, 38, "interleaved", [19], 200000000),     # (the oracle's own angles lose 2e-16 of this)
    (1, 4, 257, 256, 256, "half", [128], 1000),
    (1, 2, 7, 2, 2, "half", [1], 10),
    (1, 2, 7, 16, 0, "half", [0], 10),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:6])))
def test_against_the_oracle(case, dtype):
    B, H, N, d, dim, layout, pairs, far = case
    rng = np.random.RandomState(N + d)
    scaling = dict(factor=4.0, original_len=512.0, mscale=1.1386) if N % 2 else {}
    params, args = _args(dim, layout, pairs, **scaling)
    pos = rng.randint(-far, far, (B, len(pairs), N) if B > 1 else (len(pairs), N)).astype(np.int32)
    x = torch.from_numpy(rng.randn(B, H, N, d).astype(np.float32)).to(dtype).cuda()
    p, ctx = torch.from_numpy(pos).cuda(), dr.Context(0)
    y = torch.full_like(x, float("nan"))
    dr.dr_rope_fwd(ctx, params, x, p, y)
    _check(y, f64(x), pos, args, False, dtype == torch.bfloat16)
    dr.dr_rope_bwd(ctx, params, x, p, y)
    _check(y, f64(x), pos, args, True, dtype == torch.bfloat16)


def test_linear_scaling_equals_divided_positions():
    ctx = dr.Context(0)
    x = torch.randn(1, 2, 50, 64, device="cuda")
    pos = torch.arange(50, dtype=torch.int32, device="cuda")[None]
    a, b = torch.empty_like(x), torch.empty_like(x)
    dr.dr_rope_fwd(ctx, dr.RopeParams(64, factor=8.0), x, pos * 8, a)
    dr.dr_rope_fwd(ctx, dr.RopeParams(64), x, pos, b)
    assert torch.equal(a, b)                     # the frequencies are divided by a power of two, the positions multiplied by it


def test_the_gradient_by_differences():
    ctx = dr.Context(0)
    params = dr.RopeParams(12, layout=dr.ROPE_INTERLEAVED, axis_pairs=[3, 2, 1], mscale=1.25)
    pos = torch.randint(-40, 40, (3, 4), dtype=torch.int32, device="cuda")
    x, g = torch.randn(1, 2, 4, 16, device="cuda"), torch.randn(1, 2, 4, 16, device="cuda")
    dx, y1, y2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    dr.dr_rope_bwd(ctx, params, g, pos, dx)
    step = torch.randn_like(x)
    dr.dr_rope_fwd(ctx, params, x + step, pos, y1)
    dr.dr_rope_fwd(ctx, params, x - step, pos, y2)
    lhs, rhs = float(((y1 - y2).double() * g.double()).sum()) / 2, float((dx.double() * step.double()).sum())
    # the operator is linear: only roundings differ, at most 16 of them on each of the 128 products
    assert abs(lhs - rhs) <= 16 * ULP32 * 1.25 * float(((x.abs() + 2 * step.abs()) * g.abs()).sum()) * 2


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_strides_alignment_and_in_place(dtype):
    ctx, d, N, H = dr.Context(0), 64, 21, 3
    params, args = _args(64, "half", [32])
    pos = torch.arange(N, dtype=torch.int32, device="cuda")[None] * 7
    buf = torch.randn(2, N, 3, H, d, device="cuda").to(dtype)
    want = torch.empty(2, H, N, d, device="cuda", dtype=dtype)
    x = buf[:, :, 1].permute(0, 2, 1, 3)
    dr.dr_rope_fwd(ctx, params, x, pos, want)
    _check(want, f64(x), pos.cpu().numpy(), args, False, dtype == torch.bfloat16)
    # one element off the alignment, into rows of another stride
    flat = torch.zeros(2 * H * N * d + 1, device="cuda", dtype=dtype)
    odd = flat[1:].view(2, H, N, d)
    odd.copy_(x)
    out = torch.zeros(2, H, N, d + 3, device="cuda", dtype=dtype)
    dr.dr_rope_fwd(ctx, params, odd, pos, out[..., :d])
    # the paths contract their sums differently: two roundings of fp32, and one of the result
    _check(out[..., :d], f64(x), pos.cpu().numpy(), args, False, dtype == torch.bfloat16)
    assert (out[..., d:] == 0).all()
    # a head shared by all (stride 0)
    dr.dr_rope_fwd(ctx, params, x[:, :1].expand(2, H, N, d), pos, out[..., :d])
    assert torch.equal(out[:, 0, :, :d], out[:, 2, :, :d])
    # in place, inside the projection's buffer: the rest of it stays
    before = buf.clone()
    dr.dr_rope_fwd(ctx, params, x, pos, x)
    assert torch.equal(x, want)
    assert torch.equal(buf[:, :, 0], before[:, :, 0]) and torch.equal(buf[:, :, 2], before[:, :, 2])


def test_far_positions_lose_nothing():
    """At position 2^31 - 1 the angle of the first pair is 2^31 - 1 radians."""
    ctx = dr.Context(0)
    pos = np.array([[2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, 123456789]], np.int32)
    x = torch.zeros(1, 1, 4, 64, device="cuda")
    x[..., :32] = 1
    y = torch.empty_like(x)
    dr.dr_rope_fwd(ctx, dr.RopeParams(64), x, torch.from_numpy(pos).cuda(), y)
    import math
    for n in range(4):
        p = int(pos[0, n])
        assert abs(float(y[0, 0, n, 0]) - math.cos(p)) < 4 * 2.0 ** -24 and abs(float(y[0, 0, n, 32]) - math.sin(p)) < 4 * 2.0 ** -24


def test_values_that_are_no_numbers_stay_in_their_pair():
    ctx = dr.Context(0)
    x = torch.randn(1, 1, 3, 64, device="cuda", dtype=torch.bfloat16)
    want, y = torch.empty_like(x), torch.empty_like(x)
    pos = torch.tensor([[1, 2, 3]], dtype=torch.int32, device="cuda")
    dr.dr_rope_fwd(ctx, dr.RopeParams(64), x, pos, want)
    x[0, 0, 1, 5] = float("nan")
    dr.dr_rope_fwd(ctx, dr.RopeParams(64), x, pos, y)
    hit = torch.isnan(y)
    assert hit.nonzero().tolist() == [[0, 0, 1, 5], [0, 0, 1, 37]] and torch.equal(y[~hit], want[~hit])
