"""How far the rotation's cosines and sines are off, against angles formed with 60 digits: what include/dynamicrad.h states."""
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

import paper_2604_20470_amd as dr

pytestmark = pytest.mark.gpu
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


@pytest.mark.parametrize("theta", [10000.0, 1.0, 500000.0])
def test_cosines_and_sines(theta):
    getcontext().prec = 60
    d, n = 64, 600
    rng = np.random.RandomState(7)
    pos = np.concatenate([rng.randint(-2 ** 31, 2 ** 31, n), rng.randint(-5000, 5000, n), [0, 1, -1, 2 ** 31 - 1, -2 ** 31]]).astype(np.int64)
    x = torch.zeros(1, 1, len(pos), d, device="cuda")
    x[..., :32] = 1.0                            # y0 = cos, y1 = sin
    y = torch.empty_like(x)
    dr.dr_rope_fwd(dr.Context(0), dr.RopeParams(d, theta=theta), x, torch.from_numpy(pos.astype(np.int32))[None].cuda(), y)
    y = y[0, 0].double().cpu().numpy()
    for j in range(32):
        turns = (-(Decimal(theta).ln() * j / 32)).exp() / (2 * PI)
        phase = np.array([float((Decimal(int(p)) * turns) % 1) for p in pos]) * (2 * np.pi)
        # the angle's 2^-31 and 2^-63 for each unit of position, in radians; 2^-23 of fp32; what the 53 bits of `phase` lose
        tol = 2 * np.pi * (2.0 ** -31 + np.abs(pos) * 2.0 ** -63) + 2.0 ** -23 + 2.0 ** -49
        assert (np.abs(y[:, j] - np.cos(phase)) <= tol).all() and (np.abs(y[:, 32 + j] - np.sin(phase)) <= tol).all(), j
