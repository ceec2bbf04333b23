"""Pins of the streaming oracle: hand-made values, properties, and gradients by differences."""
import math

import numpy as np
import pytest
import torch

from oracle import streaming_oracle as o


def test_every_code_encodes_to_itself_and_matches_torch():
    c = np.arange(256, dtype=np.uint8)
    fine = (c & 0x7f) != 0x7f
    assert np.array_equal(o.encode(o.decode(c[fine])), c[fine])
    assert np.array_equal(o.decode(c)[fine], torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()[fine])
    x = np.concatenate([np.linspace(-448, 448, 20001), np.linspace(-0.05, 0.05, 20001)]).astype(np.float32)
    assert np.array_equal(o.encode(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert list(o.encode([math.inf, -math.inf, 1e9])) == [0x7e, 0xfe, 0x7e] and math.isnan(o.decode(o.encode(math.nan)))


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.0000001, 1), (224.0, -1), (1.75, -8), (1.7500001, -7), (1.0, -8), (0.0, -100), (1e-38, -100), (3.4e38, 120)])
def test_exponent(amax, e):
    assert o.exponent(amax) == e and amax <= 448.0 * 2.0 ** e


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_keeps_lengths_and_depends_on_distance(layout):
    rng = np.random.RandomState(1)
    q, k = rng.randn(1, 64), rng.randn(1, 64)
    at = lambda x, p: o.rope(x, np.array([[p]]), 64, layout)
    assert np.allclose(np.linalg.norm(at(q, 977)), np.linalg.norm(q), rtol=1e-13)
    assert np.allclose((at(q, 977) * at(k, 970)).sum(), (at(q, 7) * at(k, 0)).sum(), rtol=1e-10)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_backward_is_the_gradient_by_differences(layout):
    rng = np.random.RandomState(2)
    args = dict(dim=12, layout=layout, axis_pairs=[2, 3, 1], mscale=1.3, factor=4.0, original_len=64.0)
    pos = rng.randint(-50, 50, (3, 3))
    x, g = rng.randn(3, 16), rng.randn(3, 16)
    got = o.rope(g, pos, backward=True, **args)
    for i in np.ndindex(3, 16):
        step = np.zeros_like(x)
        step[i] = 1e-4
        diff = ((o.rope(x + step, pos, **args) - o.rope(x - step, pos, **args)) * g).sum() / 2e-4
        assert abs(diff - got[i]) < 1e-9


def test_attention_of_one_key_returns_its_value_and_hidden_rows_are_zero():
    rng = np.random.RandomState(3)
    k, v = rng.randint(0, 0x50, (2, 1, 32, 64)).astype(np.uint8), rng.randint(0, 0x50, (2, 1, 64, 32)).astype(np.uint8)
    one = np.ones((2, 1), np.float32)
    q = rng.randn(3, 2, 64)
    out, lse = o.attend(q, k, v, one, one, np.array([0, 3]), np.array([1]), np.array([[1]]), True)
    assert (out[:2] == 0).all() and np.isneginf(lse[:, :2]).all()
    assert np.allclose(out[2], o.decode(v[1, 0, :, 0])[None])
    assert np.allclose(lse[:, 2], q[2] @ o.decode(k[1, 0, 0]) / 8)


def test_appending_in_two_steps_is_appending_at_once_when_the_scale_does_not_grow():
    rng = np.random.RandomState(4)
    x = rng.randn(40, 2, 64).astype(np.float32).astype(np.float64)
    x[0] *= 8
    table = np.array([[2, 0]], np.int32)
    zero, one = np.zeros((3, 2, 32, 64), np.uint8), np.ones((3, 2))
    a = o.append(zero, one, x, [0, 40], [40], table, False)
    b = o.append(zero, one, x[:7], [0, 7], [7], table, False)
    b = o.append(*b, x[7:], [0, 33], [40], table, False)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
