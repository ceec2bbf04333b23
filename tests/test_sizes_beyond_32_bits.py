"""Sizes that the library's 32 bits do not hold are refused, where a structure would take the lower 32 of them and a call do a part of its work (no GPU needed: rows and columns without
memory of their own, and a library that must not be called)."""
import ctypes as C

import pytest
import torch

import paper_2604_20470_amd as dr

FAR = 2 ** 32 + 3


class _Cuda(torch.Tensor):
    def get_device(self):
        return 0


def _gpu(*shape, dtype=torch.float32):
    return torch.zeros((1,) * len(shape), dtype=dtype).expand(shape).as_subclass(_Cuda)


class _Ctx:
    device, _h = 0, C.c_void_p(1)

    def __init__(self):
        self._lib = type("L", (), {n: staticmethod(lambda *a: pytest.fail("the library was called")) for n in ("dr_norm_fwd", "dr_norm_bwd", "dr_rope_fwd", "dr_rope_bwd")})()


@pytest.mark.parametrize("shape", [(1, FAR, 1), (FAR, 1, 1), (1, 1, FAR), (1, 2 ** 31, 1)])
def test_norms(shape):
    x = _gpu(*shape)
    with pytest.raises(dr.DRError, match="below"):
        dr.dr_norm_fwd(_Ctx(), dr.NormParams(), x, x, stream=0)
    with pytest.raises(dr.DRError, match="below"):
        dr.dr_norm_bwd(_Ctx(), dr.NormParams(), x, x, x, stream=0)


@pytest.mark.parametrize("shape", [(1, 1, FAR, 2), (1, FAR, 1, 2), (FAR, 1, 1, 2)])
def test_rotary_positions(shape):
    x = _gpu(*shape)
    with pytest.raises(dr.DRError, match="below"):
        dr.dr_rope_fwd(_Ctx(), dr.RopeParams(2), x, _gpu(1, shape[2], dtype=torch.int32), x, stream=0)


def test_batches():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(dr.DRError, match="below"):
        dr.CacheBatch(i32(2), i32(1), i32(1, 1), FAR)
    dr.CacheBatch(i32(2), i32(1), i32(1, 1), 2 ** 31 - 1)


def test_params_do_not_wrap():
    assert dr.NormParams(mod_tokens=-2 ** 32).mod_tokens == -1 and dr.NormParams(mod_tokens=2 ** 33).mod_tokens == 2 ** 31 - 1
    assert dr.NormParams(kind=2 ** 32).kind == 2 ** 31 - 1 and dr.NormParams(kind=-2 ** 32 + 1).kind == -1
    assert dr.NormParams(dr.NORM_RMS, mod_tokens=7).kind == 1 and dr.NormParams(mod_tokens=7).mod_tokens == 7
