"""NormVectors holds tensors, not addresses: a call takes them where they are by then (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2604_20470_amd as dr


class _Cuda(torch.Tensor):
    def get_device(self):
        return 0


def _gpu(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(_Cuda)


class _Ctx:
    """Stands for a context of device 0 and keeps what the library is given: addresses and strides of the six vectors, and their type."""
    device, _h = 0, C.c_void_p(1)

    def __init__(self):
        self.seen = []
        self._lib = type("L", (), {"dr_norm_fwd": staticmethod(lambda *a: self._take(a[1], a[3])), "dr_norm_bwd": staticmethod(lambda *a: self._take(a[1], a[10]))})()

    def _take(self, call, vectors):
        v = vectors._obj
        dtype = C.cast(call, C.POINTER(C.c_int32))[4]
        self.seen.append(([(r.data, r.stride_b, r.stride_n) for r in (v.gate, v.scale, v.shift)], [v.weight, v.bias, v.branch_weight], dtype))
        return 0

    def check(self, st):
        assert st == 0


@pytest.mark.parametrize("backward", [False, True])
def test_vectors_that_moved_are_found(backward):
    ctx, x = _Ctx(), _gpu(2, 4, 8)
    vec = dict(scale=_gpu(2, 2, 8), shift=_gpu(2, 2, 8), weight=_gpu(8), bias=_gpu(8))
    held, norm = dr.NormVectors(**vec), dr.NormParams(mod_tokens=2)

    def call():
        if backward:
            dr.dr_norm_bwd(ctx, norm, x, x, x, grads=held, stream=0)
        else:
            dr.dr_norm_fwd(ctx, norm, x, x, vectors=held, stream=0)
        rows, flat, _ = ctx.seen[-1]
        assert rows[0][0] is None and flat[2] is None
        assert rows[1:] == [(vec[k].data_ptr(), vec[k].stride(0), vec[k].stride(1)) for k in ("scale", "shift")]
        assert flat[:2] == [vec[k].data_ptr() for k in ("weight", "bias")]

    call()
    for k in vec:                                               # each alone, to another place of the same form
        before = vec[k].data_ptr()
        vec[k].data = _gpu(*vec[k].shape)
        assert vec[k].data_ptr() != before
        call()
    wide = _gpu(2, 2, 3, 8)                                     # rows of another stride
    vec["scale"].data = wide[:, :, 1]
    call()
    assert ctx.seen[-1][0][1][1:] == (48, 24)


def test_vectors_that_no_longer_fit_are_refused():
    ctx, x = _Ctx(), _gpu(2, 4, 8)
    for other in (_gpu(4), _gpu(16)[::2], _gpu(8, dtype=torch.float16)):
        w, b = _gpu(8), _gpu(8)
        held = dr.NormVectors(weight=w, bias=b)
        dr.dr_norm_fwd(ctx, dr.NormParams(), x, x, vectors=held, stream=0)
        w.set_(other) if other.dtype == w.dtype else setattr(w, "data", other)
        with pytest.raises(dr.DRError):
            dr.dr_norm_fwd(ctx, dr.NormParams(), x, x, vectors=held, stream=0)
    w, b = _gpu(8), _gpu(8)
    held, first = dr.NormVectors(weight=w, bias=b), w.detach()
    w.data = _gpu(8, dtype=torch.bfloat16)                      # and back: as at first
    with pytest.raises(dr.DRError):
        dr.dr_norm_fwd(ctx, dr.NormParams(), x, x, vectors=held, stream=0)
    w.data = first
    dr.dr_norm_fwd(ctx, dr.NormParams(), x, x, vectors=held, stream=0)
    assert ctx.seen[-1][1][:2] == [w.data_ptr(), b.data_ptr()] and ctx.seen[-1][2] == 0
    w = _gpu(8)
    held = dr.NormVectors(weight=w)
    w.data = _gpu(8, dtype=torch.bfloat16)                      # all of them in another type: that type
    dr.dr_norm_fwd(ctx, dr.NormParams(), x, x, vectors=held, stream=0)
    assert ctx.seen[-1][1][0] == w.data_ptr() and ctx.seen[-1][2] == 1
