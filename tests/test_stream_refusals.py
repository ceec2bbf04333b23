"""What the streaming entry points refuse: the binding's checks (no GPU needed), and the library's own, before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2604_20470_amd as dr
from paper_2604_20470_amd import binding as bd


class _NoLibrary:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


class _Ctx:
    """Stands for a context of device 0; any call that gets through the binding's checks fails the test."""
    device, _h, _lib = 0, C.c_void_p(1), None

    def __init__(self):
        self._lib = type("L", (), {n: staticmethod(lambda *a: pytest.fail("the library was called")) for n in
                                   ("dr_rope_fwd", "dr_rope_bwd", "dr_cache_append", "dr_cache_attn_fwd")})()


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_cache_tensors_must_fit_together():
    k, v, s = torch.zeros(3, 2, 32, 64, dtype=torch.uint8), torch.zeros(3, 2, 64, 32, dtype=torch.uint8), torch.ones(3, 2)
    assert dr.PagedCache.of(k, v, s, s.clone()).page_tokens == 32
    for bad in ((k, k, s, s), (k.float(), v, s, s), (k, v, s[:2], s), (k, v, s.double(), s), (k.transpose(2, 3), v, s, s), (k[0], v[0], s, s)):
        with pytest.raises(dr.DRError):
            dr.PagedCache.of(*bad)


def test_batch_arrays_must_fit_together():
    dr.CacheBatch(_i32(3), _i32(2), _i32(2, 5), 7)
    for bad in ((_i32(2), _i32(2), _i32(2, 5)), (_i32(3), _i32(2), _i32(3, 5)), (_i32(3).long(), _i32(2), _i32(2, 5)), (_i32(3), _i32(2), _i32(5, 2).t()),
                (_i32(3), _i32(2, 1), _i32(2, 5)), (_i32(6)[::2], _i32(2), _i32(2, 5))):
        with pytest.raises(dr.DRError):
            dr.CacheBatch(*bad, 7)


def test_keys_and_values_read_back_what_the_codes_stand_for():
    cache = dr.PagedCache(2, 1, 32, 64, device="cpu")
    cache.k.view(torch.uint8)[1, 0, 3, 5] = 0x38
    cache.v.view(torch.uint8)[1, 0, 5, 3] = 0xb8
    cache.k_scale[1], cache.v_scale[1] = 4.0, 0.5
    assert float(cache.keys()[1, 0, 3, 5]) == 4.0 and float(cache.values()[1, 0, 3, 5]) == -0.5


def test_tensors_on_another_device_or_of_another_form_are_refused():
    ctx, rope = _Ctx(), dr.RopeParams(64)
    x, pos = torch.zeros(1, 2, 3, 64), _i32(1, 3)
    cache, batch = dr.PagedCache(2, 2, 32, 64, device="cpu"), dr.CacheBatch(_i32(2), _i32(1), _i32(1, 1), 3)
    t = torch.zeros(3, 2, 64)
    calls = [lambda: dr.dr_rope_fwd(ctx, rope, x, pos, x), lambda: dr.dr_rope_fwd(ctx, rope, x, pos, x[:, :1]), lambda: dr.dr_rope_bwd(ctx, rope, x[0], pos, x[0]),
             lambda: dr.dr_rope_fwd(ctx, rope, x, pos, x.bfloat16()), lambda: dr.dr_rope_fwd(ctx, rope, x.transpose(2, 3), pos, x.transpose(2, 3)),
             lambda: dr.dr_cache_append(ctx, cache, batch, t, t), lambda: dr.dr_cache_append(ctx, cache, batch, t[:2], t[:2]),
             lambda: dr.dr_cache_append(ctx, cache, batch, t, t.bfloat16()), lambda: dr.dr_cache_attn_fwd(ctx, cache, batch, t, t.clone()),
             lambda: dr.dr_cache_attn_fwd(ctx, cache, batch, t[..., :32], t[..., :32])]
    for call in calls:
        with pytest.raises(dr.DRError) as e:
            call()
        assert e.value.status_name == "DR_ERR_INVALID_ARG"


# ---- the library's own checks ------------------------------------------------------------------------------

def _status(ctx, call):
    st = call()
    return bd._STATUS[st], ctx._lib.dr_last_error(ctx._h).decode()


@pytest.mark.gpu
def test_rope_refusals():
    ctx = dr.Context(0)
    x = torch.zeros(2, 3, 4, 64, device="cuda")
    pos = torch.zeros(1, 4, dtype=torch.int32, device="cuda")

    def shape(**kw):
        f = dict(B=2, H=3, N=4, d=64, dtype=0, reserved0=0, stride_b=768, stride_h=256, stride_n=64, out_stride_b=768, out_stride_h=256, out_stride_n=64)
        f.update(kw)
        return bd.RopeShape(*f.values())

    def params(dim=64, **kw):
        p = dr.RopeParams(dim)
        for k, v in kw.items():
            if k == "axis_pairs":
                p.axis_pairs[:] = v
            elif k == "reserved":
                p.reserved[0] = v
            else:
                setattr(p, k, v)
        return p

    def call(s=None, p=None, X=x.data_ptr(), P=pos.data_ptr(), Y=x.data_ptr(), pb=0, pa=4, fn=ctx._lib.dr_rope_fwd):
        return lambda: fn(ctx._h, C.byref(s or shape()), C.byref(p or params()), X, P, pb, pa, Y, None)

    assert call()() == 0 and call(fn=ctx._lib.dr_rope_bwd)() == 0
    invalid = [call(s=shape(B=-1)), call(s=shape(dtype=2)), call(s=shape(reserved0=1)), call(s=shape(stride_n=-64)), call(s=shape(out_stride_h=0)),
               call(X=None), call(P=None), call(Y=None), call(X=x.data_ptr() + 2), call(P=pos.data_ptr() + 1), call(pb=-1), call(s=shape(stride_n=128)),
               call(p=params(dim=66, axis_pairs=[33, 0, 0])), call(p=params(dim=63)), call(p=params(dim=-2)), call(p=params(layout=2)), call(p=params(axes=0)), call(p=params(axes=4)),
               call(p=params(axis_pairs=[31, 0, 0])), call(p=params(axis_pairs=[30, 2, 0])), call(p=params(axis_pairs=[33, -1, 0], axes=2)),
               call(p=params(theta=0.0)), call(p=params(theta=float("nan"))), call(p=params(factor=0.5)), call(p=params(original_len=-1.0)),
               call(p=params(original_len=8.0, ramp_low=3.0, ramp_high=3.0)), call(p=params(mscale=float("inf"))), call(p=params(reserved=1)),
               call(p=params(theta=1e-300))]
    for c in invalid:
        st, text = _status(ctx, c)
        assert st == "DR_ERR_INVALID_ARG" and text, (invalid.index(c), st, text)
    for c in (call(s=shape(d=63)), call(s=shape(d=258)), call(s=shape(B=70000)), call(s=shape(d=0))):
        assert _status(ctx, c)[0] == "DR_ERR_UNSUPPORTED"
    assert ctx._lib.dr_rope_fwd(ctx._h, None, C.byref(params()), x.data_ptr(), pos.data_ptr(), 0, 4, x.data_ptr(), None) == 1
    assert ctx._lib.dr_rope_fwd(ctx._h, C.byref(shape()), None, x.data_ptr(), pos.data_ptr(), 0, 4, x.data_ptr(), None) == 1
    assert ctx._lib.dr_rope_fwd(None, C.byref(shape()), C.byref(params()), x.data_ptr(), pos.data_ptr(), 0, 4, x.data_ptr(), None) == 1
    # nothing to do
    assert call(s=shape(N=0), X=None, Y=None, P=None)() == 0
    empty = torch.zeros(1, 2, 0, 64, device="cuda")
    dr.dr_rope_fwd(ctx, dr.RopeParams(64), empty, torch.zeros(1, 0, dtype=torch.int32, device="cuda"), empty)


@pytest.mark.gpu
def test_cache_refusals():
    ctx = dr.Context(0)
    cache = dr.PagedCache(4, 2, 32, 64)
    arrays = [torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([0, 3], [3], [[1, 2]])]
    batch = dr.CacheBatch(*arrays, 3)
    q, o = torch.zeros(3, 4, 64, device="cuda"), torch.zeros(3, 4, 64, device="cuda")
    kv = torch.zeros(3, 2, 64, device="cuda")

    def struct(of, **kw):
        new = type(of)()
        C.memmove(C.byref(new), C.byref(of), C.sizeof(of))
        for k, v in kw.items():
            setattr(new, k, v)
        return new

    strides = bd._TokenStrides(0, 0, 128, 64, 128, 64)
    wide = bd._TokenStrides(0, 0, 256, 64, 256, 64)

    def append(c=cache.struct, b=batch.struct, s=strides, K=kv.data_ptr(), V=kv.data_ptr(), r=None, P=None, pa=0):
        return lambda: ctx._lib.dr_cache_append(ctx._h, C.byref(c), C.byref(b), C.byref(s), K, V, C.byref(r) if r else None, P, pa, None)

    def attend(c=cache.struct, b=batch.struct, s=wide, heads=4, Q=q.data_ptr(), O=o.data_ptr(), causal=1, lse=None):
        return lambda: ctx._lib.dr_cache_attn_fwd(ctx._h, C.byref(c), C.byref(b), C.byref(s), heads, Q, O, causal, lse, None)

    assert append()() == 0 and attend()() == 0
    for call in (append, attend):
        invalid = [call(c=struct(cache.struct, pages=0)), call(c=struct(cache.struct, heads=-1)), call(c=struct(cache.struct, k=None)),
                   call(c=struct(cache.struct, v_scale=None)), call(c=struct(cache.struct, v=cache.v.data_ptr() + 8)),
                   call(c=struct(cache.struct, k_scale=cache.k_scale.data_ptr() + 2)), call(b=struct(batch.struct, sequences=-1)),
                   call(b=struct(batch.struct, tokens=-1)), call(b=struct(batch.struct, max_pages=-1)), call(b=struct(batch.struct, reserved0=1)),
                   call(b=struct(batch.struct, cu=None)), call(b=struct(batch.struct, lens=None)), call(b=struct(batch.struct, page_table=None)),
                   call(b=struct(batch.struct, table_stride=1)), call(b=struct(batch.struct, lens=arrays[1].data_ptr() + 1)),
                   call(s=bd._TokenStrides(2, 0, 256, 64, 256, 64)), call(s=bd._TokenStrides(0, 1, 256, 64, 256, 64)), call(s=bd._TokenStrides(0, 0, -256, 64, 256, 64))]
        for c in invalid:
            st, text = _status(ctx, c)
            assert st == "DR_ERR_INVALID_ARG" and text, (call.__name__, invalid.index(c), st, text)
        for c in (call(c=struct(cache.struct, page_tokens=16)), call(c=struct(cache.struct, d=96)), call(c=struct(cache.struct, heads=1 << 17)),
                  call(b=struct(batch.struct, tokens=1 << 30)), call(b=struct(batch.struct, max_pages=1 << 26, table_stride=1 << 26)),
                  call(b=struct(batch.struct, sequences=1 << 24))):
            assert _status(ctx, c)[0] == "DR_ERR_UNSUPPORTED"
        assert call(b=struct(batch.struct, tokens=0, cu=None, lens=None, page_table=None))() == 0
        assert call(b=struct(batch.struct, sequences=0, cu=None, lens=None, page_table=None))() == 0
    three = dr.RopeParams(64, axis_pairs=[10, 11, 11])
    for c in (append(K=None), append(V=None), append(K=kv.data_ptr() + 1), append(r=three), append(r=dr.RopeParams(66)), append(pa=-1),
              attend(Q=None), attend(O=None), attend(O=q.data_ptr()), attend(heads=3), attend(heads=0), attend(causal=2), attend(Q=q.data_ptr() + 8),
              attend(s=bd._TokenStrides(0, 0, 258, 64, 256, 64)), attend(s=bd._TokenStrides(0, 0, 256, 64, 256, 0)), attend(lse=o.data_ptr() + 2)):
        st, text = _status(ctx, c)
        assert st == "DR_ERR_INVALID_ARG" and text, (st, text)
    with pytest.raises(dr.DRError):
        dr.dr_cache_append(ctx, cache, batch, q, q)                                        # four heads into a cache of two
    with pytest.raises(dr.DRError):
        dr.dr_cache_attn_fwd(ctx, cache, batch, q, o, lse=torch.zeros(3, 4, device="cuda"))
    with pytest.raises(dr.DRError):
        dr.dr_cache_append(ctx, cache, batch, kv, kv, positions=torch.zeros(1, 3, dtype=torch.int32, device="cuda"))
    with pytest.raises(dr.DRError):
        dr.dr_cache_attn_fwd(ctx, cache, batch, q.half(), o.half())


@pytest.mark.gpu
def test_batches_beyond_the_launch_grid_are_refused():
    ctx, cache = dr.Context(0), dr.PagedCache(2, 2, 64, 64)
    one = [torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([0, 3], [3], [[1]])]
    many = torch.zeros(1, 2, 64, device="cuda").expand((1 << 30) - 1, 2, 64)
    with pytest.raises(dr.DRError, match="UNSUPPORTED.*launch grid"):
        dr.dr_cache_append(ctx, cache, dr.CacheBatch(*one, (1 << 30) - 1), many, many)
    S = (1 << 24) - 1
    cu, lens = torch.zeros(S + 1, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
    q = torch.zeros(3, 4, 64, device="cuda")
    with pytest.raises(dr.DRError, match="UNSUPPORTED.*launch grid"):
        dr.dr_cache_attn_fwd(ctx, cache, dr.CacheBatch(cu, lens, torch.zeros(S, 1, dtype=torch.int32, device="cuda"), 3), q, torch.empty_like(q))
    # the context goes on
    o = torch.empty_like(q)
    dr.dr_cache_attn_fwd(ctx, cache, dr.CacheBatch(*one, 3), q, o)
    torch.cuda.synchronize()
    assert torch.isfinite(o).all()
