"""Results of the norms that begin inside their vectors, or inside each other, are refused; rows that lie beside each other in one tensor are not."""
import pytest
import torch

import paper_2604_20470_amd as dr

pytestmark = pytest.mark.gpu
V = dr.NormVectors


def setup(tokens=4):
    g = torch.Generator().manual_seed(0)
    x, br, dy = (torch.randn(2, tokens, 64, generator=g).cuda() for _ in range(3))
    m = {k: torch.randn(2, 2 if tokens else 0, 64, generator=g).cuda() for k in ("gate", "scale", "shift")}
    return dr.Context(0), dr.NormParams(mod_tokens=2, branch_norm=True), x, br, dy, m, torch.randn(64, generator=g).cuda()


def test_forward():
    ctx, norm, x, br, _, m, w = setup()
    rows = {k: t.repeat(1, 2, 1) for k, t in m.items()}
    each = dr.NormParams(mod_tokens=1, branch_norm=True)
    for bad in (lambda: dr.dr_norm_fwd(ctx, each, x, rows["scale"], branch=br, vectors=V(**rows)), lambda: dr.dr_norm_fwd(ctx, each, x, br.clone(), branch=br, total=rows["gate"], vectors=V(**rows))):
        with pytest.raises(dr.DRError, match="overlap"):
            bad()
    one = dr.NormParams()
    with pytest.raises(dr.DRError, match="overlap"):
        dr.dr_norm_fwd(ctx, one, x[:1, :1], w.view(1, 1, 64), vectors=V(weight=w))
    y = torch.empty(65, device="cuda")
    with pytest.raises(dr.DRError, match="overlap"):
        dr.dr_norm_fwd(ctx, one, x[:1, :1], y[1:].view(1, 1, 64), vectors=V(bias=y[:64]))
    assert torch.equal(rows["scale"], m["scale"].repeat(1, 2, 1))


@pytest.mark.parametrize("name", ["gate", "scale", "shift", "weight", "bias", "branch_weight"])
def test_a_gradient_on_a_vector(name):
    ctx, norm, x, br, dy, m, w = setup()
    vec = dict(m, weight=w, bias=w.clone(), branch_weight=w.clone())
    for other in vec:
        if vec[other].shape != vec[name].shape:
            continue
        kept = vec[other].clone()
        with pytest.raises(dr.DRError, match="overlap"):
            dr.dr_norm_bwd(ctx, norm, x, dy, torch.empty_like(x), branch=br, vectors=V(**vec), grads=V(**{name: vec[other]}))
        assert torch.equal(vec[other], kept)


def test_gradients_on_other_tensors():
    ctx, norm, x, br, dy, m, w = setup()
    each = dr.NormParams(mod_tokens=1)
    a, b = torch.empty_like(x), torch.empty(2, 2, 64, device="cuda")
    for bad in (lambda: dr.dr_norm_bwd(ctx, each, x, dy, a, grads=V(scale=x)), lambda: dr.dr_norm_bwd(ctx, each, x, dy, a, grads=V(scale=dy)),
                lambda: dr.dr_norm_bwd(ctx, each, x, dy, a, grads=V(shift=a)), lambda: dr.dr_norm_bwd(ctx, each, x, dy, a, dtotal=br, grads=V(shift=br)),
                lambda: dr.dr_norm_bwd(ctx, each, x, dy, a, branch=br, grads=V(gate=br)), lambda: dr.dr_norm_bwd(ctx, norm, x, dy, a, branch=br, grads=V(gate=b, scale=b)),
                lambda: dr.dr_norm_bwd(ctx, norm, x, dy, a, branch=br, grads=V(weight=w, bias=w)),
                lambda: dr.dr_norm_bwd(ctx, norm, x, dy, a, branch=br, grads=V(weight=b.view(-1)[:64], bias=b.view(-1)[63:127])),
                lambda: dr.dr_norm_bwd(ctx, norm, x, dy, a, branch=br, vectors=V(weight=w), grads=V(weight=b.view(-1)[:64], shift=b)),
                lambda: dr.dr_norm_bwd(ctx, dr.NormParams(mod_tokens=1), x, dy, a, vectors=V(scale=a))):
        with pytest.raises(dr.DRError, match="overlap"):
            bad()


def test_without_tokens_a_weight_stays():
    ctx, norm, x, br, dy, m, w = setup(0)
    kept = w.clone()
    with pytest.raises(dr.DRError, match="overlap"):
        dr.dr_norm_bwd(ctx, dr.NormParams(), x, dy, x, vectors=V(weight=w), grads=V(weight=w))
    assert torch.equal(w, kept)


def test_rows_beside_each_other():
    """Modulations out of one product, and their gradients into one."""
    ctx, norm, x, br, dy, m, w = setup()
    out, grad = torch.stack([m["gate"], m["scale"], m["shift"]], 2), torch.full((2, 2, 3, 64), 7.0, device="cuda")
    both = torch.cat([w, w, w, w])
    dx, dx2, db = (torch.empty_like(x) for _ in range(3))
    apart = {k: torch.empty_like(t) for k, t in m.items()}
    dw, dbias = torch.empty_like(w), torch.empty_like(w)
    dr.dr_norm_bwd(ctx, norm, x, dy, dx, branch=br, dbranch=db, vectors=V(**m, weight=w), grads=V(**apart, weight=dw, bias=dbias))
    dr.dr_norm_bwd(ctx, norm, x, dy, dx2, branch=br, vectors=V(gate=out[:, :, 0], scale=out[:, :, 1], shift=out[:, :, 2], weight=both[64:128]),
                   grads=V(gate=grad[:, :, 0], scale=grad[:, :, 1], shift=grad[:, :, 2], weight=both[:64], bias=both[128:192]))
    assert torch.equal(dx, dx2) and torch.equal(both[:64], dw) and torch.equal(both[128:192], dbias) and torch.equal(both[64:128], w)
    assert all(torch.equal(grad[:, :, i], apart[k]) for i, k in enumerate(("gate", "scale", "shift")))
