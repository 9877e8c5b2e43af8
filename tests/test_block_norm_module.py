"""The block norm's module around its two calls: what autograd hands to the leaves.  On the CPU
the calls are stood in for by their formulas."""

import pytest

torch = pytest.importorskip("torch")

from paper_2606_18114_amd import ops  # noqa: E402
from paper_2606_18114_amd.qat import BlockNorm, BlockNormFn  # noqa: E402


def _norm(residual, y, w, eps=1e-5, *, residual_out=None, x=None):
    r = residual if y is None else residual + y
    n = (r / torch.sqrt(r.pow(2).mean(-1, keepdim=True) + eps) * w).to(torch.bfloat16)
    if residual_out is not None:
        r = residual_out.copy_(r)
    return n if x is None else x.copy_(n), r


def _norm_bwd(residual, w, dx, dresidual=None, eps=1e-5, *, dr=None):
    rho = 1 / torch.sqrt(residual.pow(2).mean(-1, keepdim=True) + eps)
    a = dx.float() * w
    d = rho * a - residual * rho ** 3 * (a * residual).mean(-1, keepdim=True)
    return d if dresidual is None else d + dresidual, (dx.float() * residual * rho).sum(0)


@pytest.fixture(params=["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "cpu":
        monkeypatch.setattr(ops, "block_norm", _norm)
        monkeypatch.setattr(ops, "block_norm_bwd", _norm_bwd)
    return request.param


@pytest.mark.parametrize("shape", [(8,), (5, 8), (2, 3, 8), (0, 8), (2, 0, 8)])
@pytest.mark.parametrize("ydtype", [torch.float32, torch.bfloat16])
def test_leaves_have_gradients_of_their_own(device, shape, ydtype):
    """The residual and y have the same gradient, in arrays of their own: what is added to one later
    does not show in the other."""
    torch.manual_seed(len(shape))
    norm = BlockNorm(8, device=device)
    r = torch.randn(shape, device=device, requires_grad=True)
    y = torch.randn(shape, device=device).to(ydtype).requires_grad_()
    gx, gs = torch.randn(shape, device=device).bfloat16(), torch.randn(shape, device=device)
    x, s = norm(r, y)
    assert x.shape == s.shape == shape and x.dtype == torch.bfloat16
    torch.autograd.backward((x, s), (gx, gs))
    assert r.grad.shape == y.grad.shape == shape and y.grad.dtype == ydtype
    assert torch.equal(r.grad.to(ydtype), y.grad)
    if r.numel():
        assert r.grad.data_ptr() != y.grad.data_ptr()
    once, dr = y.grad.clone(), r.grad.clone()
    x, s = norm(r, y.detach())
    torch.autograd.backward((x, s), (gx, gs))
    assert torch.equal(y.grad, once) and torch.equal(r.grad, 2 * dr)
    x, s = norm(r, y)  # both again: twice, thrice
    torch.autograd.backward((x, s), (gx, gs))
    assert torch.equal(y.grad, 2 * once) and torch.allclose(r.grad, 3 * dr, rtol=1e-6)


def test_sum_changed_in_place_is_found(device):
    """What the backward pass reads may not be written over."""
    norm = BlockNorm(8, device=device)
    r, y = (torch.randn(2, 3, 8, device=device, requires_grad=True) for _ in range(2))
    x, s = norm(r, y)
    with torch.no_grad():
        s.add_(1.0)
    with pytest.raises(RuntimeError, match="inplace"):
        x.float().sum().backward()


def test_strided_arrays_and_one_row_each(device):
    norm = BlockNorm(8, device=device)
    base = torch.randn(8, 5, device=device)
    r, y = base.t().requires_grad_(), torch.randn(5, 16, device=device)[:, ::2]
    x, s = norm(r, y)
    x2, s2 = norm(r.detach().contiguous(), y.contiguous())
    assert torch.equal(x, x2) and torch.equal(s, s2)
    one = norm(r.detach()[0], y[0])  # no leading dimension
    assert torch.equal(one[0], x[0]) and torch.equal(one[1], s[0])
    x, s = BlockNormFn.apply(r, y, norm.weight, norm.eps)
    assert torch.equal(x, x2) and torch.equal(s, s2)


@pytest.mark.gpu
def test_function_refuses_another_width():
    w, r = torch.ones(8, device="cuda"), torch.randn(3, 16, device="cuda")
    for y in (None, r):
        with pytest.raises(ValueError):
            BlockNormFn.apply(r, y, w, 1e-5)
    with pytest.raises(ValueError):
        BlockNormFn.apply(r, r[:, :8], torch.ones(16, device="cuda"), 1e-5)
