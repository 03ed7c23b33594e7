"""NormFunction where x and its residual are the same rows in other shapes."""
import pytest
import torch

from paper_2412_06355_gb300 import NormFunction, binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


@pytest.mark.parametrize("one,other", [((2, 5, 48), (10, 48)), ((10, 48), (2, 5, 48)), ((1, 10, 48), (10, 1, 48)), ((10, 48), (10, 48))])
def test_a_residual_of_another_shape(one, other):
    """The forward takes rows of D, whatever the axes before; the residual's gradient has the residual's."""
    x, residual = torch.randn(one, device="cuda", requires_grad=True), torch.randn(other, device="cuda", requires_grad=True)
    w = torch.randn(48, device="cuda", requires_grad=True)
    y, total = NormFunction.apply(x, residual, w)
    assert y.shape == total.shape == x.shape
    gy, gt = torch.randn_like(y), torch.randn_like(total)
    got = torch.autograd.grad((y * gy).sum() + (total * gt).sum(), (x, residual, w))
    flat = [t.detach().reshape(10, 48).requires_grad_() for t in (x, residual)] + [w]
    y, total = NormFunction.apply(*flat)
    want = torch.autograd.grad((y * gy.view(10, 48)).sum() + (total * gt.view(10, 48)).sum(), flat)
    assert got[0].shape == x.shape and got[1].shape == residual.shape
    assert all(torch.equal(a.view_as(b), b) for a, b in zip(got, want))
