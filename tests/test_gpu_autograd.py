"""The autograd functions under create_graph: their gradients have no graph of their own, and a
second derivative through them is refused instead of being silently left out."""
import pytest
import torch

from paper_2412_06355_gb300 import (DendSNFunction, EmbedFunction, ScanFunction, XentFunction,
                                    binding, make_config)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def leaf(*shape):
    return torch.rand(shape, device="cuda").requires_grad_()


def embed():
    table = leaf(10, 8)
    return EmbedFunction.apply(table, torch.arange(4, device="cuda")), table


def scan():
    x, gate = leaf(5, 2, 8), leaf(5, 2, 8)
    return ScanFunction.apply(x, gate)[0], x


def xent():
    hidden, weight = leaf(6, 8), leaf(10, 8)
    return XentFunction.apply(hidden, weight, torch.arange(6, device="cuda")), hidden


def layer():
    cfg = make_config(4, 2, 64, 4, G=1, C=4, inner=16)
    x = leaf(4, 2, 64, 4)
    par = [torch.rand((4, 4), device="cuda") for _ in range(4)]
    return DendSNFunction.apply(x, *par, None, cfg), x


@pytest.mark.parametrize("fn", [embed, scan, xent, layer], ids=lambda f: f.__name__)
def test_a_second_derivative_is_refused(fn):
    out, p = fn()
    w = leaf(*out.shape)
    first, = torch.autograd.grad((out * w).sum(), p, create_graph=True)
    assert first.shape == p.shape and bool(torch.isfinite(first).all())
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (first.sum() + w.square().sum()).backward()
