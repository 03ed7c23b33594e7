"""What the autograd function of the gated delta rule keeps, and for how long."""
import pytest
import torch

from paper_2412_06355_gb300 import DeltaFunction, binding

pytestmark = pytest.mark.gpu
B, T, H, DK, DV = 2, 300, 2, 64, 48


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def leaves(seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    unit = lambda t: t / t.square().sum(-1, keepdim=True).sqrt()
    return [t.requires_grad_() for t in (unit(n(B, T, H, DK)), unit(n(B, T, H, DK)), n(B, T, H, DV), -n(B, T, H).abs(),
                                         torch.sigmoid(n(B, T, H)), n(B, H, DK, DV))]


def apply(x):
    return DeltaFunction.apply(*x, None, DK ** -0.5, "batch")


@pytest.mark.parametrize("with_o,with_last", [(True, True), (True, False), (False, True)])
def test_inputs_may_be_overwritten_after_the_forward(with_o, with_last):
    """The backward reads no input, so a buffer that is used again for the next layer is no error."""
    at = leaves()

    def loss(o, last):
        return (o.square().sum() if with_o else 0) + (last.square().sum() if with_last else 0)

    want = torch.autograd.grad(loss(*apply(at)), at)
    x = [t * 1.0 for t in at]                               # a layer's intermediate results
    value = loss(*apply(x))
    with torch.no_grad():
        for t in x:
            t.fill_(float("nan"))
    got = torch.autograd.grad(value, at)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_only_the_workspace_is_kept_and_goes_with_the_backward():
    at = leaves()
    sizes = binding.dendsn_delta_workspace_size(binding.make_delta_config(T, B, H, H, DK, DV, "f32", "batch"))
    apply(at)[0].sum().backward()                           # gradients of the leaves are there from now on
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    x = [t * 1.0 for t in at]
    o, last = apply(x)
    del x                                                   # (the products with 1.0 keep their factors, which are the leaves)
    outputs = sum((t.numel() * 4 + 511) // 512 * 512 for t in (o, last))
    assert torch.cuda.memory_allocated() - before <= outputs + (sizes[0] + 511) // 512 * 512
    loss = o.sum()
    loss.backward()
    assert loss.grad_fn is not None                         # the graph is still held
    assert torch.cuda.memory_allocated() - before <= outputs + 512
    with pytest.raises(RuntimeError, match="second time"):
        loss.backward()


def test_backward_twice_where_the_graph_is_retained():
    at = leaves()
    o, last = apply(at)
    first = torch.autograd.grad(o.sum() + last.sum(), at, retain_graph=True)
    again = torch.autograd.grad(o.sum() + last.sum(), at)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
