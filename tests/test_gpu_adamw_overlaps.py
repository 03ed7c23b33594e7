"""AdamW with a parameter that is listed twice, or states that share memory."""
import pytest
import torch

from paper_2412_06355_gb300 import AdamW, binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def test_tensors_that_share_memory_are_refused():
    cfg, z = binding.make_adamw_config(), lambda n=300: torch.zeros(n, device="cuda")
    p, m, v = z(), z(), z()
    with pytest.raises(ValueError, match="param of tensor 1 lies in the memory of param of tensor 0"):
        binding.adamw_plan(cfg, [p, p], [m, z()], [v, z()])
    with pytest.raises(ValueError, match="v of tensor 0"):
        binding.adamw_plan(cfg, [p], [m], [m])
    flat = z(600)
    with pytest.raises(ValueError, match="memory"):
        binding.adamw_plan(cfg, [flat[:300], flat[299:599]], [m, z()], [v, z()])
    binding.adamw_plan(cfg, [flat[:300], flat[300:], z(0), z(0)], [m, z(), z(0), z(0)], [v, z(), z(0), z(0)])


def test_a_parameter_that_is_listed_twice_is_refused_by_the_optimizer():
    p = torch.nn.Parameter(torch.zeros(10, device="cuda"))
    view = torch.nn.Parameter(p.detach()[2:])
    opt = AdamW([p, view])
    p.grad, view.grad = torch.ones(10, device="cuda"), torch.ones(8, device="cuda")
    with pytest.raises(ValueError, match="memory"):
        opt.step()
    assert not p.any() and int(opt._step) == 0
