"""AdamW's step in a CUDA graph beside eager steps of the same optimizer."""
import gc
import weakref

import pytest
import torch

from paper_2412_06355_gb300 import AdamW, binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def setup(state):
    torch.manual_seed(3)
    ps = [torch.nn.Parameter(torch.randn(k, device="cuda")) for k in (700, 33)]
    for i, p in enumerate(ps):
        p.grad = torch.randn(p.shape, device="cuda")
    return ps, AdamW(ps, lr=1e-2, weight_decay=0.1, state=state, max_norm=0.5, seed=2)


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_a_graph_outlives_a_change_of_weight_decay(state):
    """An eager step with another weight decay makes another table; the graph's stays where it is."""
    ps, opt = setup(state)
    twins, twin = setup(state)
    opt.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    held = weakref.ref(opt._plan)
    opt.param_groups[0]["weight_decay"] = 0.3
    opt.step()
    gc.collect()
    assert held() is not None and held() is not opt._plan
    for _ in range(2):
        graph.replay()
    torch.full((4096,), 255, dtype=torch.uint8, device="cuda")
    graph.replay()
    for decay in (0.1, 0.3, 0.1, 0.1, 0.1):
        twin.param_groups[0]["weight_decay"] = decay
        twin.step()
    assert all(torch.equal(a, b) for a, b in zip(ps, twins))
    assert int(opt._step) == 5


def test_tables_of_eager_steps_go():
    ps, opt = setup("f32")
    opt.step()
    held = weakref.ref(opt._plan)
    opt.param_groups[0]["weight_decay"] = 0.3
    opt.step()
    gc.collect()
    assert held() is None and not opt._captured
