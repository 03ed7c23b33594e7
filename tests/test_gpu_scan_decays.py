"""Logistic decays of the gated scan, gate by gate: a and 1 - a against float64."""
import pytest
import torch

from paper_2412_06355_gb300 import binding

pytestmark = pytest.mark.gpu


def gates(dtype):
    if dtype == "bf16":
        g = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
        return g[g.float().abs() <= 79]                    # NaN drops out too
    g = torch.Generator().manual_seed(1)
    return torch.cat([torch.linspace(-79, 79, 200001), torch.randn(100000, generator=g) * 3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 70])
def test_decays_and_their_complements(dtype, T):
    """Exponential 2^-22, reciprocal 2^-23 and three roundings of 2^-24 stay within 2^-21, also
    where the gate is far from 0."""
    if not torch.cuda.is_available():
        pytest.fail("needs a CUDA device")
    g = gates(dtype).cuda()
    N = g.numel()
    gate = torch.full((T, 1, N), 100.0, dtype=g.dtype, device="cuda")     # a = 1 before
    gate[-1, 0] = g
    x, one = torch.zeros_like(gate), torch.ones(1, N, device="cuda")
    cfg = binding.make_scan_config(T, 1, N, dtype, "logit", "plain")
    a = binding.scan_forward(cfg, x, gate, None, one, want_last=True)[1]
    x[-1] = 1
    cfg = binding.make_scan_config(T, 1, N, dtype, "logit", "complement")
    na = binding.scan_forward(cfg, x, gate, None, None, want_last=True)[1]
    for got, want in ((a, torch.sigmoid(g.double())), (na, torch.sigmoid(-g.double()))):
        assert float(((got[0].double() - want) / want).abs().max()) <= 2.0 ** -21


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_beyond_the_exponential(dtype):
    if not torch.cuda.is_available():
        pytest.fail("needs a CUDA device")
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.tensor([float("inf"), 3e38, 150.0, -float("inf"), -3e38, -150.0, float("nan")], device="cuda").to(dt)
    N = g.numel()
    one = torch.ones(1, N, device="cuda")
    cfg = binding.make_scan_config(1, 1, N, dtype, "logit", "plain")
    a = binding.scan_forward(cfg, torch.zeros(1, 1, N, dtype=dt, device="cuda"), g.view(1, 1, N), None, one, want_last=True)[1][0]
    cfg = binding.make_scan_config(1, 1, N, dtype, "logit", "complement")
    na = binding.scan_forward(cfg, torch.ones(1, 1, N, dtype=dt, device="cuda"), g.view(1, 1, N), None, None, want_last=True)[1][0]
    assert bool(((a[:3] - 1).abs() < 1e-30).all() and (a[3:6] < 1e-30).all() and (a[3:6] >= 0).all())
    assert bool((na[:3] < 1e-30).all() and (na[:3] >= 0).all() and (na[3:6] == 1).all())
    assert bool(torch.isnan(a[6]) and torch.isnan(na[6]))
