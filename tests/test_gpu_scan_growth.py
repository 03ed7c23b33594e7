"""Gated scans whose decays are above 1: products of decays that leave float32 within a block's
steps although no state does, against the recurrence in float64."""
import pytest
import torch

import seq_reference as ref
from paper_2412_06355_gb300 import binding

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def decays(T, factor, run, shape, g):
    """`run` steps that multiply by 2^factor, `run` that divide by it, and so on; some channels the
    other way round, some with decays below 1 throughout."""
    sign = torch.where(torch.arange(T) // run % 2 == 0, 1.0, -1.0).cuda()
    e = (sign * factor).view(T, 1, 1).expand(shape)
    kind = torch.randint(0, 4, shape[1:], generator=g, device="cuda")
    e = torch.where(kind == 1, -e, e)
    a = torch.exp2(e.float()) * torch.where(torch.rand(shape, generator=g, device="cuda") < 0.1, -1.0, 1.0)
    return torch.where(kind == 2, 0.5, a)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,N", [(7, 2, 40), (40, 3, 33), (300, 2, 40), (300, 16, 700), (1500, 1, 64),
                                   (130, 20, 1001)])
@pytest.mark.parametrize("factor,run", [(4, 48), (50, 2), (100, 1), (90, 2)])
@pytest.mark.parametrize("starts", [0.0, 0.01])
def test_growth_that_falls_back(dtype, T, B, N, factor, run, starts):
    """States from 2^-100 up to at most 2^100, whose products of decays reach 2^+-200 in a block's
    steps. h grows where the state's gradient falls, so gradients stay in float32 too."""
    g = torch.Generator(device="cuda")
    g.manual_seed(T + factor)
    shape = (T, B, N)
    gate = decays(T, factor, run, shape, g).to(DT[dtype])
    tiny = lambda s, e: torch.randn(s, generator=g, device="cuda") * 2.0 ** e
    x, gh = tiny(shape, -112).to(DT[dtype]), tiny(shape, -112).to(DT[dtype])
    h0, glast = tiny((B, N), -104), tiny((B, N), -110)
    st = None
    if starts:
        st = (torch.rand((T, B), generator=g, device="cuda") < starts).to(torch.uint8)
    cfg = binding.make_scan_config(T, B, N, dtype)
    saved = binding.scan_workspace(cfg)
    h, last = binding.scan_forward(cfg, x, gate, st, h0, saved, want_last=True)
    got = dict(h=h, last=last)
    got.update(binding.scan_backward(cfg, x, gate, gh, st, h0, glast, saved))
    want = ref.scan(x, gate, st, h0, gh, glast, "decay", "plain", "time")
    assert float(want["h"][0].abs().max()) < 2.0 ** 120
    for k in got:
        if k != "ggate":                   # a product of two such values
            assert float(want[k][0].abs().max()) < 2.0 ** 126
            ref.check(k, got[k], want[k])
        else:
            v, b = want[k]
            ref.check(k, torch.where(v.abs() < 2.0 ** 127, got[k].double(), v), (v, b))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,N", [(40, 2, 40), (1500, 1, 64), (300, 16, 700)])
def test_a_state_of_zero_stays_zero(dtype, T, B, N):
    """Whatever the decays multiply to; and a channel beside it that does grow is infinite."""
    x = torch.zeros(T, B, N, dtype=DT[dtype], device="cuda")
    gate = torch.full_like(x, 1e30)
    h0 = torch.zeros(B, N, device="cuda")
    h0[:, 1] = 1.0
    cfg = binding.make_scan_config(T, B, N, dtype)
    h, last = binding.scan_forward(cfg, x, gate, None, h0, want_last=True)
    zero = torch.arange(N, device="cuda") != 1
    assert torch.count_nonzero(h[..., zero]) == 0 and torch.count_nonzero(last[:, zero]) == 0
    assert bool(torch.isinf(last[:, 1]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,N", [(150, 3, 33), (150, 5, 1001), (1500, 1, 64), (300, 16, 700)])
def test_a_channel_does_not_depend_on_the_one_beside_it(dtype, T, B, N):
    """Growing channels, infinities and NaN beside channels whose decays are below 1."""
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    shape = (T, B, N)
    x, gh = (torch.randn(shape, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    gate = torch.rand(shape, generator=g, device="cuda").to(DT[dtype])
    st = (torch.rand((T, B), generator=g, device="cuda") < 0.02).to(torch.uint8)
    cfg = binding.make_scan_config(T, B, N, dtype, mix="complement")
    saved = binding.scan_workspace(cfg)
    beside = torch.arange(N, device="cuda") % 2 == 1

    def run(gate):
        h, last = binding.scan_forward(cfg, x, gate, st, None, saved, want_last=True)
        out = binding.scan_backward(cfg, x, gate, gh, st, None, None, saved)
        return [h, last, out["gx"], out["ggate"]]

    want = run(gate)
    for value in (1e20, -3.0, float("inf"), float("nan")):
        other = gate.clone()
        other[..., beside] = value
        for a, b in zip(run(other), want):
            assert torch.equal(a[..., ~beside], b[..., ~beside])
