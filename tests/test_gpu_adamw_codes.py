"""AdamW's 8-bit states to the bit: scales, and codes as the formulas draw them. The formulas are written out here in
elementary float32 operations, each rounded once; nothing is shared with the library."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2412_06355_gb300 import binding
from paper_2412_06355_gb300 import build as lib_build

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))
F32, E4M3 = torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("probe") / "adamw_probe.so")
    subprocess.run([lib_build.nvcc(), *lib_build.ARCH, *lib_build.NVCC_FLAGS, "-shared", "-o", so,
                    os.path.join(HERE, "adamw_probe.cu")], check=True)
    lib = ctypes.CDLL(so)
    lib.run_quotients.argtypes = lib.run_roots.argtypes = [ctypes.c_uint32, ctypes.c_uint32, ctypes.c_void_p]
    return lib


def bits(exponent):
    return (exponent + 127) << 23


@pytest.mark.parametrize("exponent", [-110, -109, -30, 0, 1, 100, 126, 127])
def test_quotients_with_448_are_the_divisions(probe, exponent):
    """All mantissas, from the smallest top a block is stored with to float32's largest."""
    wrong = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert probe.run_quotients(bits(exponent), 1 << 23, wrong.data_ptr()) == 0
    assert wrong.tolist() == [0, 0]


@pytest.mark.parametrize("exponent", [-102, -30, 0, 1, 126, 127])
def test_roots_are_the_square_roots(probe, exponent):
    """All mantissas of numbers whose root's correction is no denormal number; even and odd exponents."""
    wrong = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert probe.run_roots(bits(exponent), 1 << 23, wrong.data_ptr()) == 0
    assert wrong.tolist() == [0, 0]


@pytest.mark.parametrize("exponent", [-126, -125, -104, -103])
def test_roots_of_small_numbers(probe, exponent):
    wrong = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert probe.run_roots(bits(exponent), 1 << 23, wrong.data_ptr()) == 0
    assert wrong[1] == 0


def test_tiny_gradients_have_roots():
    """Squares that are denormal numbers: v = g^2 rounded to float32, then its root. With a first step of betas 0 and no
    eps the parameter moves by g / root, which the square's own rounding (half of 2^-149) takes from 1 by less than
    2^-150 / g^2; a root without the numbers below 2^-126 was off by half and more."""
    n = 1 << 16
    g = gradients(n, 4).sign() * torch.exp2(-65.0 - 4.0 * torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)))
    s = Eight(n).run(g, lr=1.0, betas=(0.0, 0.0), eps=0.0)
    # the root of denormal numbers is within 2^-19 of theirs where v has 8 bits and more (g above 2^-71); one of few
    # bits is corrected by whole steps of 2^-149 at most: off by 2^-150 / v in half
    off = (-s.p.double() * g.sign() - 1.0).abs()
    assert bool((off <= 2.0 ** -19 + 2.0 ** -149 / g.double().square()).all())
    top = g.double().abs().view(-1, 256).amax(1)
    assert bool(((s.scales[:, 1].double() * 448 - top).abs() <= top * (2.0 ** -18 + 2.0 ** -149 / top.square())).all())


class Eight:
    """One tensor with 8-bit states, from zeros or from what is given."""

    def __init__(self, n, seed=0, param=None, first=0):
        self.n, self.seed, self.first = n, seed, first
        z = lambda dt, *s: torch.zeros(s, dtype=dt, device="cuda")
        self.p = z(F32, n) if param is None else param.clone()
        self.m, self.v, self.scales = z(E4M3, n), z(E4M3, n), z(F32, (n + 255) // 256, 2)
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def run(self, g, **kw):
        """One step; `first` empty tensors stand before this one in the list."""
        cfg = binding.make_adamw_config(state="e4m3", seed=self.seed, **kw)
        e = [torch.zeros(0, dtype=dt, device="cuda") for dt in (F32, E4M3)]
        k = self.first
        plan = binding.adamw_plan(cfg, [e[0]] * k + [self.p], [e[1]] * k + [self.m], [e[1]] * k + [self.v],
                                  [torch.zeros(0, 2, device="cuda")] * k + [self.scales])
        binding.adamw_step(cfg, plan, [e[0]] * k + [g], self.step)
        return self


def gradients(n, seed, std=0.01):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(n, generator=g, device="cuda") * std


def test_scales_are_the_largest_divided_by_448():
    """With betas of 0 the states are g and |g| themselves: m = g, v = g^2."""
    n = 1 << 22
    g = gradients(n, 3)
    s = Eight(n).run(g, betas=(0.0, 0.0))
    top_m = g.cpu().view(-1, 256).abs().amax(1)
    top_v = g.cpu().square().sqrt().view(-1, 256).amax(1)
    assert torch.equal(s.scales[:, 0].cpu(), top_m / 448.0)
    assert torch.equal(s.scales[:, 1].cpu(), top_v / 448.0)


@pytest.mark.parametrize("eps", [0.02, 1e-8])
def test_parameters_take_the_quotient_that_a_division_gives(eps):
    """With betas of 0, parameters of zero and no decay a step is -lr times g / (sqrt(g^2) + eps), and each operation's
    rounding is known: the product with lr in the step's last operation, onto zero."""
    n, lr = 1 << 22, 0.125                                  # a power of two: the product is exact
    g = gradients(n, 6)
    s = Eight(n).run(g, lr=lr, betas=(0.0, 0.0), eps=eps)
    c = g.cpu()
    want = -lr * (c / (c.square().sqrt() + torch.tensor(eps)))
    same = s.p.cpu() == want
    # the correction's own last bit is decided by less than 2^-45 of the quotient: fewer than one in a million
    assert int((~same).sum()) <= n // 1000000
