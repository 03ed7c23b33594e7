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


# ------------------------------------------------------------------ the draw, as the formulas have it
def mixed(h):
    """32-bit integers held in 64 bits, scrambled."""
    h = ((h ^ (h >> 16)) * 0x6A09E667) & 0xFFFFFFFF
    h = ((h ^ (h >> 15)) * 0xADF85459) & 0xFFFFFFFF
    return h ^ (h >> 16)


def random_numbers(seed, step, index, n):
    """Two numbers in (0, 1) for each element, of 16 bits each: from seed, step, the tensor's and the element's place."""
    t = lambda v: torch.tensor(v, dtype=torch.int64, device="cuda")
    start = mixed((mixed(t((step * 0x9E3779B1 + seed) & 0xFFFFFFFF)) + index) & 0xFFFFFFFF)
    h = mixed((torch.arange(n, device="cuda") * 0x9E3779B1 + start) & 0xFFFFFFFF)
    return ((h & 0xFFFF).float() + 0.5) / 65536.0, ((h >> 16).float() + 0.5) / 65536.0


def drawn(x, u, squared):
    """(values of the codes, scales): the largest of 256 becomes 448, the upper neighbour where u is below the share that
    makes the expectation of the value, or of its square, right."""
    blocks = x.view(-1, 256)
    top = blocks.abs().amax(1, keepdim=True)
    value = (blocks * (torch.full_like(top, 448.0) / top)).abs().view(-1)
    step = torch.exp2((torch.frexp(value.clamp_min(2.0 ** -6)).exponent - 4).float())
    low = torch.floor(value / step) * step
    share = (value - low) * (value + low) / (step * (2.0 * low + step)) if squared else (value - low) / step
    return torch.copysign(torch.where(u < share, low + step, low).clamp_max(448.0), x), (top / torch.full_like(top, 448.0))[:, 0]


def decoded(codes, scale):
    return codes.float() * scale.repeat_interleave(256)


@pytest.mark.parametrize("seed,first", [(0, 0), (77, 3), (2 ** 32 - 1, 1)])
def test_codes_are_drawn_as_the_formulas_say(seed, first):
    """Five steps, each from the library's own states before. The library may join a product with the sum behind it, so
    its m and v are within two last bits (2^-22) of those rounded one by one here. That moves a scale by as much, and a
    value by as much of itself, which is 16 steps of a code at most: 2^-18 of a step, for the value and for the block's
    largest each, so that a draw may fall on the other side in 2^-17 of the elements at most (8 in a million)."""
    n = 1 << 20
    s, rest = Eight(n, seed, first=first), [torch.tensor(v, device="cuda") for v in (1.0 - 0.9, 1.0 - 0.999)]
    for step in range(1, 6):
        g = gradients(n, 20 + step)
        m, v = decoded(s.m, s.scales[:, 0]), decoded(s.v, s.scales[:, 1]).square()
        s.run(g)
        um, uv = random_numbers(seed, step, first, n)
        for got, scale, x, u, squared in ((s.m, s.scales[:, 0], m + rest[0] * (g - m), um, False),
                                          (s.v, s.scales[:, 1], (v + rest[1] * (g.square() - v)).sqrt(), uv, True)):
            want, want_scale = drawn(x, u, squared)
            assert bool(((scale - want_scale).abs() <= want_scale * 2.0 ** -22).all())
            assert int((got.float() != want).sum()) <= n * 2.0 ** -17, (step, squared)


def test_codes_depend_on_seed_step_and_place():
    """Equal states and gradients: a third of the codes differ with the seed, the step, the tensor's place in the list,
    and from one half of a tensor to the other (a share s gives 2 s (1 - s); its mean over even shares is 1/3)."""
    n = 1 << 16
    g = gradients(n // 2, 9).repeat(2)
    base = Eight(n).run(g)
    late = Eight(n)
    late.step.fill_(5)                                      # scales and shares are the same: the states start as zeros
    others = [Eight(n, seed=1).run(g), Eight(n, first=1).run(g), late.run(g)]
    half = Eight(n)
    half.m, half.v = (torch.cat([t[n // 2:], t[:n // 2]]) for t in (base.m, base.v))
    for o in (*others, half):
        for a, b in ((base.m, o.m), (base.v, o.v)):
            assert 0.25 < float((a.float() != b.float()).double().mean()) < 0.42
    again = Eight(n).run(g)
    assert torch.equal(base.m.float(), again.m.float()) and torch.equal(base.v.float(), again.v.float())


def test_expectations_hold_over_hundreds_of_steps():
    """m and v are linear in what they were, so codes drawn with the right expectations keep them: the mean over many
    elements of state / float32 state is 1 within five standard errors, after 300 steps as after one."""
    n = 1 << 19
    scale = torch.exp2(-3.0 * torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)))
    eight = Eight(n, seed=5)
    cfg = binding.make_adamw_config(state="f32")
    z = [torch.zeros(n, device="cuda") for _ in range(3)]
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    plan = binding.adamw_plan(cfg, [z[0]], [z[1]], [z[2]])
    for i in range(300):
        g = gradients(n, 100 + i) * scale + scale * 0.005
        eight.run(g)
        binding.adamw_step(cfg, plan, [g], step)
    v = decoded(eight.v, eight.scales[:, 1]).double().square() / z[2].double()
    m = (decoded(eight.m, eight.scales[:, 0]).double() - z[1].double()) / z[2].double().sqrt()
    for name, x, mean in (("v", v, 1.0), ("m", m, 0.0)):
        error = float(x.std()) / n ** 0.5
        # 16 random bits at their middle: no bias of their own; 300 steps of float32 roundings, 2^-24 each
        assert abs(float(x.mean()) - mean) < 5 * error + 300 * 2.0 ** -24, (name, float(x.mean()), error)


def test_a_v_of_zero_beside_an_m_that_is_not():
    """A v whose code was drawn as zero counts in the quotient as the smallest code, 2^-9 of the scale; above it as it is."""
    n, lr, scales = 1024, 0.5, (3e-4, 2e-3)
    s = Eight(n)
    s.m.copy_(torch.linspace(-448, 448, n, device="cuda").to(E4M3))
    codes = torch.tensor([0.0, 2.0 ** -9, 2.0 ** -8, 448.0], device="cuda").repeat(n // 4)
    s.v.copy_(codes.to(E4M3))
    s.scales[:] = torch.tensor(scales, device="cuda")
    s.step.fill_(50)
    m = decoded(s.m, s.scales[:, 0]).double() * 0.9
    s.run(torch.zeros(n, device="cuda"), lr=lr, eps=1e-10)
    root = torch.maximum((0.999 * codes.double().square()).sqrt(), torch.tensor(2.0 ** -9, device="cuda").double()) * s_of(scales[1])
    want = -lr / (1 - 0.9 ** 51) * m / (root / (1 - 0.999 ** 51) ** 0.5 + 1e-10)
    # m and the quotient are some ten float32 operations; m cancels nowhere
    assert bool(((s.p.double() - want).abs() <= 16 * 2.0 ** -24 * want.abs()).all())
    assert not s.v.float()[codes == 0].any()                # the state itself stays zero


def s_of(v):
    return float(torch.tensor(v, dtype=F32))


@pytest.mark.parametrize("span", [4, 16, 20, 24])
def test_steps_stay_steps_where_a_blocks_gradients_differ_widely(span):
    """Gradients from 2^-span of their block's largest on. Float32's m is at most 7.3 sqrt(v) whatever the gradients do
    (0.1 / sqrt(0.001) / sqrt(1 - 0.81 / 0.999)); a code of m is within an eighth of its value or the smallest, a root
    counts as no less than the smallest code of v: four times that leaves room for both."""
    n = 1 << 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    scale = torch.exp2(-span * torch.rand(n, device="cuda", generator=gen))
    s, largest = Eight(n), 0.0
    for i in range(300):
        before = s.p.clone()
        s.run(torch.randn(n, device="cuda", generator=gen) * scale, lr=1.0)
        if i >= 20:
            largest = max(largest, float((s.p - before).abs().max()))
    assert largest < 4 * 7.3


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 1e25])
def test_a_gradient_whose_square_is_no_number_gives_no_number(bad):
    """A v that leaves float32 is no v of zero: the parameter does not move by a number then."""
    s = Eight(512).run(gradients(512, 1)).run(gradients(512, 2))
    g, before = gradients(512, 3), s.p.clone()
    g[7] = bad
    s.run(g)
    assert torch.isnan(s.p[7]) and torch.isfinite(s.p[256:]).all() and float((s.p - before)[8:].abs().max()) < 0.01
