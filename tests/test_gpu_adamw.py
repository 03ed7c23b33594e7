"""The AdamW step over many tensors on the GPU against float64 (block_reference.py). An element's update
is some ten float32 operations; the bounds count 16 U32 of the magnitudes that enter a sum."""
import math
import random

import pytest
import torch

import block_reference as ref
from block_reference import HALF_STEP, U32, within
from paper_2412_06355_gb300 import AdamW, binding

pytestmark = pytest.mark.gpu
BETAS, EPS, LR = (0.9, 0.999), 1e-8, 1e-2
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def zeros(n, dtype=F32, shift=0):
    return torch.zeros(n + shift, dtype=dtype, device="cuda")[shift:]


class Set:
    """Tensors of an optimizer with random states after `step` steps."""

    def __init__(self, sizes, param=F32, state="f32", copies=False, shift=0, seed=0, decay=0.01):
        g = gen(seed)
        n = lambda k, std, dt=F32: zeros(k, dt, shift).copy_((torch.randn(k, generator=g, device="cuda") * std).to(dt))
        self.sizes, self.state = sizes, state
        self.p = [n(k, 0.1, param) for k in sizes]
        self.copies = [zeros(k, BF16, shift) for k in sizes] if copies else None
        if state == "f32":
            self.m = [n(k, 0.01) for k in sizes]
            self.v = [n(k, 0.02).square_() for k in sizes]
            for t, k in zip(self.v, sizes):
                assert t.numel() == k
            self.scales = None
        else:
            self.m = [zeros(k, E4M3, shift).copy_(torch.randn(k, generator=g, device="cuda").mul(100).to(E4M3)) for k in sizes]
            self.v = [zeros(k, E4M3, shift).copy_(torch.rand(k, generator=g, device="cuda").mul(400).to(E4M3)) for k in sizes]
            self.scales = [torch.rand((k + 255) // 256, 2, generator=g, device="cuda") * 1e-4 for k in sizes]
        self.step = torch.full((1,), 9, dtype=torch.int64, device="cuda")
        self.decay = decay

    def plan(self, cfg):
        return binding.adamw_plan(cfg, self.p, self.m, self.v, self.scales, self.copies, self.decay)

    def copy(self):
        s = object.__new__(Set)
        s.__dict__.update(self.__dict__)
        for name in ("p", "m", "v", "scales", "copies"):
            ts = getattr(self, name)
            setattr(s, name, None if ts is None else [t.clone() for t in ts])
        s.step = self.step.clone()
        return s

    def bits(self):
        out = []
        for name in ("p", "m", "v", "scales", "copies"):
            out += [t.clone().view(torch.uint8) for t in (getattr(self, name) or [])]
        return out + [self.step.clone()]


def grads_of(sizes, dtype, shift=0, seed=5, std=0.03):
    g = gen(seed)
    kinds = [dtype] * len(sizes) if dtype != "mixed" else [(F32, BF16)[i % 2] for i in range(len(sizes))]
    return [zeros(k, d, shift).copy_((torch.randn(k, generator=g, device="cuda") * std).to(d)) for k, d in zip(sizes, kinds)]


SIZES = [1, 7, 8, 255, 256, 257, 4096, 4097, 5000, 12288, 100003]


@pytest.mark.parametrize("param", [F32, BF16])
@pytest.mark.parametrize("grad", [F32, BF16, "mixed"])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("clip", [0.0, 0.5])
def test_float32_states(param, grad, shift, clip):
    s = Set(SIZES, param, copies=param == F32, shift=shift)
    g = grads_of(SIZES, grad, shift)
    before = s.copy()
    cfg = binding.make_adamw_config(LR, BETAS, EPS, max_norm=clip)
    norm = binding.adamw_step(cfg, s.plan(cfg), g, s.step)
    assert int(s.step) == 10
    factor = 1.0
    if clip:
        want = math.sqrt(sum(float(t.double().square().sum()) for t in g))
        # sums of 16 squares in float32, the rest in float64, one rounding
        assert abs(float(norm) - want) <= want * 20 * U32
        factor = min(1.0, clip / want)
    else:
        assert norm is None
    for i in range(len(SIZES)):
        p, m, v = ref.adamw(before.p[i], g[i], before.m[i], before.v[i], 10, LR, BETAS, EPS, 0.01, factor)
        gm = g[i].double().abs() * factor
        within("m", s.m[i], m, 16 * U32 * (before.m[i].double().abs() + gm) + (20 * U32 * gm if clip else 0))
        within("v", s.v[i], v, 16 * U32 * (before.v[i].double() + gm * gm) + (40 * U32 * gm * gm if clip else 0))
        # m may cancel: its bound goes into the update
        unit = (16 * U32 * (before.m[i].double().abs() + 3 * gm) / (1 - BETAS[0] ** 10)) / (torch.sqrt(v / (1 - BETAS[1] ** 10)) + EPS)
        move = (p - before.p[i].double()).abs()
        bound = LR * unit + 64 * U32 * move + 4 * U32 * before.p[i].double().abs()
        within("p", s.p[i], p, bound + (p.abs() + bound) * HALF_STEP[param])
        if s.copies:
            assert torch.equal(s.copies[i], s.p[i].bfloat16())


@pytest.mark.parametrize("param,grad", [(F32, F32), (BF16, BF16), (F32, "mixed")])
@pytest.mark.parametrize("clip", [0.0, 0.5])
def test_eight_bit_states(param, grad, clip):
    s = Set(SIZES, param, "e4m3")
    g = grads_of(SIZES, grad)
    before = s.copy()
    cfg = binding.make_adamw_config(LR, BETAS, EPS, "e4m3", clip, seed=3)
    norm = binding.adamw_step(cfg, s.plan(cfg), g, s.step)
    factor = min(1.0, clip / float(norm)) if clip else 1.0
    for i, n in enumerate(SIZES):
        m0 = ref.decoded(before.m[i], before.scales[i][:, 0])
        v0 = ref.decoded(before.v[i], before.scales[i][:, 1]).square()
        p, m, v = ref.adamw(before.p[i], g[i], m0, v0, 10, LR, BETAS, EPS, 0.01, factor)
        # the square root and the quotient are approximate: 2^-22 of the update, 2^-20 with what m and v carry
        bound = LR * 2.0 ** -20 * (m0.abs() + g[i].double().abs()) / (torch.sqrt(v) + EPS) * 3 + 8 * U32 * before.p[i].double().abs()
        # some of m's random values are above what a code holds and became NaN: the parameter's element is NaN,
        # and the block's states are from then on
        lost = torch.isnan(m)
        assert torch.equal(torch.isnan(s.p[i]), lost)
        keep = ~lost
        within("p", s.p[i][keep], p[keep], (bound + (p.abs() + bound) * HALF_STEP[param])[keep])
        for codes, scale, want in ((s.m[i], s.scales[i][:, 0], m), (s.v[i], s.scales[i][:, 1], v.sqrt())):
            top = torch.stack([x.abs().max() for x in want.split(256)])
            assert torch.equal(torch.isnan(scale), torch.isnan(top))
            whole = ~torch.isnan(top)
            within("scale", scale[whole], (top / 448)[whole], (top * 2.0 ** -20 / 448)[whole])
            keep = whole.repeat_interleave(256)[:n]
            want, codes = want[keep], codes[keep]
            value = (want / (top / 448).repeat_interleave(256)[:n][keep]).abs()
            got = codes.double().abs()
            within("code", got, value, ref.spacing(value) * (1 + 2.0 ** -12) + value * 2.0 ** -18)
            away = value > 1.0
            assert bool((codes.double().sign()[away] == want.sign()[away]).all())


def test_codes_are_right_on_average():
    """The mean of m's codes, and of the squares of v's, over many elements of equal states."""
    n = 2 ** 20
    for value, square in ((3.3, False), (0.0131, False), (7.77, True), (0.0031, True)):
        p, g = zeros(n), zeros(n)
        m, v = zeros(n, E4M3), zeros(n, E4M3)
        g[::256] = 1.0                                      # the block's largest: code 448 where the others are value
        others = torch.arange(n, device="cuda") % 256 != 0
        g[others] = value / 448
        scales = torch.zeros(n // 256, 2, device="cuda")
        cfg = binding.make_adamw_config(LR, BETAS, EPS, "e4m3", seed=11)
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        binding.adamw_step(cfg, binding.adamw_plan(cfg, [p], [m], [v], [scales]), [g], step)
        codes = (v if square else m).double()[others]
        if square:
            codes, mean = codes.square(), value ** 2
        else:
            mean = value
        spread = float(codes.std()) / math.sqrt(codes.numel())
        assert codes.unique().numel() == 2
        # five standard errors, and 16 random bits' half step
        assert abs(float(codes.mean()) - mean) < 5 * spread + 2.0 ** -16 * mean, (value, square)


@pytest.mark.parametrize("state", ["f32", "e4m3"])
@pytest.mark.parametrize("clip", [0.0, 0.3])
def test_places_and_runs_give_the_same_bits(state, clip):
    """Aligned tensors take other loads than misaligned ones, and more than 500 tensors more launches."""
    sizes = [random.Random(2).choice((8, 256, 264, 4104, 9000)) + 8 * (i % 3) for i in range(40)]
    a, b = Set(sizes, BF16, state, shift=0), Set(sizes, BF16, state, shift=1)
    for x, y in zip((*a.p, *a.m, *a.v), (*b.p, *b.m, *b.v)):
        y.copy_(x)
    again = a.copy()
    cfg = binding.make_adamw_config(LR, BETAS, EPS, state, clip, seed=1)
    for s, shift in ((a, 0), (again, 0), (b, 1)):
        plan = s.plan(cfg)
        for _ in range(3):
            binding.adamw_step(cfg, plan, grads_of(sizes, "mixed", shift), s.step)
    assert all(torch.equal(x, y) for x, y in zip(a.bits(), again.bits()))
    assert all(torch.equal(x, y) for x, y in zip(a.bits(), b.bits()))


def test_very_many_tensors():
    sizes = [3 + i % 5 for i in range(1203)]
    s = Set(sizes)
    before = s.copy()
    g = grads_of(sizes, F32)
    cfg = binding.make_adamw_config(LR, BETAS, EPS, max_norm=1e-3)
    norm = binding.adamw_step(cfg, s.plan(cfg), g, s.step)
    want = math.sqrt(sum(float(t.double().square().sum()) for t in g))
    assert abs(float(norm) - want) < 1e-5 * want and int(s.step) == 10
    for i in (0, 499, 500, 999, 1000, 1202):
        m = ref.adamw(before.p[i], g[i], before.m[i], before.v[i], 10, LR, BETAS, EPS, 0.01, 1e-3 / want)[1]
        within("m", s.m[i], m, 64 * U32 * (before.m[i].double().abs() + g[i].double().abs()))


def test_missing_gradients_and_empty_tensors():
    sizes = [300, 0, 4100, 8]
    s = Set(sizes)
    before = s.copy()
    g = grads_of(sizes, F32)
    cfg = binding.make_adamw_config(LR, BETAS, EPS, max_norm=1.0)
    norm = binding.adamw_step(cfg, s.plan(cfg), [g[0], g[1], None, g[3]], s.step)
    assert torch.equal(s.p[2], before.p[2]) and torch.equal(s.m[2], before.m[2]) and torch.equal(s.v[2], before.v[2])
    assert not torch.equal(s.p[0], before.p[0]) and not torch.equal(s.p[3], before.p[3])
    want = math.sqrt(float(g[0].double().square().sum() + g[3].double().square().sum()))
    assert abs(float(norm) - want) <= want * 20 * U32
    empty = binding.adamw_plan(cfg, [], [], [])
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    assert float(binding.adamw_step(cfg, empty, [], step)) == 0 and int(step) == 1
    with pytest.raises(ValueError, match="grads"):
        binding.adamw_step(cfg, empty, g, step)
    with pytest.raises(ValueError, match="elements"):
        binding.adamw_step(cfg, s.plan(cfg), [g[3], g[1], g[2], g[0]], s.step)
    with pytest.raises(ValueError, match="contiguous"):
        binding.adamw_step(cfg, s.plan(cfg), [torch.zeros(600, device="cuda")[::2], g[1], g[2], g[3]], s.step)
    with pytest.raises(ValueError, match="state"):
        binding.adamw_step(binding.make_adamw_config(state="e4m3"), s.plan(cfg), g, s.step)


def test_strange_gradients():
    n = 1024
    for state in ("f32", "e4m3"):
        s = Set([n], F32, state)
        clean = s.copy()
        g = grads_of([n], F32)[0]
        cfg = binding.make_adamw_config(LR, BETAS, EPS, state)
        binding.adamw_step(cfg, clean.plan(cfg), [g], clean.step)
        bad = g.clone()
        bad[300], bad[600] = float("nan"), float("inf")
        binding.adamw_step(cfg, s.plan(cfg), [bad], s.step)
        touched = torch.zeros(n, dtype=torch.bool, device="cuda")
        if state == "f32":
            touched[[300, 600]] = True
        else:
            touched[256:768] = True
        assert torch.equal(s.p[0][~touched], clean.p[0][~touched])
        assert torch.isnan(s.p[0][300])
        if state == "e4m3":
            assert torch.isnan(s.scales[0][1]).all() and not torch.isfinite(s.scales[0][2]).any()
            assert torch.equal(s.scales[0][[0, 3]], clean.scales[0][[0, 3]])
    # all zeros stay zeros; tiny values do not become infinite
    for state, dt in (("f32", F32), ("e4m3", E4M3)):
        p, m, v = zeros(512), zeros(512, dt), zeros(512, dt)
        sc = [torch.zeros(2, 2, device="cuda")] if state == "e4m3" else None
        cfg = binding.make_adamw_config(LR, BETAS, EPS, state)
        plan, step = binding.adamw_plan(cfg, [p], [m], [v], sc), torch.zeros(1, dtype=torch.int64, device="cuda")
        binding.adamw_step(cfg, plan, [zeros(512)], step)
        assert not p.any() and not m.float().any() and not v.float().any()
        binding.adamw_step(cfg, plan, [zeros(512) + 1e-38], step)
        assert torch.isfinite(p).all() and torch.isfinite(m.float()).all()


def test_a_first_step_moves_by_lr():
    p, m, v, step = zeros(100), zeros(100), zeros(100), torch.zeros(1, dtype=torch.int64, device="cuda")
    cfg = binding.make_adamw_config(LR, BETAS, 0.0)
    g = torch.linspace(-1, 1, 100, device="cuda")
    binding.adamw_step(cfg, binding.adamw_plan(cfg, [p], [m], [v]), [g], step)
    # m / (1 - beta1) and v / (1 - beta2) are g and g^2 up to a few roundings
    within("p", p, -LR * g.double().sign(), torch.full((100,), LR * 32 * U32, dtype=torch.float64, device="cuda"))


def test_a_captured_step_counts_on_and_takes_the_rate_from_the_device():
    sizes = [5000, 33]
    s = Set(sizes, BF16, "e4m3")
    e = s.copy()
    g = grads_of(sizes, BF16)
    lr = torch.full((1,), 1e-2, device="cuda")
    cfg = binding.make_adamw_config(99.0, BETAS, EPS, "e4m3", 0.5, seed=4)
    plan, norm = s.plan(cfg), torch.empty(1, device="cuda")
    warm = s.copy()
    binding.adamw_step(cfg, warm.plan(cfg), g, warm.step, lr, norm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.adamw_step(cfg, plan, g, s.step, lr, norm)
    eager = e.plan(cfg)
    for i in range(4):
        lr.fill_(1e-2 / (i + 1))
        for t, seed in ((g[0], i), (g[1], i + 50)):
            t.copy_(torch.randn(t.shape, generator=gen(seed), device="cuda").bfloat16())
        graph.replay()
        binding.adamw_step(cfg, eager, g, e.step, lr)
    assert int(s.step) == 13 and all(torch.equal(x, y) for x, y in zip(s.bits(), e.bits()))


# ------------------------------------------------------------------ the optimizer
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_optimizer_groups_schedule_and_checkpoint(state):
    torch.manual_seed(0)
    ps = [torch.nn.Parameter(torch.randn(k, device="cuda")) for k in (300, 17)]
    opt = AdamW([dict(params=[ps[0]], weight_decay=0.1), dict(params=[ps[1]])], lr=LR, state=state, max_norm=1.0, seed=2)

    def run(opt, ps, n, seed):
        g = gen(seed)
        for _ in range(n):
            for p in ps:
                p.grad = torch.randn(p.shape, generator=g, device="cuda")
            opt.step()

    run(opt, ps, 3, 1)
    kept, at = opt.state_dict(), [p.detach().clone() for p in ps]
    kept = torch.load(_through(kept), weights_only=True)
    for group in opt.param_groups:
        group["lr"] = LR / 2
    run(opt, ps, 2, 7)
    assert float(opt.grad_norm) > 1.0
    ps2 = [torch.nn.Parameter(p) for p in at]
    opt2 = AdamW([dict(params=[ps2[0]], weight_decay=0.1), dict(params=[ps2[1]])], lr=LR, state=state, max_norm=1.0, seed=2)
    opt2.load_state_dict(kept)
    for group in opt2.param_groups:
        group["lr"] = LR / 2
    run(opt2, ps2, 2, 7)
    assert all(torch.equal(a, b) for a, b in zip(ps, ps2))
    opt2.param_groups[1]["lr"] = 1.0
    with pytest.raises(ValueError, match="lr"):
        opt2.step()


def _through(obj):
    import io
    buf = io.BytesIO()
    torch.save(obj, buf)
    buf.seek(0)
    return buf


def test_optimizer_follows_torch():
    """The same steps as torch.optim.AdamW, which updates in another order of float32 operations."""
    torch.manual_seed(0)
    a = [torch.nn.Parameter(torch.randn(k, device="cuda")) for k in (1000, 3)]
    b = [torch.nn.Parameter(p.detach().clone()) for p in a]
    x = AdamW(a, lr=LR, weight_decay=0.1)
    y = torch.optim.AdamW(b, lr=LR, weight_decay=0.1)
    for i in range(20):
        for p, q in zip(a, b):
            p.grad = torch.randn(p.shape, generator=gen(i), device="cuda")
            q.grad = p.grad.clone()
        x.step()
        y.step()
    for p, q in zip(a, b):                                  # 20 steps of lr with some ten roundings each
        assert float((p - q).abs().max()) < 20 * (LR * 32 + 4) * U32 * 4
