"""The norm with the residual's addition on the GPU against float64 (block_reference.py). Tolerances
are first-order bounds of a float32 evaluation, element by element, and half a step of the output's type."""
import pytest
import torch

import block_reference as ref
from block_reference import HALF_STEP, U32, within
from paper_2412_06355_gb300 import NormFunction, binding

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def tensors(M, D, dtype, residual, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(M * 31 + D + seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    return (n(M, D).to(DT[dtype]), (2 * n(M, D)).to(DT[dtype]) if residual else None, 1 + 0.2 * n(D),
            n(M, D).to(DT[dtype]), n(M, D).to(DT[dtype]) if residual else None)


def moved(t, k=1):
    """The same values k elements into a buffer."""
    if t is None:
        return None
    buf = torch.empty(t.numel() + k, dtype=t.dtype, device=t.device)
    v = buf[k:].view(t.shape)
    v.copy_(t)
    return v


def check(M, D, dtype, x, residual, w, gy, gsum):
    cfg = binding.make_norm_config(M, D, dtype, EPS)
    y, total, scales = binding.norm_forward(cfg, x, w, residual)
    z, want, _ = ref.norm(x, residual, w, float(torch.tensor(EPS)))
    assert scales is None and torch.equal(total, z)
    c = (D + 16) * U32
    within("y", y, want, want.abs() * (c + HALF_STEP[x.dtype] * (1 + c)))
    gx, bound, gw, gw_bound = ref.norm_backward(z, w, gy, gsum, float(torch.tensor(EPS)))
    got = binding.norm_backward(cfg, total, w, gy, gsum)
    within("gx", got["gx"], gx, bound + (gx.abs() + bound) * HALF_STEP[x.dtype])
    within("gweight", got["gweight"], gw, gw_bound)
    again = binding.norm_backward(cfg, total, w, gy, gsum)
    assert all(torch.equal(got[n], again[n]) for n in got)
    return y, got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,D", [(1, 1), (3, 7), (5, 33), (2, 128), (64, 384), (9, 1000), (700, 1024), (3, 1025),
                                 (4, 2056), (1009, 1001), (5, 4104), (3, 8191), (2, 16384), (2, 16383), (5000, 40)])
def test_norm(dtype, residual, M, D):
    check(M, D, dtype, *tensors(M, D, dtype, residual))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_misaligned_tensors_give_the_same(dtype):
    x, r, w, gy, gs = tensors(50, 512, dtype, True)
    a = check(50, 512, dtype, x, r, w, gy, gs)
    b = check(50, 512, dtype, moved(x), moved(r), moved(w), moved(gy), moved(gs))
    # single elements are summed in another order than vectors: both results are within check's bound of the
    # exact value, (c + half a step) of it, so they are within twice that of each other
    c, half = (512 + 16) * U32, HALF_STEP[x.dtype]
    within("both", a[0].float(), b[0].double(), 2 * (c + half * (1 + c)) / (1 - c - half * (1 + c)) * b[0].double().abs())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("M,D", [(1, 1), (7, 100), (5, 128), (6, 129), (64, 384), (3, 1001), (9, 2048), (2, 8200), (2, 16384), (2, 16383)])
def test_codes(dtype, group, M, D):
    x, r, w, _, _ = tensors(M, D, dtype, True)
    x[0, :5] = 0
    r[0, :5] = 0
    if M > 1:
        x[1], r[1] = 0, 0                                   # a row of zeros: scale 1, codes 0
    cfg = binding.make_norm_config(M, D, dtype, EPS, "e4m3", group)
    y, total, scales = binding.norm_forward(cfg, x, w, r)
    z, want, _ = ref.norm(x, r, w, float(torch.tensor(EPS)))
    assert torch.equal(total, z) and y.dtype == torch.float8_e4m3fn
    width = group or D
    c = (D + 16) * U32
    for n in range((D + width - 1) // width):
        part, codes = want[:, n * width:(n + 1) * width], y[:, n * width:(n + 1) * width]
        top = part.abs().amax(1)
        s = torch.where(top > 0, top / 448, torch.ones_like(top))
        within("scale", scales[:, n], s, s * (c + 4 * U32))
        # half a step of the code: 2^-4 of it from 2^-6 on, 2^-10 below
        value = part / s[:, None]
        within("code", codes, value, value.abs() * (2.0 ** -4 + 2 * c) + 2.0 ** -10)
        assert bool((codes.float().abs().amax(1)[top > 0] == 448).all())


def test_strange_rows_stay_among_themselves():
    M, D = 6, 300
    x, _, w, gy, _ = tensors(M, D, "f32", False)
    cfg = binding.make_norm_config(M, D, "f32", EPS)
    plain, _, _ = binding.norm_forward(cfg, x, w)
    bad = x.clone()
    bad[2, 7], bad[4, 9] = float("nan"), float("inf")
    y, total, _ = binding.norm_forward(cfg, bad, w)
    keep = [0, 1, 3, 5]
    assert torch.equal(y[keep], plain[keep]) and torch.isnan(y[2]).all() and torch.isnan(y[4, 9])
    assert torch.equal(y[4][torch.arange(D, device="cuda") != 9], torch.zeros(D - 1, device="cuda"))
    gx = binding.norm_backward(cfg, total, w, gy)["gx"]
    assert torch.equal(gx[keep], binding.norm_backward(cfg, x, w, gy)["gx"][keep]) and torch.isnan(gx[2]).all()
    for group in (0, 128):
        e = binding.make_norm_config(M, D, "f32", EPS, "e4m3", group)
        _, _, s0 = binding.norm_forward(e, x, w)
        _, _, s1 = binding.norm_forward(e, bad, w)
        assert torch.equal(s0[keep], s1[keep]) and torch.isnan(s1[2]).all()


def test_zero_rows_and_eps():
    x = torch.zeros(3, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    y, _, _ = binding.norm_forward(binding.make_norm_config(3, 64), x, w)
    assert torch.equal(y, x)
    y, _, _ = binding.norm_forward(binding.make_norm_config(3, 64, eps=4.0), x + 2, w)
    within("y", y, torch.full_like(x, 2 / 8 ** 0.5).double(), torch.full_like(x, 8 * U32).double())


def test_in_place_and_empty():
    M, D = 40, 256
    x, r, w, gy, gs = tensors(M, D, "bf16", True)
    cfg = binding.make_norm_config(M, D, "bf16", EPS)
    y, total, _ = binding.norm_forward(cfg, x, w, r)
    g = binding.norm_backward(cfg, total, w, gy, gs)
    scratch = torch.empty(binding.dendsn_norm_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    r2, y2, gs2, gw = r.clone(), torch.empty_like(x), gs.clone(), torch.empty_like(w)
    binding.dendsn_norm_forward(cfg, x, r2, w, r2, y2)
    binding.dendsn_norm_backward(cfg, r2, w, gy, gs2, gs2, gw, scratch)
    assert torch.equal(y, y2) and torch.equal(total, r2) and torch.equal(gs2, g["gx"]) and torch.equal(gw, g["gweight"])
    none = binding.make_norm_config(0, D, "bf16")
    e = x[:0]
    assert binding.norm_forward(none, e, w, e)[0].shape == (0, D)
    assert torch.count_nonzero(binding.norm_backward(none, e, w, e)["gweight"]) == 0


def test_rows_beyond_32_bits():
    M, D = 135000, 16384                                    # M * D > 2^31
    cfg = binding.make_norm_config(M, D, "bf16", EPS)
    x = torch.zeros(M, D, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.randn(D, device="cuda").bfloat16()
    w = torch.ones(D, device="cuda")
    y, _, _ = binding.norm_forward(cfg, x, w)
    one = binding.make_norm_config(1, D, "bf16", EPS)
    assert torch.equal(y[-1:], binding.norm_forward(one, x[-1:].clone(), w)[0]) and not y[:-1].any()


def test_autograd_with_both_outputs_against_differences():
    torch.manual_seed(0)
    M, D = 11, 52
    x, r = torch.randn(M, D, device="cuda", requires_grad=True), torch.randn(M, D, device="cuda", requires_grad=True)
    w = torch.rand(D, device="cuda").add_(0.5).requires_grad_()
    a, b = torch.randn(M, D, device="cuda"), torch.randn(M, D, device="cuda")
    y, s = NormFunction.apply(x, r, w, EPS)
    grads = torch.autograd.grad((y * a + s * b).sum(), (x, r, w))
    assert torch.equal(grads[0], grads[1])

    def loss(x, w):
        z = x + r.detach().double()
        return float((z / torch.sqrt(z.square().mean(1, keepdim=True) + EPS) * w * a + z * b).sum())

    for which, g in ((0, grads[0]), (1, grads[2])):
        at = [x.detach().double(), w.detach().double()]
        d = torch.randn_like(at[which])
        h = 1e-4
        plus, minus = list(at), list(at)
        plus[which], minus[which] = at[which] + h * d, at[which] - h * d
        slope = (loss(*plus) - loss(*minus)) / (2 * h)
        # truncation h^2 of third derivatives (some units here), and float32 gradients
        assert abs(slope - float((g.double() * d).sum())) < 1e-5 * (1 + float((g.double() * d).abs().sum()))
    y, s = NormFunction.apply(x, None, w)
    gx, = torch.autograd.grad((y * a + s * b).sum(), x)
    cfg = binding.make_norm_config(M, D, "f32", 1e-6)
    assert torch.equal(gx, binding.norm_backward(cfg, x.detach(), w.detach(), a, b)["gx"])
    y, s = NormFunction.apply(x, r, w)
    assert torch.equal(torch.autograd.grad((s * b).sum(), r)[0], b)      # nothing reaches y
