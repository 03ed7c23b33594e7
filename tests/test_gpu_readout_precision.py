"""Precision of the readout's cross entropy on the GPU, against float64: what the kernels hold in
fewer bits than float32 only where the caller chose it."""
import math

import pytest
import torch

import seq_reference as ref
from paper_2412_06355_gb300 import XentFunction, binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def inputs(M, V, D, dtype, seed, spread=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    H = torch.randn((M, D), generator=g, device="cuda").to(dtype)
    W = (torch.randn((V, D), generator=g, device="cuda") * (spread / math.sqrt(D))).to(dtype)
    y = torch.randint(0, V, (M,), generator=g, device="cuda")
    y[::7] = -100
    c = torch.rand(M, generator=g, device="cuda") + 0.5
    return H, W, y, c


def terms_reference(H, W, y, c):
    """Gradients in float64 and the bounds of a float32 evaluation that has G within 2^-16 and
    rounds its results to bfloat16 once."""
    want = ref.xent(H.float(), W.float(), y, -100, c)
    keep = (y >= 0).unsqueeze(1)
    Hd, Wd = torch.where(keep, H.double(), 0.0), W.double()
    G = torch.softmax(Hd @ Wd.t(), 1)
    G[torch.arange(len(y), device=y.device), y.clamp_min(0)] -= 1
    G = (G * torch.where(keep, c.double().unsqueeze(1), 0.0)).abs()
    add = dict(ghidden=G @ Wd.abs(), gweight=G.t() @ Hd.abs())
    return {k: (want[k][0], want[k][1] + 2.0 ** -16 * add[k] + ref.rounding(torch.bfloat16, want[k][0]))
            for k in add}


@pytest.mark.parametrize("M,V,D", [(1, 300, 64), (70, 1000, 72), (300, 5000, 520), (513, 777, 65)])
def test_bfloat16_gradients_round_only_the_result(M, V, D):
    H, W, y, c = inputs(M, V, D, torch.bfloat16, M + V)
    if M == 1:
        y[:] = 5
    cfg = binding.make_xent_config(M, V, D, "bf16")
    _, lse = binding.xent_forward(cfg, H, W, y)
    got = binding.xent_backward(cfg, H, W, y, lse, c)
    want = terms_reference(H, W, y, c)
    for k in want:
        ref.check(k, got[k], want[k])


def test_a_rounded_logit_gradient_is_the_callers_choice():
    H, W, y, c = inputs(300, 5000, 264, torch.bfloat16, 3)
    want = ref.xent(H, W, y, -100, c)
    full = terms_reference(H, W, y, c)
    out = {}
    for choice in ("split", "bf16"):
        cfg = binding.make_xent_config(300, 5000, 264, "bf16", logit_grad=choice)
        _, lse = binding.xent_forward(cfg, H, W, y)
        out[choice] = binding.xent_backward(cfg, H, W, y, lse, c)
        h, w = H.clone().requires_grad_(), W.clone().requires_grad_()
        (XentFunction.apply(h, w, y, -100, choice) * c).sum().backward()
        for k, p in (("ghidden", h), ("gweight", w)):
            ref.check(k, p.grad, want[k])
    for k in full:
        ref.check(k, out["bf16"][k], want[k])
        over = (out["bf16"][k].double() - full[k][0]).abs() > full[k][1]
        assert bool(over.any()), k               # the two forms do differ


def exact_logits(M, V, dtype, first, seed):
    """Operands whose logits, first 64 + k with small whole k, are exact in any order of the sum."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    H = torch.zeros(M, 8, device="cuda")
    H[:, 0], H[:, 5] = 64.0, 1.0
    W = torch.zeros(V, 8, device="cuda")
    W[:, 0] = first
    W[:, 5] = torch.randint(-9, 10, (V,), generator=g, device="cuda").float()
    return H.to(dtype), W.to(dtype), torch.randint(0, V, (M,), generator=g, device="cuda")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [3, 20, 200])
@pytest.mark.parametrize("first", [0.0, 62.5, -62.5])
def test_loss_rounds_no_more_than_the_logarithm(dtype, M, first):
    """Exact logits around +-4000: the loss keeps the precision of log(sum exp(l - max)), whose
    terms and sum are off by 2^-18 of it at most, and lse has one rounding of its own."""
    V = 1500
    H, W, y = exact_logits(M, V, torch.float32 if dtype == "f32" else torch.bfloat16, first, M)
    loss, lse = binding.xent_forward(binding.make_xent_config(M, V, 8, dtype), H, W, y)
    logits = H.double() @ W.double().t()
    want = torch.logsumexp(logits, 1)
    wloss = want - logits.gather(1, y.unsqueeze(1)).squeeze(1)
    assert bool(((loss.double() - wloss).abs() <= 2.0 ** -18 + 2 * ref.U32 * wloss.abs()).all())
    assert bool(((lse.double() - want).abs() <= 2.0 ** -18 + ref.U32 * want.abs()).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [3, 20, 200])
@pytest.mark.parametrize("scale", [2.0 ** 31, 2.0 ** 60, 2.0 ** 120])
def test_logits_of_any_finite_size(dtype, M, scale):
    """Two equal logits far above the others, or far below zero with them: the loss is log 2."""
    V = 700
    H = torch.zeros(M, 8, device="cuda")
    H[:, 0] = 2.0 ** 20
    W = torch.full((V, 8), -3.0, device="cuda")
    W[5] = W[650] = -2.0
    W[:, 0] *= scale / 2.0 ** 20
    y = torch.full((M,), 650, device="cuda")
    y[0] = 5
    H[1::2] *= 0.5
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    loss, lse = binding.xent_forward(binding.make_xent_config(M, V, 8, dtype), H.to(dt), W.to(dt), y)
    assert bool(((loss.double() - math.log(2)).abs() <= 2.0 ** -20).all())
    top = H[:, 0].double() * W[5, 0].double()
    assert torch.equal(lse.double(), top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [3, 20, 200, 1500])
def test_probabilities_of_an_autograd_step_keep_their_precision(dtype, M):
    """Exact logits around 4000 (no two rows with the same), one label 10 above the others. The
    probabilities of a row sum to 1 within 2^-18 (exponentials, their sum, the quotient), and with G
    in two bfloat16 terms within another 2^-16; a float32 lse there is off by up to 2^-13. All
    weights share their first column, so grad_hidden's first column is that sum."""
    V = 1500
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    H, W, y = exact_logits(M, V, dt, 62.5, M)
    H[:, 0] = 64 + torch.arange(M, device="cuda") % 50 / 2
    W[:, 5] = -1 - (torch.arange(V, device="cuda") % 9).to(dt)
    W[0, 5] = 9
    y[:] = 0
    y[1::3] = 700
    H.requires_grad_()
    W.requires_grad_()
    loss = XentFunction.apply(H, W, y)
    loss.sum().backward()
    p = torch.softmax(H.detach().double() @ W.detach().double().t(), 1)
    p[torch.arange(M, device="cuda"), y] -= 1
    tol = 2.0 ** -18 + (2.0 ** -15 if dtype == "bf16" else 0)
    assert bool((H.grad[:, 0].double().abs() <= 62.5 * tol).all())
    want = p @ W.detach().double()
    bound = 62.5 * tol + ref.rounding(dt, want) * (1 if dtype == "bf16" else 16)
    assert bool(((H.grad.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [20, 300, 1100])
def test_statistics_as_maximum_and_sum(dtype, M):
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    H, W, y, c = inputs(M, 500, 72, dt, 11)
    y[2] = 500
    out = {}
    for form in ("lse", "max_sum"):
        cfg = binding.make_xent_config(M, 500, 72, dtype, statistics=form)
        loss, lse = binding.xent_forward(cfg, H, W, y)
        out[form] = loss, lse, binding.xent_backward(cfg, H, W, y, lse, c)
    top, total = out["max_sum"][1]
    keep = (y >= 0) & (y < 500)
    assert bool((top[y < 0] == 0).all() and (total[y < 0] == 0).all())
    assert bool(torch.isnan(top[2]) and torch.isnan(total[2]))
    lse = (top.double() + total.double().log())[keep]
    assert bool(((lse - out["lse"][1][keep].double()).abs() <= 4 * (72 ** 0.5) * 2.0 ** -20).all())
    want = ref.xent(H, W, y, -100, c)
    for form in out:
        ref.check("loss", out[form][0], want["loss"])
        for k in ("ghidden", "gweight"):
            ref.check(k, out[form][2][k], want[k])
    with pytest.raises(ValueError, match="lse"):
        binding.xent_backward(cfg, H, W, y, out["lse"][1], c)


@pytest.mark.parametrize("M", [20, 300])
@pytest.mark.parametrize("offset", [0, 1])
def test_weights_read_in_place_or_copied_give_the_same(M, offset):
    H, W, y, c = inputs(M, 500, 72, torch.bfloat16, 12)
    buf = torch.empty(500 * 72 + 8, dtype=torch.bfloat16, device="cuda")
    moved = buf[offset:offset + 500 * 72].view(500, 72).copy_(W)
    cfg = binding.make_xent_config(M, 500, 72, "bf16")
    sizes = binding.dendsn_xent_workspace_size(cfg)
    scratch = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")
    want = binding.xent_forward(cfg, H, W, y, scratch)
    got = binding.xent_forward(cfg, H, moved, y)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    a = binding.xent_backward(cfg, H, W, y, want[1], c, scratch)
    b = binding.xent_backward(cfg, H, moved, y, want[1], c)
    assert all(torch.equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_terms_that_are_left_out_of_float32_products(sign):
    """Operands whose left-out products of terms all have one sign, 2^-24 of each product: the
    logit, which the loss of a hopeless label is, stays within that, its sum's roundings (at most
    2^-23 of the running sum for each of 10 instructions, which are partial) and its own."""
    x = 1 + 2.0 ** -9 * (1 + 126 / 128 + 1 / 256)
    M, V, D = 40, 300, 64
    H = torch.full((M, D), x, device="cuda")
    W = torch.zeros(V, D, device="cuda")
    W[7] = sign * x
    y = torch.full((M,), 3 if sign > 0 else 7, device="cuda")
    loss, _ = binding.xent_forward(binding.make_xent_config(M, V, D), H, W, y)
    l = D * float(torch.tensor(x)) ** 2
    want = l if sign > 0 else math.log(V - 1) + l
    assert bool(((loss.double() - want).abs() <= l * 2.0 ** -21 + 2.0 ** -20).all())
