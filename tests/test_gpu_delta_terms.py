"""The gated delta rule's factors in three bfloat16 terms, for bfloat16 inputs too: results that are small differences of
large products, so that what a factor was rounded by stands far above the output's own rounding.

Bound. Of the magnitudes M of the products that an output sums: three terms leave at most U32 of either factor and of
the products that are left out (4 U32); the matrix instruction cuts a sum off by up to 2 U32 with every 16 summed
places, 128 at most (16 U32); a power of two is within 4 U32; some four operations around. 28 U32 M, and half a
step of the output. A factor in two terms may be off by 128 U32 of itself, so by 64 U32 of M where two products
cancel; over the 500 and more outputs of a case the largest come near that."""
import pytest
import torch

import block_reference as ref
from block_reference import HALF_STEP, U32, within
from paper_2412_06355_gb300 import binding

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
B, H, DV, EPS = 4, 4, 128, 2.0 ** -12


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def rand(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.rand(shape, generator=g, device="cuda") + 1.0       # one binade, 24 bits


def run(dtype, T, Dk, Dv=DV, grads=None, **given):
    """Zeros but for what is given (by name, [B, T, H, ...] or a state's shape); gate 0, beta 1, scale 1. Returns the
    outputs and the float64 recurrence's, whose gradients are autograd's."""
    x = dict(q=torch.zeros(B, T, H, Dk), k=torch.zeros(B, T, H, Dk), v=torch.zeros(B, T, H, Dv), gate=torch.zeros(B, T, H),
             beta=torch.ones(B, T, H), s0=torch.zeros(B, H, Dk, Dv), go=torch.zeros(B, T, H, Dv), glast=torch.zeros(B, H, Dk, Dv))
    x = {n: given.get(n, t.cuda()).contiguous() for n, t in x.items()}
    for n in ("q", "k", "v", "go"):
        x[n] = x[n].to(DT[dtype])
    cfg = binding.make_delta_config(T, B, H, H, Dk, Dv, dtype, "batch", 1.0)
    ins = [x[n] for n in ("q", "k", "v", "gate", "beta")]
    saved = binding.delta_workspace(cfg)
    o, last = binding.delta_forward(cfg, *ins, None, x["s0"], saved=saved, want_last=True)
    got = {"o": o, "last": last, **binding.delta_backward(cfg, *ins, x["go"], None, x["s0"], x["glast"], saved)}
    served, _ = binding.delta_forward(cfg, *ins, None, x["s0"])       # the build that keeps nothing
    leaves = [t.double().reshape(B * T, *t.shape[2:]).requires_grad_() for t in ins] + [x["s0"].double().requires_grad_()]
    wo, wlast = ref.delta(*leaves, ref.sequences("batch", T, B, None), 1.0)
    g = torch.autograd.grad((wo * x["go"].double().view_as(wo)).sum() + (wlast * x["glast"].double()).sum(), leaves)
    want = {"o": wo.detach().view(o.shape), "last": wlast.detach()}
    want.update({n: t.view(got[n].shape) for n, t in zip(("gq", "gk", "gv", "ggate", "gbeta", "gs0"), g)})
    return got, want, served


def small(name, got, want, M):
    """M: magnitudes of the products summed, as `want` lies."""
    assert float(want.abs().max()) < 2.0 ** -8 * float(torch.as_tensor(M).max()), "nothing cancels"
    within(name, got, want, 28 * U32 * M + HALF_STEP[got.dtype] * (want.abs() + 28 * U32 * M))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_read_the_state_in_three_terms(dtype):
    a = rand(1, B, H, DV)
    s0 = torch.stack([a, a * (1 + EPS)], 2)
    q = torch.tensor([1.0, -1.0], device="cuda").expand(B, 9, H, 2)
    got, want, served = run(dtype, 9, 2, s0=s0, q=q)
    M = 2 * a.double()[:, None]
    small("o", got["o"], want["o"], M)
    small("o", served, want["o"], M)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gates", [False, True])
def test_outputs_read_the_writes_in_three_terms(dtype, gates):
    """Two tokens write along two keys, the others read the difference: factors u, and exp(G_i - G_j) with gates."""
    T = 12
    k, q = torch.zeros(B, T, H, 2, device="cuda"), torch.zeros(B, T, H, 2, device="cuda")
    k[:, 0, :, 0] = k[:, 1, :, 1] = 1
    q[:, 2:, :, 0], q[:, 2:, :, 1] = 1, -1
    beta = torch.ones(B, T, H, device="cuda")
    beta[:, 0] = rand(2, B, H) / 2
    beta[:, 1] = beta[:, 0] * (1 - EPS)
    gate = torch.zeros(B, T, H, device="cuda")
    if gates:
        gate[:, 1] = -EPS * 0.9
        gate[:, 2:] = -0.1 * rand(3, B, T - 2, H)
    v = rand(4, B, 1, H, DV).to(DT[dtype]).float().repeat(1, T, 1, 1)
    got, want, served = run(dtype, T, 2, k=k, q=q, beta=beta, gate=gate, v=v)
    M = (2 * v * beta[:, :1, :, None]).double()[:, 2:] * torch.exp(gate.double().cumsum(1))[:, 2:, :, None]
    small("o", got["o"][:, 2:], want["o"][:, 2:], M)
    small("o", served[:, 2:], want["o"][:, 2:], M)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gk_reads_the_states_gradient_in_three_terms(dtype):
    a, v = rand(5, B, H, 64), torch.zeros(B, 2, H, 2, device="cuda")
    v[..., 0], v[..., 1] = 1, -1
    got, want, _ = run(dtype, 2, 64, 2, v=v, glast=torch.stack([a, a * (1 + EPS)], 3))
    small("gk", got["gk"], want["gk"], 2 * a.double()[:, None])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("which", ["e", "y"])
def test_gk_reads_e_and_y_in_three_terms(dtype, which):
    """gk = D e - S y of one token with k along the first place, whose row one of the two matrices has."""
    Dk = 64
    a = rand(6, B, H)
    first, other = torch.zeros(B, H, Dk, 2, device="cuda"), torch.zeros(B, H, Dk, 2, device="cuda")
    first[:, :, 0, 0], first[:, :, 0, 1] = a, a * (1 + EPS)
    other[:, :, 1:, 0], other[:, :, 1:, 1] = 1, -1
    k = torch.zeros(B, 1, H, Dk, device="cuda")
    k[..., 0] = 1
    got, want, _ = run(dtype, 1, Dk, 2, k=k, **(dict(s0=first, glast=other) if which == "e" else dict(s0=other, glast=first)))
    M = (2 * a.double())[:, None, :, None]
    small("gk", got["gk"][..., 1:], want["gk"][..., 1:], M.expand(B, 1, H, Dk - 1))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gk_reads_the_chunks_matrices_in_three_terms(dtype):
    """go_i . u_j along tokens whose queries cancel, and y_i . u_j, b_i near 1, against what comes through the state."""
    T, Dk = 40, 8
    q = torch.zeros(B, T, H, Dk, device="cuda")
    q[:, 20], q[:, 21] = 1, -1
    beta, go = rand(7, B, T, H) / 2, torch.zeros(B, T, H, DV, device="cuda")
    gate = torch.zeros(B, T, H, device="cuda")
    gate[:, 21] = -EPS
    go[:, 20] = go[:, 21] = rand(8, B, H, DV)
    v = rand(9, B, T, H, DV)
    got, want, _ = run(dtype, T, Dk, q=q, beta=beta, gate=gate, go=go, v=v)
    dot = (go[:, 20:21].to(DT[dtype]).double() * v.to(DT[dtype]).double()).sum(-1) * beta.double()
    small("gk", got["gk"][:, :20], want["gk"][:, :20], 2 * dot[:, :20, :, None].expand(B, 20, H, Dk))

    k = torch.zeros(B, T, H, Dk, device="cuda")
    k[:, 20:, :, 0] = 1
    beta = torch.ones(B, T, H, device="cuda")
    beta[:, :20] = rand(10, B, 20, H) / 2
    beta[:, 20] = 1 - 2.0 ** -9 * rand(11, B, H)
    beta[:, 21:] = 0
    glast = torch.zeros(B, H, Dk, DV, device="cuda")
    glast[:, :, 0] = rand(12, B, H, DV)
    got, want, _ = run(dtype, T, Dk, k=k, beta=beta, v=v, glast=glast)
    dot = (glast[:, None, :, 0].double() * v.to(DT[dtype]).double()).sum(-1) * beta.double()
    small("gk", got["gk"][:, :20, :, 0], want["gk"][:, :20, :, 0], 2 * dot[:, :20])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gq_reads_the_state_in_three_terms(dtype):
    a, go = rand(13, B, H, 64), torch.zeros(B, 9, H, 2, device="cuda")
    go[..., 0], go[..., 1] = 1, -1
    got, want, _ = run(dtype, 9, 64, 2, go=go, s0=torch.stack([a, a * (1 + EPS)], 3))
    small("gq", got["gq"], want["gq"], 2 * a.double()[:, None])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gq_reads_the_chunks_matrix_in_three_terms(dtype):
    """Two tokens write along keys that cancel each other for every later token's gradient: A_i0 k_0 + A_i1 k_1."""
    T, Dk = 40, 8
    k, v, beta = torch.zeros(B, T, H, Dk, device="cuda"), torch.zeros(B, T, H, DV, device="cuda"), rand(14, B, T, H) / 2
    half = torch.tensor([1.0, -1.0] * (Dk // 2), device="cuda") / 256        # so short that token 1 reads 2^-13 of what token 0 wrote
    k[:, 0], k[:, 1] = half, -half
    v[:, 0] = v[:, 1] = rand(15, B, H, DV)
    beta[:, 1] = beta[:, 0] * (1 + EPS)
    go = rand(16, B, T, H, DV)
    gate = torch.zeros(B, T, H, device="cuda")
    gate[:, 1] = -EPS / 2
    got, want, _ = run(dtype, T, Dk, k=k, v=v, beta=beta, gate=gate, go=go)
    dot = (go.to(DT[dtype]).double() * v[:, :1].to(DT[dtype]).double()).sum(-1) * beta[:, :1].double()
    small("gq", got["gq"][:, 2:], want["gq"][:, 2:], (2 * dot[:, 2:, :, None] / 256).expand(B, T - 2, H, Dk))
