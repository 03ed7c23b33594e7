"""The gated delta rule over packed tokens where there is little or nothing to do: no sequence, no token."""
import pytest
import torch

from paper_2412_06355_gb300 import DeltaFunction, binding

pytestmark = pytest.mark.gpu
HK, HV, DK, DV = 1, 2, 40, 24


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def tensors(T, dtype):
    n = lambda *s: torch.randn(T, *s, device="cuda")
    return [n(HK, DK).to(dtype), n(HK, DK).to(dtype), n(HV, DV).to(dtype), -n(HV).abs(), torch.sigmoid(n(HV))], n(HV, DV).to(dtype)


def dirty(sizes):
    """Leaves sevens in the memory that the allocator hands out next for tensors of these sizes."""
    kept = [torch.full((s,), 7, dtype=torch.uint8, device="cuda") for s in sizes for _ in range(4)]
    del kept


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [5, 200])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("at", [0, 3])
def test_no_sequence_gives_zeros(dtype, T, kept, at):
    """A token buffer that holds no sequence: every token is one of no sequence."""
    ins, go = tensors(T, dtype)
    offsets = torch.full((1,), at, dtype=torch.int32, device="cuda")
    cfg = binding.make_delta_config(T, 0, HK, HV, DK, DV, "f32" if dtype is torch.float32 else "bf16", "packed")
    sizes = [t.numel() * t.element_size() for t in ins]
    dirty(sizes)
    saved = binding.delta_workspace(cfg) if kept else None
    o, last = binding.delta_forward(cfg, *ins, offsets, saved=saved, want_last=True)
    assert o.shape == go.shape and not o.any() and last.shape == (0, HV, DK, DV)
    if kept:
        dirty(sizes)
        g = binding.delta_backward(cfg, *ins, go, offsets, saved=saved)
        assert set(g) == {"gq", "gk", "gv", "ggate", "gbeta"} and not any(t.any() for t in g.values())


def test_no_sequence_keeps_what_was_there():
    ins, go = tensors(9, torch.float32)
    offsets = torch.zeros(1, dtype=torch.int32, device="cuda")
    cfg = binding.make_delta_config(9, 0, HK, HV, DK, DV, "f32", "packed", rest="keep")
    saved = binding.delta_workspace(cfg)
    scratch = torch.empty(binding.dendsn_delta_workspace_size(cfg)[2] + 16, dtype=torch.uint8, device="cuda")
    outs = [torch.full_like(t, 7.0) for t in (go, *ins)]
    binding.dendsn_delta_forward(cfg, *ins, offsets, None, outs[0], None, saved, scratch)
    binding.dendsn_delta_backward(cfg, go, offsets, None, saved, *outs[1:], None, scratch)
    assert all(bool((t == 7).all()) for t in outs)


def test_no_sequence_through_autograd():
    ins, go = tensors(70, torch.float32)
    leaves = [t.requires_grad_() for t in ins]
    dirty([t.numel() * 4 for t in ins])
    o, _ = DeltaFunction.apply(*leaves, None, torch.zeros(1, dtype=torch.int32, device="cuda"), 1.0, "packed")
    assert not o.any()
    assert not any(g.any() for g in torch.autograd.grad((o * go).sum(), leaves))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B", [1, 2, 70])
def test_sequences_without_a_token(dtype, B):
    """Two value heads share a key head, and there is no token whose gradients could be added up."""
    ins, go = tensors(0, dtype)
    offsets = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    s0, glast = (torch.randn(B, HV, DK, DV, device="cuda") for _ in range(2))
    cfg = binding.make_delta_config(0, B, HK, HV, DK, DV, "f32" if dtype is torch.float32 else "bf16", "packed")
    _, last = binding.delta_forward(cfg, *ins, offsets, s0, want_last=True)
    assert torch.equal(last, s0)
    saved = binding.delta_workspace(cfg)
    o, last = binding.delta_forward(cfg, *ins, offsets, s0, saved=saved, want_last=True)
    assert o.shape == (0, HV, DV) and torch.equal(last, s0)
    g = binding.delta_backward(cfg, *ins, go, offsets, s0, glast, saved)
    assert torch.equal(g["gs0"], glast) and g["gk"].shape == (0, HK, DK)
    leaves = [t.requires_grad_() for t in ins] + [s0.requires_grad_()]
    _, last = DeltaFunction.apply(*leaves, offsets, 1.0, "packed")
    grads = torch.autograd.grad((last * glast).sum(), leaves)
    assert torch.equal(grads[5], glast)
