"""Host-side checks of norm, gated delta rule and AdamW: no GPU, no kernel is launched."""
import ctypes

import pytest
import torch

import test_abi_host
from paper_2412_06355_gb300 import binding

P = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    return binding.load()


@pytest.mark.parametrize("struct", [binding.dendsn_norm_config, binding.dendsn_delta_config,
                                    binding.dendsn_adamw_config, binding.dendsn_adamw_tensor],
                         ids=lambda s: s.__name__)
def test_layout_matches_c(struct):
    test_abi_host.test_config_layout_matches_c(struct)


@pytest.mark.parametrize("field,value,status", [
    ("M", -1, 1), ("D", 0, 1), ("x_dtype", 2, 1), ("out", 2, 1), ("group", 64, 1), ("eps", -1.0, 1),
    ("eps", float("nan"), 1), ("eps", float("inf"), 1), ("D", 16385, 2), ("M", 2 ** 40, 0), ("eps", 0.0, 0)])
def test_norm_config_is_checked(field, value, status):
    cfg = binding.make_norm_config(10, 20)
    setattr(cfg, field, value)
    assert test_abi_host.status_of(binding.dendsn_norm_workspace_size, cfg) == status


@pytest.mark.parametrize("field,value,status", [
    ("T", -1, 1), ("B", -1, 1), ("Hk", 0, 1), ("Hv", 3, 1), ("Dk", 0, 1), ("Dv", 0, 1), ("x_dtype", 2, 1),
    ("layout", 3, 1), ("rest", 2, 1), ("scale", float("inf"), 1), ("Dk", 129, 2), ("Dv", 129, 2),
    ("Hv", 65536, 2), ("T", 0, 0), ("B", 0, 0)])
def test_delta_config_is_checked(field, value, status):
    cfg = binding.make_delta_config(10, 2, 2, 4, 8, 8)
    setattr(cfg, field, value)
    assert test_abi_host.status_of(binding.dendsn_delta_workspace_size, cfg) == status


def test_delta_with_too_many_chunks():
    cfg = binding.make_delta_config(2 ** 20, 2 ** 20, 1, 1, 8, 8)
    assert test_abi_host.status_of(binding.dendsn_delta_workspace_size, cfg) == 2


@pytest.mark.parametrize("field,value", [
    ("lr", float("nan")), ("beta1", 1.0), ("beta1", -0.1), ("beta2", 1.5), ("eps", -1e-8),
    ("max_norm", -1.0), ("max_norm", float("inf")), ("state", 2)])
def test_adamw_config_is_checked(lib, field, value):
    cfg = binding.make_adamw_config()
    setattr(cfg, field, value)
    assert lib.dendsn_adamw_plan(ctypes.byref(cfg), None, 0, None, None) == 1


def test_names_are_checked():
    with pytest.raises(ValueError, match="out"):
        binding.make_norm_config(1, 2, out="fp8")
    with pytest.raises(ValueError, match="layout"):
        binding.make_delta_config(1, 1, 1, 1, 8, 8, layout="ragged")
    with pytest.raises(ValueError, match="rest"):
        binding.make_delta_config(1, 1, 1, 1, 8, 8, rest="nan")
    with pytest.raises(ValueError, match="state"):
        binding.make_adamw_config(state="int8")


def test_pointers_are_checked(lib):
    ok, odd, half = P(4096), P(4097), P(4098)
    n = ctypes.byref(binding.make_norm_config(10, 20))
    assert lib.dendsn_norm_forward(n, ok, None, None, None, ok, None, None) == 1
    assert lib.dendsn_norm_forward(n, ok, ok, ok, None, ok, None, None) == 1            # residual without sum
    assert lib.dendsn_norm_forward(n, ok, None, ok, ok, ok, None, None) == 1            # sum without residual
    assert lib.dendsn_norm_forward(n, half, None, ok, None, ok, None, None) == 3
    e = ctypes.byref(binding.make_norm_config(10, 20, out="e4m3"))
    assert lib.dendsn_norm_forward(e, ok, None, ok, None, odd, None, None) == 1         # scales
    assert lib.dendsn_norm_forward(e, ok, None, ok, None, odd, odd, None) == 3
    assert lib.dendsn_norm_backward(n, ok, ok, ok, None, ok, ok, None, None) == 1
    assert b"scratch" in lib.dendsn_last_error()
    assert lib.dendsn_norm_backward(n, ok, ok, ok, None, ok, ok, P(4104), None) == 3
    d = binding.make_delta_config(100, 2, 2, 4, 8, 8)
    c = ctypes.byref(d)
    assert lib.dendsn_delta_forward(c, ok, ok, ok, ok, ok, None, None, ok, None, None, None, None) == 1
    assert b"scratch" in lib.dendsn_last_error()
    assert lib.dendsn_delta_forward(c, ok, ok, ok, ok, ok, ok, None, ok, None, None, ok, None) == 1     # offsets
    assert lib.dendsn_delta_forward(c, ok, None, ok, ok, ok, None, None, ok, None, None, ok, None) == 1
    assert lib.dendsn_delta_forward(c, ok, ok, half, ok, ok, None, None, ok, None, None, ok, None) == 3
    assert lib.dendsn_delta_forward(c, ok, ok, ok, ok, ok, None, None, ok, None, P(4224), None, None) == 3
    assert lib.dendsn_delta_backward(c, ok, None, None, ok, ok, ok, ok, ok, ok, None, None, None) == 1
    assert lib.dendsn_delta_backward(c, ok, None, None, None, ok, ok, ok, ok, ok, None, ok, None) == 1
    assert lib.dendsn_delta_backward(c, ok, None, odd, ok, ok, ok, ok, ok, ok, None, ok, None) == 3
    d.layout = binding.DELTA_PACKED
    assert lib.dendsn_delta_forward(c, ok, ok, ok, ok, ok, None, None, ok, None, None, ok, None) == 1
    assert b"offsets" in lib.dendsn_last_error()
    a = ctypes.byref(binding.make_adamw_config())
    sizes, grads, kinds = (ctypes.c_int64 * 1)(4), (P * 1)(4098), (ctypes.c_int32 * 1)(0)
    assert lib.dendsn_adamw_step(a, None, sizes, 1, grads, kinds, ok, None, None, None) == 1
    assert lib.dendsn_adamw_step(a, ok, sizes, 1, grads, kinds, ok, None, None, None) == 3
    assert lib.dendsn_adamw_step(a, ok, sizes, 1, None, kinds, ok, None, None, None) == 1
    kinds[0] = 7
    assert lib.dendsn_adamw_step(a, ok, sizes, 1, grads, kinds, ok, None, None, None) == 1
    kinds[0] = 1
    assert lib.dendsn_adamw_step(a, ok, sizes, 1, grads, kinds, odd, None, None, None) == 3


def test_adamw_plan_checks_its_tensors(lib):
    def plan(state="f32", **kw):
        t = binding.dendsn_adamw_tensor(4096, 8192, 16384, 0, 0, 10, 0.0, binding.F32, 0)
        for name, value in kw.items():
            setattr(t, name, value)
        need = ctypes.c_size_t(0)
        st = lib.dendsn_adamw_plan(ctypes.byref(binding.make_adamw_config(state=state)), ctypes.byref(t), 1,
                                   None, ctypes.byref(need))
        return st if st else need.value

    small = plan()
    assert small > 64 and plan(n=4096) == small and plan(n=4097) == small + 4
    assert plan(n=-1) == 1 and plan(param_dtype=3) == 1 and plan(weight_decay=float("nan")) == 1
    assert plan(param=None) == 1 and plan(m=None) == 1 and plan(state="e4m3") == 1
    assert plan(state="e4m3", scales=4096) == small and plan(state="e4m3", scales=4100) == 3
    assert plan(param=4098) == 3 and plan(param=4098, param_dtype=binding.BF16) == small
    assert plan(copy=4097) == 3 and plan(m=4097) == 3
    assert plan(n=0, param=None, m=None, v=None) == small - 4
    assert plan(n=2 ** 31 * 4096) == 2


def test_binding_refuses_other_shapes_and_dtypes():
    cfg = binding.make_norm_config(4, 8)
    x, w = torch.zeros(2, 2, 8), torch.zeros(8)
    for bad in (dict(x=x[:1]), dict(x=x.bfloat16()), dict(weight=w.bfloat16()), dict(residual=torch.zeros(4, 7)),
                dict(y=torch.zeros(8, 4)), dict(y=None)):
        kw = dict(x=x, residual=None, weight=w, sum=None, y=x.clone())
        kw.update(bad)
        with pytest.raises(ValueError, match=next(iter(bad))):
            binding.dendsn_norm_forward(cfg, **kw)
    with pytest.raises(ValueError, match="CUDA"):
        binding.dendsn_norm_forward(cfg, x, None, w, None, x.clone())
    eight = binding.make_norm_config(4, 300, out="e4m3", group=128)
    y = torch.zeros(4, 300, dtype=binding.E4M3)
    with pytest.raises(ValueError, match="scales"):
        binding.dendsn_norm_forward(eight, torch.zeros(4, 300), None, torch.zeros(300), None, y, torch.zeros(4, 2))
    with pytest.raises(ValueError, match="scratch"):
        binding.dendsn_norm_backward(cfg, x, w, x, None, x.clone(), w.clone(), None)

    cfg = binding.make_delta_config(70, 2, 1, 2, 8, 4, layout="batch")
    q, v, gt, s = torch.zeros(2, 70, 1, 8), torch.zeros(2, 70, 2, 4), torch.zeros(2, 70, 2), torch.zeros(2, 2, 8, 4)
    for bad in (dict(q=torch.zeros(70, 2, 1, 8)), dict(v=v.bfloat16()), dict(gate=gt.bfloat16()), dict(beta=gt[:1]),
                dict(s0=s[:, :1]), dict(last=s.bfloat16()), dict(saved=torch.zeros(3)), dict(scratch=None),
                dict(offsets=torch.zeros(3, dtype=torch.int32))):
        kw = dict(q=q, k=q, v=v, gate=gt, beta=gt, offsets=None, s0=s, o=v.clone(), scratch=torch.zeros(2 ** 20))
        kw.update(bad)
        with pytest.raises(ValueError, match=next(iter(bad))):
            binding.dendsn_delta_forward(cfg, **kw)
    with pytest.raises(ValueError, match="saved"):
        binding.dendsn_delta_backward(cfg, v, None, None, None, q, q, v, gt, gt, None, None)
    packed = binding.make_delta_config(70, 2, 1, 2, 8, 4, layout="packed")
    with pytest.raises(ValueError, match="offsets"):
        binding.dendsn_delta_forward(packed, q[0], q[0], v[0], gt[0], gt[0], None, None, v[0].clone(),
                                     scratch=torch.zeros(2 ** 20))


def test_adamw_lists_are_checked():
    cfg, p = binding.make_adamw_config(), torch.zeros(300)
    with pytest.raises(ValueError, match="CUDA"):
        binding.adamw_plan(cfg, [p], [p], [p])
    with pytest.raises(ValueError, match="ms"):
        binding.adamw_plan(cfg, [p], [], [p])
    with pytest.raises(ValueError, match="weight_decay"):
        binding.adamw_plan(cfg, [p], [p], [p], weight_decay=[0.1, 0.2])
    with pytest.raises(ValueError, match="m of tensor 0"):
        binding.adamw_plan(cfg, [p], [p[:3]], [p])
    with pytest.raises(ValueError, match="dtype"):
        binding.adamw_plan(cfg, [p.half()], [p], [p])
    with pytest.raises(ValueError, match="copy"):
        binding.adamw_plan(cfg, [p], [p], [p], copies=[p])
    eight, c = binding.make_adamw_config(state="e4m3"), torch.zeros(300, dtype=binding.E4M3)
    with pytest.raises(ValueError, match="scales"):
        binding.adamw_plan(eight, [p], [c], [c])
    with pytest.raises(ValueError, match="scales"):
        binding.adamw_plan(eight, [p], [c], [c], scales=[torch.zeros(1, 2)])


def test_packed_slots_never_meet():
    """A sequence from token lo on has the chunk slots from lo // 64 + its number on: disjoint, below
    T // 64 + B, for any lengths (the kernels place tiles by them)."""
    g = torch.Generator().manual_seed(1)
    for _ in range(300):
        B = int(torch.randint(1, 9, (1,), generator=g))
        lens = torch.randint(0, 200, (B,), generator=g).tolist()
        T, at, seen = sum(lens) + int(torch.randint(0, 3, (1,), generator=g)), 0, set()
        for b, n in enumerate(lens):
            for c in range((n + 63) // 64):
                slot = at // 64 + b + c
                assert slot not in seen and slot < T // 64 + B
                seen.add(slot)
            at += n
