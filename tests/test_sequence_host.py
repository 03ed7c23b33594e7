"""Host-side checks of the token-sequence operators: no GPU, no kernel is launched."""
import ctypes

import pytest
import torch

import test_abi_host
from paper_2412_06355_gb300 import binding

P = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    return binding.load()


@pytest.mark.parametrize("struct", [binding.dendsn_embed_config, binding.dendsn_scan_config,
                                    binding.dendsn_xent_config], ids=lambda s: s.__name__)
def test_config_layout_matches_c(struct):
    test_abi_host.test_config_layout_matches_c(struct)


@pytest.mark.parametrize("field,value,status", [
    ("n", -1, 1), ("V", 0, 1), ("D", 0, 1), ("D", -4, 1), ("x_dtype", 2, 1), ("ids_dtype", 2, 1),
    ("n", 2 ** 31, 2)])
def test_embed_config_is_checked(field, value, status):
    cfg = binding.make_embed_config(10, 20, 8)
    setattr(cfg, field, value)
    assert test_abi_host.status_of(binding.dendsn_embed_workspace_size, cfg) == status


@pytest.mark.parametrize("field,value,status", [
    ("T", -1, 1), ("B", -1, 1), ("N", -1, 1), ("x_dtype", 2, 1), ("gate", 2, 1), ("mix", -1, 1),
    ("layout", 2, 1)])
def test_scan_config_is_checked(field, value, status):
    cfg = binding.make_scan_config(10, 2, 8)
    setattr(cfg, field, value)
    assert test_abi_host.status_of(binding.dendsn_scan_workspace_size, cfg) == status


def test_scan_config_with_too_many_channels():
    cfg = binding.make_scan_config(1, 2 ** 20, 2 ** 20)
    assert test_abi_host.status_of(binding.dendsn_scan_workspace_size, cfg) == 2


@pytest.mark.parametrize("field,value,status", [
    ("M", -1, 1), ("V", 0, 1), ("D", 0, 1), ("x_dtype", 2, 1), ("labels_dtype", 2, 1)])
def test_xent_config_is_checked(field, value, status):
    cfg = binding.make_xent_config(10, 20, 8)
    setattr(cfg, field, value)
    assert test_abi_host.status_of(binding.dendsn_xent_workspace_size, cfg) == status


@pytest.mark.parametrize("scale", [float("nan"), float("inf")])
def test_embed_scale_has_to_be_finite(scale):
    cfg = binding.make_embed_config(10, 20, 8, scale=scale)
    assert test_abi_host.status_of(binding.dendsn_embed_workspace_size, cfg) == 1


def test_xent_scratch_is_bounded():
    """The backward's scratch holds one piece of the vocabulary, not M V values."""
    M, V, D = 8192, 131072, 64
    fwd, bwd = binding.dendsn_xent_workspace_size(binding.make_xent_config(M, V, D, "bf16"))
    assert bwd < M * V * 2 / 3 and fwd < M * V * 4 / 16
    _, more = binding.dendsn_xent_workspace_size(binding.make_xent_config(M, 4 * V, D, "bf16"))
    assert more - bwd < 3 * V * D * 2 + (1 << 20)          # the packed weights, nothing of G


def test_make_configs_refuse_unknown_names():
    for f, kw in ((binding.make_embed_config, dict(n=1, V=2, D=3)),
                  (binding.make_scan_config, dict(T=1, B=2, N=3)),
                  (binding.make_xent_config, dict(M=1, V=2, D=3))):
        with pytest.raises(ValueError, match="dtype"):
            f(**kw, dtype="f16")
    with pytest.raises(ValueError, match="gate"):
        binding.make_scan_config(1, 2, 3, gate="sigmoid")
    with pytest.raises(ValueError, match="layout"):
        binding.make_scan_config(1, 2, 3, layout="paper")
    with pytest.raises(ValueError, match="labels_dtype"):
        binding.make_xent_config(1, 2, 3, labels_dtype="i8")


def test_scan_checkpoints_every_64_steps():
    size = lambda T: binding.dendsn_scan_workspace_size(binding.make_scan_config(T, 2, 8))
    assert [size(T) for T in (0, 1, 64, 65, 128, 129)] == [0, 0, 0, 64, 64, 128]


def test_null_and_misaligned_pointers_are_refused(lib):
    ok, odd = P(4096), P(4097)
    e = ctypes.byref(binding.make_embed_config(10, 20, 8))
    assert lib.dendsn_embed_forward(e, None, ok, ok, None) == 1
    assert lib.dendsn_embed_forward(e, odd, ok, ok, None) == 3
    assert lib.dendsn_embed_backward(e, ok, ok, None, ok, None) == 1
    assert lib.dendsn_embed_backward(e, ok, ok, P(4098), ok, None) == 3
    assert lib.dendsn_embed_backward(e, P(4100), ok, ok, ok, None) == 3     # int64 ids
    s = ctypes.byref(binding.make_scan_config(100, 2, 8))
    assert lib.dendsn_scan_forward(s, ok, None, None, None, ok, None, None, None) == 1
    assert lib.dendsn_scan_forward(s, ok, ok, None, odd, ok, None, None, None) == 3
    assert lib.dendsn_scan_forward(s, ok, ok, None, None, ok, None, P(4104), None) == 3
    assert lib.dendsn_scan_backward(s, ok, ok, None, None, ok, None, None, ok, ok, None, None) == 1
    assert b"saved" in lib.dendsn_last_error()
    x = ctypes.byref(binding.make_xent_config(10, 20, 8))
    assert lib.dendsn_xent_forward(x, ok, ok, None, ok, ok, ok, None) == 1
    assert lib.dendsn_xent_forward(x, ok, ok, ok, ok, odd, ok, None) == 3
    assert lib.dendsn_xent_backward(x, ok, ok, ok, ok, ok, ok, ok, None, None) == 1
    assert b"scratch" in lib.dendsn_last_error()
    assert lib.dendsn_xent_backward(x, ok, ok, ok, ok, ok, ok, ok, P(4112), None) == 3
    assert lib.dendsn_xent_backward(None, ok, ok, ok, ok, ok, ok, ok, ok, None) == 1


def test_binding_refuses_other_shapes_and_dtypes():
    cfg = binding.make_embed_config(4, 10, 8)
    ids, table = torch.zeros(4, dtype=torch.int64), torch.zeros(10, 8)
    for bad in (dict(table=torch.zeros(9, 8)), dict(table=table.bfloat16()), dict(ids=ids.int()),
                dict(ids=ids[:3]), dict(out=torch.zeros(4, 9))):
        kw = dict(table=table, ids=ids, out=torch.zeros(4, 8))
        kw.update(bad)
        with pytest.raises(ValueError, match=next(iter(bad))):
            binding.dendsn_embed_forward(cfg, **kw)
    with pytest.raises(ValueError, match="CUDA"):
        binding.dendsn_embed_forward(cfg, table, ids, torch.zeros(4, 8))
    cfg = binding.make_scan_config(70, 2, 8, layout="batch")
    x = torch.zeros(2, 70, 8)
    for bad in (dict(x=torch.zeros(70, 2, 8)), dict(starts=torch.zeros(70, 2, dtype=torch.uint8)),
                dict(starts=torch.zeros(2, 70)), dict(h0=torch.zeros(2, 7)),
                dict(saved=torch.zeros(3))):
        kw = dict(x=x, gate=x, starts=None, h0=None, h=x.clone(), saved=None)
        kw.update(bad)
        with pytest.raises(ValueError, match=next(iter(bad))):
            binding.dendsn_scan_forward(cfg, **kw)
    with pytest.raises(ValueError, match="saved"):
        binding.dendsn_scan_backward(cfg, x, x, None, None, x, None, None, x.clone(), x.clone())
    cfg = binding.make_xent_config(4, 10, 8)
    h, w, y, r = torch.zeros(4, 8), torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    for bad in (dict(hidden=torch.zeros(5, 8)), dict(weight=torch.zeros(10, 9)), dict(labels=y.int()),
                dict(lse=torch.zeros(4, dtype=torch.float64))):
        kw = dict(hidden=h, weight=w, labels=y, loss=r, lse=r.clone(), scratch=None)
        kw.update(bad)
        with pytest.raises(ValueError, match=next(iter(bad))):
            binding.dendsn_xent_forward(cfg, **kw)
    with pytest.raises(ValueError, match="scratch"):
        binding.dendsn_xent_backward(cfg, h, w, y, r, r, h.clone(), w.clone(), None)
