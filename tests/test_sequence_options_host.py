"""Host-side checks of the token-sequence operators' options: no GPU, no kernel is launched."""
import contextlib
import ctypes
import subprocess

import pytest
import torch

import test_abi_host
from paper_2412_06355_gb300 import binding, build


def test_logit_grad_is_checked():
    cfg = binding.make_xent_config(10, 20, 8, "bf16", logit_grad="bf16")
    assert test_abi_host.status_of(binding.dendsn_xent_workspace_size, cfg) == 0
    cfg.logit_grad = 2
    assert test_abi_host.status_of(binding.dendsn_xent_workspace_size, cfg) == 1
    cfg = binding.make_xent_config(10, 20, 8, "f32", logit_grad="bf16")
    assert test_abi_host.status_of(binding.dendsn_xent_workspace_size, cfg) == 1
    with pytest.raises(ValueError, match="logit_grad"):
        binding.make_xent_config(10, 20, 8, "bf16", logit_grad="f16")


# ------------------------------------------------------------------ wrappers and streams
class FakeLibrary:
    """The library with calls that launch replaced by nothing."""

    def __init__(self, lib):
        self.lib = lib

    def __getattr__(self, name):
        real = getattr(self.lib, name)
        return real if name.endswith(("_size", "_error")) else lambda *a: 0


class Recorder:
    """Stands in for torch.cuda.stream: which stream is current at every allocation."""

    def __init__(self, monkeypatch):
        self.current, self.seen = None, []
        lib = FakeLibrary(binding.load())
        monkeypatch.setattr(binding, "load", lambda: lib)
        monkeypatch.setattr(binding, "_pointers", lambda *t: [None] * len(t))
        monkeypatch.setattr(binding, "_ptr", lambda t: None)
        monkeypatch.setattr(binding, "_stream", lambda s: None)
        monkeypatch.setattr(torch.cuda, "stream", self.use)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: ("external", handle))
        for name in ("empty", "empty_like"):
            monkeypatch.setattr(torch, name, self.recorded(getattr(torch, name)))

    @contextlib.contextmanager
    def use(self, stream):
        before, self.current = self.current, stream
        yield
        self.current = before

    def recorded(self, fn):
        def call(*a, **kw):
            self.seen.append(self.current)
            return fn(*a, **kw)
        return call


def wrappers():
    """name -> (call of an allocating wrapper with a stream, tensors it allocates)."""
    z = torch.zeros
    ce, ids = binding.make_embed_config(4, 10, 8), z(4, dtype=torch.int64)
    cs, x = binding.make_scan_config(3, 2, 8), z(3, 2, 8)
    cx, h, w, y, r = binding.make_xent_config(4, 10, 8), z(4, 8), z(10, 8), z(4, dtype=torch.int64), z(4)
    cl = binding.make_lif_config(3, 2, 8)
    cd = binding.make_config(T=4, B=2, N=64, K=4, C=4, inner=16)
    xd, ck, cb, sp = z(4, 2, 64, 4), z(4, 4), z(4, 4 // cd.G), z(4, 2, 64)
    return {
        "embed_forward": (lambda s: binding.embed_forward(ce, w, ids, stream=s), 1),
        "embed_backward": (lambda s: binding.embed_backward(ce, ids, h, stream=s), 2),
        "scan_forward": (lambda s: binding.scan_forward(cs, x, x, want_last=True, stream=s), 2),
        "scan_backward": (lambda s: binding.scan_backward(cs, x, x, x, None, z(2, 8), stream=s), 3),
        "xent_forward": (lambda s: binding.xent_forward(cx, h, w, y, stream=s), 3),
        "xent_backward": (lambda s: binding.xent_backward(cx, h, w, y, r, r, None, s), 3),
        "lif_forward": (lambda s: binding.lif_forward(cl, x, True, None, s), 2),
        "lif_backward": (lambda s: binding.lif_backward(cl, x, x, stream=s), 1),
        "forward": (lambda s: binding.forward(cd, xd, ck, ck, cb, cb, want_v=True, stream=s), 2),
        "backward": (lambda s: binding.backward(cd, xd, ck, ck, cb, cb, None, sp, stream=s), 6),
    }


class SideStream:
    cuda_stream = 64


@pytest.mark.parametrize("name", list(wrappers()))
def test_wrappers_allocate_under_the_stream_they_launch_on(name, monkeypatch):
    """Memory of another stream could be handed out again while the kernels still use it."""
    call, count = wrappers()[name]
    rec = Recorder(monkeypatch)
    side = SideStream()
    for given, current in ((None, None), (side, side), (4096, ("external", 4096)),
                           (1, ("external", 0))):
        rec.seen.clear()
        call(given)
        assert len(rec.seen) >= count and all(s == current for s in rec.seen), (given, rec.seen)
        assert rec.current is None


def test_statistics_are_checked():
    cfg = binding.make_xent_config(10, 20, 8, "bf16", statistics="max_sum")
    assert test_abi_host.status_of(binding.dendsn_xent_workspace_size, cfg) == 0
    cfg.statistics = 2
    assert test_abi_host.status_of(binding.dendsn_xent_workspace_size, cfg) == 1
    with pytest.raises(ValueError, match="statistics"):
        binding.make_xent_config(10, 20, 8, "bf16", statistics="sum")


# ------------------------------------------------------------------ the embedding's index
INDEX_GRID = r"""
#include <stdio.h>
#include "seq/embed_plan.h"
int main() {
    long long n, V;
    int sms;
    while (scanf("%lld %lld %d", &n, &V, &sms) == 3) {
        const dendsn::IndexGrid g = dendsn::index_grid(n, V, sms);
        printf("%d %d %d\n", (int)g.cluster, g.blocks, g.chunk);
    }
}
"""


def test_the_index_grid_fits_the_device(tmp_path):
    """A cooperative grid with more blocks than run at the same time is refused at the launch."""
    src, exe = tmp_path / "grid.cpp", str(tmp_path / "grid")
    src.write_text(INDEX_GRID)
    subprocess.run(["g++", "-std=c++17", f"-I{build.CSRC}", str(src), "-o", exe], check=True)
    cases = [(n, V, sms) for n in (1, 1000, 8192, 8193, 100000, 155648, 151553, 2 ** 31 - 1)
             for V in (1, 5000, 2 ** 18, 2 ** 18 + 1, 2 ** 31 - 1) for sms in (1, 7, 76, 148, 152, 200)]
    out = subprocess.run([exe], input="\n".join("%d %d %d" % c for c in cases), check=True,
                         capture_output=True, text=True).stdout.split("\n")
    for (n, V, sms), line in zip(cases, out):
        cluster, blocks, chunk = (int(v) for v in line.split())
        assert 1 <= blocks <= (8 if cluster else min(sms, 152)), (n, V, sms)
        assert blocks * chunk >= V and (not cluster or blocks in (1, 2, 4, 8))
        if sms >= 152 and not cluster:
            assert blocks == min(152, max(-(-n // 1024), -(-V // 4096)))


# ------------------------------------------------------------------ scratch of the cross entropy
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,D", [(1, 1000, 64), (16, 131072, 1024), (32, 5000, 100),
                                   (33, 5000, 100), (4096, 50000, 1024)])
def test_scratch_sizes_do_not_depend_on_what_else_is_asked(dtype, M, V, D):
    lib, cfg = binding.load(), binding.make_xent_config(M, V, D, dtype)
    size = [ctypes.c_size_t(0) for _ in range(4)]
    ask = lambda f, b: lib.dendsn_xent_workspace_size(ctypes.byref(cfg), f, b)
    assert ask(ctypes.byref(size[0]), ctypes.byref(size[1])) == 0
    assert ask(ctypes.byref(size[2]), None) == 0 and ask(None, ctypes.byref(size[3])) == 0
    assert size[0].value == size[2].value and size[1].value == size[3].value
    if dtype == "f32" and M <= 32:             # no copy of the weights
        assert size[0].value < V * D * 4


def test_scratch_without_a_copy_of_aligned_weights():
    """bfloat16 weights whose rows are read in place take no room in either pass."""
    M, V, D = 64, 100000, 1024
    free = binding.dendsn_xent_workspace_size(binding.make_xent_config(M, V, D, "bf16"))
    sure = binding.dendsn_xent_workspace_size(binding.make_xent_config(M, V, D, "bf16", weight_aligned=True))
    assert all(a - b >= V * D * 2 for a, b in zip(free, sure)) and sure[0] < V * D * 2 / 10
    for kw in (dict(dtype="f32", D=1024), dict(dtype="bf16", D=1023)):      # copied in any case
        a, b = (binding.dendsn_xent_workspace_size(binding.make_xent_config(M, V, weight_aligned=w, **kw))
                for w in (False, True))
        assert a == b
    cfg = binding.make_xent_config(4, 20, 8, "bf16")
    cfg.weight_aligned = 2
    assert test_abi_host.status_of(binding.dendsn_xent_workspace_size, cfg) == 1
    lib, P = binding.load(), ctypes.c_void_p
    ok, odd = P(4096), P(4104)
    x = ctypes.byref(binding.make_xent_config(4, 20, 8, "bf16", weight_aligned=True))
    assert lib.dendsn_xent_forward(x, ok, odd, ok, ok, ok, ok, None) == 3
    assert b"weight_aligned" in lib.dendsn_last_error()
    assert lib.dendsn_xent_backward(x, ok, odd, ok, ok, ok, ok, ok, ok, None) == 3


@pytest.mark.parametrize("offset,aligned", [(0, 1), (8, 1), (3, 0)])
def test_wrappers_ask_the_weights_address(offset, aligned, monkeypatch):
    Recorder(monkeypatch)
    cfg = binding.make_xent_config(4, 100, 64, "bf16")
    buf = torch.zeros(100 * 64 + 64, dtype=torch.bfloat16)
    first = (-buf.data_ptr() // 2) % 8 + offset
    w, h = buf[first:first + 6400].view(100, 64), torch.zeros(4, 64, dtype=torch.bfloat16)
    asked = []
    real = binding._xent_scratch
    monkeypatch.setattr(binding, "_xent_scratch", lambda c, b: asked.append(c.weight_aligned) or real(c, b))
    y, r = torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    binding.xent_forward(cfg, h, w, y)
    binding.xent_backward(cfg, h, w, y, r, r)
    assert asked == [aligned, aligned] and cfg.weight_aligned == 0
