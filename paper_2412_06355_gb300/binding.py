"""Thin ctypes binding of libdendsn (include/dendsn.h).

Argument marshalling only: every step of the DendSN forward and backward runs in
the library's CUDA kernels. torch supplies device memory and the current stream.
There is no fallback: if the library cannot be loaded, every call raises.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
import os
import threading
from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import build as _build

F32, BF16 = 0, 1
PSI_IDENTITY, PSI_MEXHAT = 0, 1
RESET_HARD, RESET_SOFT = 0, 1
SG_ATAN = 0

STATUS = {0: "ok", 1: "invalid argument", 2: "unsupported configuration",
          3: "misaligned pointer", 4: "CUDA error"}


class DendSNError(RuntimeError):
    def __init__(self, fn: str, status: int, msg: str):
        super().__init__(f"{fn}: {STATUS.get(status, status)}: {msg}")
        self.status = status


class dendsn_config(ctypes.Structure):
    """Mirror of the C struct dendsn_config."""
    _fields_ = [("T", ctypes.c_int32), ("B", ctypes.c_int32), ("N", ctypes.c_int32),
                ("K", ctypes.c_int32), ("G", ctypes.c_int32), ("C", ctypes.c_int32),
                ("inner", ctypes.c_int32), ("x_dtype", ctypes.c_int32),
                ("psi", ctypes.c_int32), ("reset", ctypes.c_int32),
                ("surrogate", ctypes.c_int32), ("theta", ctypes.c_float),
                ("beta", ctypes.c_float), ("detach_reset", ctypes.c_int32),
                ("mask_per_neuron", ctypes.c_int32), ("stateless", ctypes.c_int32),
                ("residual", ctypes.c_int32), ("layout", ctypes.c_int32)]

    @property
    def Kb(self) -> int:
        return self.K // self.G


LAYOUT_KINNER, LAYOUT_PAPER = 0, 1


def make_config(T, B, N, K, G=1, C=1, inner=1, dtype="f32", psi="mh", reset="hard",
                theta=1.0, beta=0.5, detach_reset=False, mask_per_neuron=False,
                stateless=False, residual=False, surrogate=SG_ATAN,
                layout="kinner") -> dendsn_config:
    return dendsn_config(T, B, N, K, G, C, inner, BF16 if dtype == "bf16" else F32,
                         PSI_MEXHAT if psi == "mh" else PSI_IDENTITY,
                         RESET_SOFT if reset == "soft" else RESET_HARD, surrogate,
                         float(theta), float(beta), int(detach_reset), int(mask_per_neuron),
                         int(stateless), int(residual),
                         LAYOUT_PAPER if layout == "paper" else LAYOUT_KINNER)


def config_of(w) -> dendsn_config:
    """Config of a workloads.Workload."""
    return make_config(w.T, w.B, w.N, w.K, w.G, w.C, w.inner, w.dtype, w.psi, w.reset,
                       w.theta, w.beta, w.detach_reset, w.mask_per_neuron, w.stateless,
                       w.residual, layout=w.layout)


I32, I64 = 0, 1
GATE_DECAY, GATE_LOGIT = 0, 1
MIX_PLAIN, MIX_COMPLEMENT = 0, 1
TIME_FIRST, BATCH_FIRST = 0, 1
LOGIT_GRAD_SPLIT, LOGIT_GRAD_BF16 = 0, 1
STATISTICS_LSE, STATISTICS_MAX_SUM = 0, 1


class dendsn_embed_config(ctypes.Structure):
    """Mirror of the C struct dendsn_embed_config."""
    _fields_ = [("n", ctypes.c_int64), ("padding_id", ctypes.c_int64), ("V", ctypes.c_int32),
                ("D", ctypes.c_int32), ("x_dtype", ctypes.c_int32),
                ("ids_dtype", ctypes.c_int32), ("scale", ctypes.c_float)]


class dendsn_scan_config(ctypes.Structure):
    """Mirror of the C struct dendsn_scan_config (the gated compartment scan)."""
    _fields_ = [("T", ctypes.c_int32), ("B", ctypes.c_int32), ("N", ctypes.c_int32),
                ("x_dtype", ctypes.c_int32), ("gate", ctypes.c_int32), ("mix", ctypes.c_int32),
                ("layout", ctypes.c_int32)]


class dendsn_xent_config(ctypes.Structure):
    """Mirror of the C struct dendsn_xent_config (cross entropy of a linear readout)."""
    _fields_ = [("ignore_index", ctypes.c_int64), ("M", ctypes.c_int32), ("V", ctypes.c_int32),
                ("D", ctypes.c_int32), ("x_dtype", ctypes.c_int32),
                ("labels_dtype", ctypes.c_int32), ("logit_grad", ctypes.c_int32),
                ("statistics", ctypes.c_int32), ("weight_aligned", ctypes.c_int32)]


def _code(what, value, codes):
    try:
        return codes[value]
    except KeyError:
        raise ValueError(f"{what} must be one of {sorted(codes)}, got {value!r}") from None


_DTYPES = {"f32": F32, "bf16": BF16}
_INDEX = {"i32": I32, "i64": I64}


_GATES = {"decay": GATE_DECAY, "logit": GATE_LOGIT}
_MIXES = {"plain": MIX_PLAIN, "complement": MIX_COMPLEMENT}
_SCAN_LAYOUTS = {"time": TIME_FIRST, "batch": BATCH_FIRST}
_LOGIT_GRADS = {"split": LOGIT_GRAD_SPLIT, "bf16": LOGIT_GRAD_BF16}
_STATISTICS = {"lse": STATISTICS_LSE, "max_sum": STATISTICS_MAX_SUM}


def make_embed_config(n, V, D, dtype="f32", scale=1.0, padding_id=None,
                      ids_dtype="i64") -> dendsn_embed_config:
    """padding_id: the token whose row is zero and has no gradient; None: there is none."""
    return dendsn_embed_config(n, -1 if padding_id is None else padding_id, V, D,
                               _code("dtype", dtype, _DTYPES),
                               _code("ids_dtype", ids_dtype, _INDEX), scale)


def make_scan_config(T, B, N, dtype="f32", gate="decay", mix="plain",
                     layout="time") -> dendsn_scan_config:
    return dendsn_scan_config(T, B, N, _code("dtype", dtype, _DTYPES), _code("gate", gate, _GATES),
                              _code("mix", mix, _MIXES), _code("layout", layout, _SCAN_LAYOUTS))


def make_xent_config(M, V, D, dtype="f32", ignore_index=-100,
                     labels_dtype="i64", logit_grad="split",
                     statistics="lse", weight_aligned=False) -> dendsn_xent_config:
    """logit_grad: how bfloat16 products take the logits' gradient, "split" in two terms or "bf16"
    rounded to one (faster; an error of up to 2^-8 of each). statistics: the rows that the forward
    leaves for the backward, "lse" [M] (rounded to float32) or "max_sum" [2, M], each row's largest
    logit and the sum relative to it, which keep the probabilities' precision. weight_aligned: the
    weight's address is a multiple of 16 bytes, so that scratch needs no room for a copy of it (the
    wrappers that allocate their scratch find out by themselves)."""
    return dendsn_xent_config(ignore_index, M, V, D, _code("dtype", dtype, _DTYPES),
                              _code("labels_dtype", labels_dtype, _INDEX),
                              _code("logit_grad", logit_grad, _LOGIT_GRADS),
                              _code("statistics", statistics, _STATISTICS), int(weight_aligned))


class dendsn_lif_config(ctypes.Structure):
    """Mirror of the C struct dendsn_lif_config (the point-neuron LIF layer)."""
    _fields_ = [("T", ctypes.c_int32), ("B", ctypes.c_int32), ("N", ctypes.c_int32),
                ("x_dtype", ctypes.c_int32), ("reset", ctypes.c_int32),
                ("theta", ctypes.c_float), ("beta", ctypes.c_float),
                ("detach_reset", ctypes.c_int32)]


def make_lif_config(T, B, N, dtype="f32", reset="hard", theta=1.0, beta=0.5,
                    detach_reset=False) -> dendsn_lif_config:
    return dendsn_lif_config(T, B, N, BF16 if dtype == "bf16" else F32,
                             RESET_SOFT if reset == "soft" else RESET_HARD, float(theta),
                             float(beta), int(detach_reset))


_lib = None
_lock = threading.Lock()


def library_path() -> str:
    return _build.LIB


def load() -> ctypes.CDLL:
    """Load libdendsn.so, building it first when it is missing or stale."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            path = _build.build()
            lib = ctypes.CDLL(path)
            P, cfgp = ctypes.c_void_p, ctypes.POINTER(dendsn_config)
            lib.dendsn_workspace_size.argtypes = [cfgp, ctypes.POINTER(ctypes.c_size_t),
                                                  ctypes.POINTER(ctypes.c_size_t)]
            lib.dendsn_forward.argtypes = [cfgp] + [P] * 10
            lib.dendsn_backward.argtypes = [cfgp] + [P] * 16
            lib.dendsn_backward_plif.argtypes = [cfgp] + [P] * 17
            lib.dendsn_backward_plif.restype = ctypes.c_int
            lcfgp = ctypes.POINTER(dendsn_lif_config)
            lib.dendsn_lif_workspace_size.argtypes = [lcfgp, ctypes.POINTER(ctypes.c_size_t)]
            lib.dendsn_lif_forward.argtypes = [lcfgp] + [P] * 5
            lib.dendsn_lif_backward.argtypes = [lcfgp] + [P] * 6
            for fn in (lib.dendsn_workspace_size, lib.dendsn_forward, lib.dendsn_backward,
                       lib.dendsn_lif_workspace_size, lib.dendsn_lif_forward,
                       lib.dendsn_lif_backward):
                fn.restype = ctypes.c_int
            for name, cfg_t, sizes, forward, backward in (
                    ("embed", dendsn_embed_config, 1, 4, 5), ("scan", dendsn_scan_config, 1, 8, 11),
                    ("xent", dendsn_xent_config, 2, 7, 9)):
                cp = ctypes.POINTER(cfg_t)
                for fn, args in (("workspace_size", [ctypes.POINTER(ctypes.c_size_t)] * sizes),
                                 ("forward", [P] * forward), ("backward", [P] * backward)):
                    f = getattr(lib, f"dendsn_{name}_{fn}")
                    f.argtypes = [cp] + args
                    f.restype = ctypes.c_int
            lib.dendsn_status_string.argtypes = [ctypes.c_int]
            lib.dendsn_status_string.restype = ctypes.c_char_p
            lib.dendsn_last_error.argtypes = []
            lib.dendsn_last_error.restype = ctypes.c_char_p
            lib.dendsn_launch_count.argtypes = []
            lib.dendsn_launch_count.restype = ctypes.c_uint64
            _lib = lib
    return _lib


def _check(fn: str, status: int):
    if status != 0:
        raise DendSNError(fn, status, load().dendsn_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("DendSN tensors must live on a CUDA device")
    if not t.is_contiguous():
        raise ValueError("DendSN tensors must be contiguous")
    return t.data_ptr()


# The current stream's handle without a Stream object around it (3 us less a call); the public
# way where torch does not offer it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _allocates(fn):
    """Decorates an allocating wrapper with a `stream` argument (a torch stream or a raw handle,
    None: the current one): its outputs and its scratch belong to that stream. Scratch given back on
    return is then handed out again behind the kernels that use it, which the current stream's
    memory would not be. The inputs have to be ready on the stream, and a caller who takes the
    outputs to another stream orders the two, as with any torch operator."""
    at = list(inspect.signature(fn).parameters).index("stream")

    @functools.wraps(fn)
    def wrapper(*args, **kw):
        stream = args[at] if len(args) > at else kw.get("stream")
        if stream is None:
            return fn(*args, **kw)
        if not hasattr(stream, "cuda_stream"):
            handle = int(stream)                  # 1 is the driver's other name of the default stream
            stream = torch.cuda.ExternalStream(0 if handle == 1 else handle)
        with torch.cuda.stream(stream):
            return fn(*args, **kw)
    return wrapper


def launch_count() -> int:
    """Kernels the library has enqueued since it was loaded."""
    return int(load().dendsn_launch_count())


def dendsn_workspace_size(cfg: dendsn_config):
    """(saved_bytes, scratch_bytes) for this config."""
    s, w = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check("dendsn_workspace_size",
           load().dendsn_workspace_size(ctypes.byref(cfg), ctypes.byref(s), ctypes.byref(w)))
    return int(s.value), int(w.value)


def _need(cfg, **tensors):
    """Refuses on the host any tensor smaller than what the config makes the kernels touch."""
    T, B, N, K, C, Kb = cfg.T, cfg.B, cfg.N, cfg.K, cfg.C, cfg.K // cfg.G
    sx = 2 if cfg.x_dtype == BF16 else 4
    elems = {"x": T * B * N * K * sx, "grad_x": T * B * N * K * sx,
             "spikes": T * B * N * sx, "grad_spikes": T * B * N * sx,
             "v_out": T * B * N * 4, "grad_v": T * B * N * 4,
             "alpha": C * K * 4, "xi": C * K * 4, "grad_alpha": C * K * 4, "grad_xi": C * K * 4,
             "zeta": C * Kb * 4, "kappa": C * Kb * 4, "grad_zeta": C * Kb * 4,
             "grad_kappa": C * Kb * 4, "mask": (N if cfg.mask_per_neuron else C) * Kb,
             "grad_beta": C * 4}
    sizes = None
    for name, t in tensors.items():
        if t is None:
            continue
        if name in ("saved", "scratch"):
            if sizes is None:
                sizes = dict(zip(("saved", "scratch"), dendsn_workspace_size(cfg)))
            need = sizes[name]
        else:
            need = elems[name]
        have = t.numel() * t.element_size()
        if have < need:
            raise ValueError(f"{name}: {have} bytes, the config needs {need}")


def dendsn_forward(cfg, x, alpha, xi, zeta, kappa, mask, spikes, v_out=None, saved=None,
                   stream=None):
    _need(cfg, x=x, alpha=alpha, xi=xi, zeta=zeta, kappa=kappa, mask=mask, spikes=spikes,
          v_out=v_out, saved=saved)
    _check("dendsn_forward", load().dendsn_forward(
        ctypes.byref(cfg), _ptr(x), _ptr(alpha), _ptr(xi), _ptr(zeta), _ptr(kappa),
        _ptr(mask), _ptr(spikes), _ptr(v_out), _ptr(saved), _stream(stream)))


def dendsn_backward(cfg, x, alpha, xi, zeta, kappa, mask, grad_spikes, grad_v, saved, grad_x,
                    grad_alpha, grad_xi, grad_zeta, grad_kappa, scratch, stream=None):
    _need(cfg, x=x, alpha=alpha, xi=xi, zeta=zeta, kappa=kappa, mask=mask,
          grad_spikes=grad_spikes, grad_v=grad_v, saved=saved, grad_x=grad_x,
          grad_alpha=grad_alpha, grad_xi=grad_xi, grad_zeta=grad_zeta, grad_kappa=grad_kappa,
          scratch=scratch)
    _check("dendsn_backward", load().dendsn_backward(
        ctypes.byref(cfg), _ptr(x), _ptr(alpha), _ptr(xi), _ptr(zeta), _ptr(kappa),
        _ptr(mask), _ptr(grad_spikes), _ptr(grad_v), _ptr(saved), _ptr(grad_x),
        _ptr(grad_alpha), _ptr(grad_xi), _ptr(grad_zeta), _ptr(grad_kappa), _ptr(scratch),
        _stream(stream)))


def dendsn_backward_plif(cfg, x, alpha, xi, zeta, kappa, mask, grad_spikes, grad_v, saved,
                         grad_x, grad_alpha, grad_xi, grad_zeta, grad_kappa, grad_beta, scratch,
                         stream=None):
    """dendsn_backward plus grad_beta [C], the gradient of a learnable somatic decay."""
    _need(cfg, x=x, alpha=alpha, xi=xi, zeta=zeta, kappa=kappa, mask=mask,
          grad_spikes=grad_spikes, grad_v=grad_v, saved=saved, grad_x=grad_x,
          grad_alpha=grad_alpha, grad_xi=grad_xi, grad_zeta=grad_zeta, grad_kappa=grad_kappa,
          grad_beta=grad_beta, scratch=scratch)
    _check("dendsn_backward_plif", load().dendsn_backward_plif(
        ctypes.byref(cfg), _ptr(x), _ptr(alpha), _ptr(xi), _ptr(zeta), _ptr(kappa),
        _ptr(mask), _ptr(grad_spikes), _ptr(grad_v), _ptr(saved), _ptr(grad_x),
        _ptr(grad_alpha), _ptr(grad_xi), _ptr(grad_zeta), _ptr(grad_kappa), _ptr(grad_beta),
        _ptr(scratch), _stream(stream)))


_noalloc_ready = False


def dendsn_backward_noalloc(cfg, x, alpha, xi, zeta, kappa, mask, grad_spikes, grad_v, saved,
                            grad_x, grad_alpha, grad_xi, grad_zeta, grad_kappa, stream=None):
    """dendsn_backward without a scratch buffer (the library's built-in 8 MiB one).

    For callers that cannot allocate device scratch memory per call; see the header
    for the sharing rules of the built-in buffer.
    """
    global _noalloc_ready
    _need(cfg, x=x, alpha=alpha, xi=xi, zeta=zeta, kappa=kappa, mask=mask,
          grad_spikes=grad_spikes, grad_v=grad_v, saved=saved, grad_x=grad_x,
          grad_alpha=grad_alpha, grad_xi=grad_xi, grad_zeta=grad_zeta, grad_kappa=grad_kappa)
    lib = load()
    if not _noalloc_ready:
        lib.dendsn_backward_noalloc.argtypes = [ctypes.POINTER(dendsn_config)] + \
            [ctypes.c_void_p] * 15
        lib.dendsn_backward_noalloc.restype = ctypes.c_int
        _noalloc_ready = True
    _check("dendsn_backward_noalloc", lib.dendsn_backward_noalloc(
        ctypes.byref(cfg), _ptr(x), _ptr(alpha), _ptr(xi), _ptr(zeta), _ptr(kappa),
        _ptr(mask), _ptr(grad_spikes), _ptr(grad_v), _ptr(saved), _ptr(grad_x),
        _ptr(grad_alpha), _ptr(grad_xi), _ptr(grad_zeta), _ptr(grad_kappa), _stream(stream)))


# ------------------------------------------------------------------ point-neuron LIF layer
def dendsn_lif_workspace_size(cfg: dendsn_lif_config) -> int:
    """saved_bytes of the LIF layer (checkpoints; 0 for T <= 8)."""
    s = ctypes.c_size_t(0)
    _check("dendsn_lif_workspace_size",
           load().dendsn_lif_workspace_size(ctypes.byref(cfg), ctypes.byref(s)))
    return int(s.value)


def _lif_need(cfg, **tensors):
    sx = 2 if cfg.x_dtype == BF16 else 4
    n = cfg.T * cfg.B * cfg.N
    for name, t in tensors.items():
        if t is None:
            continue
        need = (dendsn_lif_workspace_size(cfg) if name == "saved" else
                n * 4 if name in ("v_out", "grad_v") else n * sx)
        have = t.numel() * t.element_size()
        if have < need:
            raise ValueError(f"{name}: {have} bytes, the config needs {need}")


def dendsn_lif_forward(cfg, x, spikes, v_out=None, saved=None, stream=None):
    _lif_need(cfg, x=x, spikes=spikes, v_out=v_out, saved=saved)
    _check("dendsn_lif_forward", load().dendsn_lif_forward(
        ctypes.byref(cfg), _ptr(x), _ptr(spikes), _ptr(v_out), _ptr(saved), _stream(stream)))


def dendsn_lif_backward(cfg, x, grad_spikes, grad_v, saved, grad_x, stream=None):
    _lif_need(cfg, x=x, grad_spikes=grad_spikes, grad_v=grad_v, saved=saved, grad_x=grad_x)
    _check("dendsn_lif_backward", load().dendsn_lif_backward(
        ctypes.byref(cfg), _ptr(x), _ptr(grad_spikes), _ptr(grad_v), _ptr(saved),
        _ptr(grad_x), _stream(stream)))


@_allocates
def lif_forward(cfg, x, want_v=False, saved=None, stream=None):
    """Allocating LIF forward of x [T, B, N]. Returns (spikes, v or None)."""
    if tuple(x.shape) != (cfg.T, cfg.B, cfg.N) or x.dtype != _xdtype(cfg):
        raise ValueError(f"x must be {_xdtype(cfg)} [{cfg.T},{cfg.B},{cfg.N}]")
    spikes = torch.empty_like(x)
    v = torch.empty(x.shape, dtype=torch.float32, device=x.device) if want_v else None
    dendsn_lif_forward(cfg, x, spikes, v, saved, stream)
    return spikes, v


@_allocates
def lif_backward(cfg, x, grad_spikes, grad_v=None, saved=None, stream=None):
    """Allocating LIF backward. Returns dL/dX with x's shape and dtype."""
    gx = torch.empty_like(x)
    dendsn_lif_backward(cfg, x, grad_spikes, grad_v, saved, gx, stream)
    return gx


def lif_workspace(cfg, device=None):
    """The LIF checkpoint buffer, or None when T <= 8."""
    sb = dendsn_lif_workspace_size(cfg)
    return torch.empty(sb, dtype=torch.uint8, device=device or torch.device("cuda")) if sb else None


# ------------------------------------------------------------------ token-sequence operators
def _expect(shape, dtype, **tensors):
    """Refuses on the host tensors of another shape or dtype than the config's."""
    for name, t in tensors.items():
        if t is None:
            raise ValueError(f"{name} is required")
        if t.shape != shape or t.dtype is not dtype:
            raise ValueError(f"{name} must be {dtype} {list(shape)}, got {t.dtype} {list(t.shape)}")


def _pointers(*tensors):
    """Device addresses (None for None), checked as _ptr does."""
    return [None if t is None else t.data_ptr() if t.is_cuda and t.is_contiguous() else _ptr(t)
            for t in tensors]


def _idtype(code) -> torch.dtype:
    return torch.int64 if code == I64 else torch.int32


def _bytes(name, t, need):
    have = 0 if t is None else t.numel() * t.element_size()
    if have < need:
        raise ValueError(f"{name}: {have} bytes, the config needs {need}")


def _scratch(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def dendsn_embed_workspace_size(cfg: dendsn_embed_config) -> int:
    """scratch_bytes of the embedding's backward."""
    s = ctypes.c_size_t(0)
    _check("dendsn_embed_workspace_size",
           load().dendsn_embed_workspace_size(ctypes.byref(cfg), ctypes.byref(s)))
    return int(s.value)


def _expect_ids(cfg, ids):
    _expect(ids.shape if ids.numel() == cfg.n else (cfg.n,), _idtype(cfg.ids_dtype), ids=ids)


def dendsn_embed_forward(cfg, table, ids, out, stream=None):
    """out = scale * table[ids]; table [V, D], ids of n tokens (any shape), out n rows of D."""
    dt = _xdtype(cfg)
    _expect((cfg.V, cfg.D), dt, table=table)
    _expect_ids(cfg, ids)
    _expect((*ids.shape, cfg.D), dt, out=out)
    _check("dendsn_embed_forward", load().dendsn_embed_forward(
        ctypes.byref(cfg), *_pointers(table, ids, out), _stream(stream)))


def _embed_backward(cfg, ids, grad_out, grad_table, scratch, stream):
    dt = _xdtype(cfg)
    _expect_ids(cfg, ids)
    _expect((*ids.shape, cfg.D), dt, grad_out=grad_out)
    _expect((cfg.V, cfg.D), dt, grad_table=grad_table)
    _check("dendsn_embed_backward", load().dendsn_embed_backward(
        ctypes.byref(cfg), *_pointers(ids, grad_out, grad_table, scratch), _stream(stream)))


def dendsn_embed_backward(cfg, ids, grad_out, grad_table, scratch, stream=None):
    """grad_table [V, D] (overwritten) from grad_out, n rows of D."""
    _bytes("scratch", scratch, dendsn_embed_workspace_size(cfg))
    _embed_backward(cfg, ids, grad_out, grad_table, scratch, stream)


@_allocates
def embed_forward(cfg, table, ids, stream=None):
    """Allocating embedding: scale * table[ids], of shape [*ids.shape, D]."""
    out = torch.empty(tuple(ids.shape) + (cfg.D,), dtype=table.dtype, device=table.device)
    dendsn_embed_forward(cfg, table, ids, out, stream)
    return out


@_allocates
def embed_backward(cfg, ids, grad_out, scratch=None, stream=None):
    """Allocating gradient of the embedding table, [V, D] in grad_out's dtype."""
    need = dendsn_embed_workspace_size(cfg)
    if scratch is None:
        scratch = _scratch(need, ids.device)
    _bytes("scratch", scratch, need)
    gtable = torch.empty((cfg.V, cfg.D), dtype=grad_out.dtype, device=grad_out.device)
    _embed_backward(cfg, ids, grad_out, gtable, scratch, stream)
    return gtable


def dendsn_scan_workspace_size(cfg: dendsn_scan_config) -> int:
    """saved_bytes of the gated scan (states every 64 steps; 0 for T <= 64)."""
    s = ctypes.c_size_t(0)
    _check("dendsn_scan_workspace_size",
           load().dendsn_scan_workspace_size(ctypes.byref(cfg), ctypes.byref(s)))
    return int(s.value)


def _scan_expect(cfg, starts, states, **seq):
    lead = (cfg.B, cfg.T) if cfg.layout == BATCH_FIRST else (cfg.T, cfg.B)
    _expect((*lead, cfg.N), _xdtype(cfg), **seq)
    if starts is not None:
        _expect(lead, torch.uint8, starts=starts)
    _expect((cfg.B, cfg.N), torch.float32, **{k: t for k, t in states.items() if t is not None})


def dendsn_scan_forward(cfg, x, gate, starts, h0, h, h_last=None, saved=None, stream=None):
    _scan_expect(cfg, starts, dict(h0=h0, h_last=h_last), x=x, gate=gate, h=h)
    if saved is not None:
        _bytes("saved", saved, dendsn_scan_workspace_size(cfg))
    _check("dendsn_scan_forward", load().dendsn_scan_forward(
        ctypes.byref(cfg), *_pointers(x, gate, starts, h0, h, h_last, saved), _stream(stream)))


def dendsn_scan_backward(cfg, x, gate, starts, h0, grad_h, grad_last, saved, grad_x, grad_gate,
                         grad_h0=None, stream=None):
    _scan_expect(cfg, starts, dict(h0=h0, grad_last=grad_last, grad_h0=grad_h0), x=x, gate=gate,
                 grad_h=grad_h, grad_x=grad_x, grad_gate=grad_gate)
    _bytes("saved", saved, dendsn_scan_workspace_size(cfg))
    _check("dendsn_scan_backward", load().dendsn_scan_backward(
        ctypes.byref(cfg),
        *_pointers(x, gate, starts, h0, grad_h, grad_last, saved, grad_x, grad_gate, grad_h0),
        _stream(stream)))


def scan_workspace(cfg, device=None):
    """The gated scan's checkpoint buffer, or None when T <= 64."""
    return _scratch(dendsn_scan_workspace_size(cfg), device or torch.device("cuda"))


@_allocates
def scan_forward(cfg, x, gate, starts=None, h0=None, saved=None, want_last=False, stream=None):
    """Allocating gated scan. Returns (h, h_last or None); h_last [B, N] float32."""
    h = torch.empty_like(x)
    last = torch.empty((cfg.B, cfg.N), dtype=torch.float32, device=x.device) if want_last else None
    dendsn_scan_forward(cfg, x, gate, starts, h0, h, last, saved, stream)
    return h, last


@_allocates
def scan_backward(cfg, x, gate, grad_h, starts=None, h0=None, grad_last=None, saved=None,
                  stream=None):
    """Allocating backward of the gated scan. Returns dict gx, ggate, and gh0 where h0 is given."""
    out = dict(gx=torch.empty_like(x), ggate=torch.empty_like(gate))
    gh0 = None
    if h0 is not None:
        gh0 = out["gh0"] = torch.empty_like(h0)
    dendsn_scan_backward(cfg, x, gate, starts, h0, grad_h, grad_last, saved, out["gx"],
                         out["ggate"], gh0, stream)
    return out


def dendsn_xent_workspace_size(cfg: dendsn_xent_config):
    """(forward_bytes, backward_bytes) of scratch."""
    return _xent_scratch(cfg, False), _xent_scratch(cfg, True)


def _xent_scratch(cfg, backward) -> int:
    b = ctypes.c_size_t(0)
    where = (None, ctypes.byref(b)) if backward else (ctypes.byref(b), None)
    _check("dendsn_xent_workspace_size",
           load().dendsn_xent_workspace_size(ctypes.byref(cfg), *where))
    return b.value


def _for_weight(cfg, weight):
    """cfg with weight_aligned where that saves scratch and is so."""
    if cfg.x_dtype == BF16 and cfg.D % 8 == 0 and not cfg.weight_aligned and weight.data_ptr() % 16 == 0:
        cfg = dendsn_xent_config.from_buffer_copy(cfg)
        cfg.weight_aligned = 1
    return cfg


def _statistics_shape(cfg):
    return (2, cfg.M) if cfg.statistics == STATISTICS_MAX_SUM else (cfg.M,)


def _xent_expect(cfg, hidden, weight, labels, lse, **rows):
    dt = _xdtype(cfg)
    _expect(_statistics_shape(cfg), torch.float32, lse=lse)
    _expect((cfg.M, cfg.D), dt, hidden=hidden)
    _expect((cfg.V, cfg.D), dt, weight=weight)
    _expect((cfg.M,), _idtype(cfg.labels_dtype), labels=labels)
    _expect((cfg.M,), torch.float32, **rows)


def _xent_forward(cfg, hidden, weight, labels, loss, lse, scratch, stream):
    _xent_expect(cfg, hidden, weight, labels, loss=loss, lse=lse)
    _check("dendsn_xent_forward", load().dendsn_xent_forward(
        ctypes.byref(cfg), *_pointers(hidden, weight, labels, loss, lse, scratch),
        _stream(stream)))


def dendsn_xent_forward(cfg, hidden, weight, labels, loss, lse, scratch, stream=None):
    _xent_expect(cfg, hidden, weight, labels, loss=loss, lse=lse)
    _bytes("scratch", scratch, _xent_scratch(cfg, False))
    _xent_forward(cfg, hidden, weight, labels, loss, lse, scratch, stream)


def _xent_backward(cfg, hidden, weight, labels, lse, grad_loss, grad_hidden, grad_weight, scratch,
                   stream):
    _xent_expect(cfg, hidden, weight, labels, lse=lse, grad_loss=grad_loss)
    _expect((cfg.M, cfg.D), hidden.dtype, grad_hidden=grad_hidden)
    _expect((cfg.V, cfg.D), hidden.dtype, grad_weight=grad_weight)
    _check("dendsn_xent_backward", load().dendsn_xent_backward(
        ctypes.byref(cfg),
        *_pointers(hidden, weight, labels, lse, grad_loss, grad_hidden, grad_weight, scratch),
        _stream(stream)))


def dendsn_xent_backward(cfg, hidden, weight, labels, lse, grad_loss, grad_hidden, grad_weight,
                         scratch, stream=None):
    _xent_expect(cfg, hidden, weight, labels, lse=lse, grad_loss=grad_loss)
    _bytes("scratch", scratch, _xent_scratch(cfg, True))
    _xent_backward(cfg, hidden, weight, labels, lse, grad_loss, grad_hidden, grad_weight, scratch,
                   stream)


@_allocates
def xent_forward(cfg, hidden, weight, labels, scratch=None, stream=None):
    """Allocating cross entropy of hidden [M, D] read out by weight [V, D]: (loss [M], lse), lse
    [M] or, where the config's statistics are "max_sum", [2, M]."""
    if scratch is None:
        cfg = _for_weight(cfg, weight)
        scratch = _scratch(_xent_scratch(cfg, False), hidden.device)
    else:
        _bytes("scratch", scratch, _xent_scratch(cfg, False))
    loss = torch.empty((cfg.M,), dtype=torch.float32, device=hidden.device)
    lse = torch.empty(_statistics_shape(cfg), dtype=torch.float32, device=hidden.device)
    _xent_forward(cfg, hidden, weight, labels, loss, lse, scratch, stream)
    return loss, lse


@_allocates
def xent_backward(cfg, hidden, weight, labels, lse, grad_loss, scratch=None, stream=None):
    """Allocating backward. Returns dict ghidden [M, D], gweight [V, D] in hidden's dtype."""
    if scratch is None:
        cfg = _for_weight(cfg, weight)
        scratch = _scratch(_xent_scratch(cfg, True), hidden.device)
    else:
        _bytes("scratch", scratch, _xent_scratch(cfg, True))
    out = dict(ghidden=torch.empty_like(hidden), gweight=torch.empty_like(weight))
    _xent_backward(cfg, hidden, weight, labels, lse, grad_loss, out["ghidden"],
                         out["gweight"], scratch, stream)
    return out


# ------------------------------------------------------------------ tensor-level helpers
def _xdtype(cfg) -> torch.dtype:
    return torch.bfloat16 if cfg.x_dtype == BF16 else torch.float32


def _check_shapes(cfg, x, alpha, xi, zeta, kappa, mask):
    T, B, N, K, C, Kb = cfg.T, cfg.B, cfg.N, cfg.K, cfg.C, cfg.K // cfg.G
    if cfg.layout == LAYOUT_PAPER:
        # [T, B, N / inner, K, inner] in any contiguous shape with that element order
        if x.numel() != T * B * N * K or x.dtype != _xdtype(cfg) or x.dim() < 2 or \
                tuple(x.shape[:2]) != (T, B):
            raise ValueError(f"x must be {_xdtype(cfg)} [{T},{B},...] with {T * B * N * K} elements")
    elif tuple(x.shape) != (T, B, N, K) or x.dtype != _xdtype(cfg):
        raise ValueError(f"x must be {_xdtype(cfg)} [{T},{B},{N},{K}], got {x.dtype} {tuple(x.shape)}")
    for name, t, shp in (("alpha", alpha, (C, K)), ("xi", xi, (C, K)), ("zeta", zeta, (C, Kb)),
                         ("kappa", kappa, (C, Kb))):
        if tuple(t.shape) != shp or t.dtype != torch.float32:
            raise ValueError(f"{name} must be float32 {shp}, got {t.dtype} {tuple(t.shape)}")
    if mask is not None:
        rows = N if cfg.mask_per_neuron else C
        if tuple(mask.shape) != (rows, Kb) or mask.dtype != torch.uint8:
            raise ValueError(f"mask must be uint8 [{rows},{Kb}]")


def workspace(cfg, device=None):
    """Allocates (saved, scratch) byte buffers; None where zero bytes are needed."""
    sb, wb = dendsn_workspace_size(cfg)
    dev = device or torch.device("cuda")
    saved = torch.empty(sb, dtype=torch.uint8, device=dev) if sb else None
    scratch = torch.empty(max(wb, 16), dtype=torch.uint8, device=dev)
    return saved, scratch


@_allocates
def forward(cfg, x, alpha, xi, zeta, kappa, mask=None, want_v=False, saved=None, stream=None):
    """Allocating forward. Returns (spikes, v or None)."""
    _check_shapes(cfg, x, alpha, xi, zeta, kappa, mask)
    shape = (cfg.T, cfg.B, cfg.N)
    spikes = torch.empty(shape, dtype=x.dtype, device=x.device)
    v = torch.empty(shape, dtype=torch.float32, device=x.device) if want_v else None
    dendsn_forward(cfg, x, alpha, xi, zeta, kappa, mask, spikes, v, saved, stream)
    return spikes, v


@_allocates
def backward(cfg, x, alpha, xi, zeta, kappa, mask, grad_spikes, grad_v=None, saved=None,
             scratch=None, stream=None, want_beta=False):
    """Allocating backward. Returns dict gx, galpha, gxi, gzeta, gkappa, and with want_beta
    also gbeta (the gradient of a learnable somatic decay, per channel; computed by the
    separate dendsn_backward_plif kernel build)."""
    _check_shapes(cfg, x, alpha, xi, zeta, kappa, mask)
    if scratch is None:
        _, scratch = workspace(cfg, x.device)
    dev = x.device
    C, K, Kb = cfg.C, cfg.K, cfg.K // cfg.G
    out = dict(gx=torch.empty_like(x),
               galpha=torch.empty((C, K), dtype=torch.float32, device=dev),
               gxi=torch.empty((C, K), dtype=torch.float32, device=dev),
               gzeta=torch.empty((C, Kb), dtype=torch.float32, device=dev),
               gkappa=torch.empty((C, Kb), dtype=torch.float32, device=dev))
    grads = (out["gx"], out["galpha"], out["gxi"], out["gzeta"], out["gkappa"])
    if want_beta:
        out["gbeta"] = torch.empty((C,), dtype=torch.float32, device=dev)
        dendsn_backward_plif(cfg, x, alpha, xi, zeta, kappa, mask, grad_spikes, grad_v, saved,
                             *grads, out["gbeta"], scratch, stream)
    else:
        dendsn_backward(cfg, x, alpha, xi, zeta, kappa, mask, grad_spikes, grad_v, saved,
                        *grads, scratch, stream)
    return out


class DendSNFunction(torch.autograd.Function):
    """autograd wrapper: S = DendSN(X; alpha, xi, zeta, kappa[, beta]) (Eq. dendsn).

    alpha may be a scalar tensor (the paper's layer-wide decay) or [C, K]; its gradient is
    reduced to its own shape. The mask is a constant. beta: None (the somatic decay is
    cfg.beta, a constant) or a 0-dim tensor, a learnable decay (PLIF soma); its value
    replaces cfg.beta and its gradient is the sum of the per-channel dL/dbeta.
    """

    @staticmethod
    def forward(ctx, x, alpha, xi, zeta, kappa, mask, cfg, beta=None):
        if beta is not None:
            cfg = dendsn_config.from_buffer_copy(cfg)
            cfg.beta = float(beta)
        a = alpha.expand(cfg.C, cfg.K).contiguous().float()
        saved, scratch = workspace(cfg, x.device)
        s, _ = forward(cfg, x.contiguous(), a, xi.contiguous(), zeta.contiguous(),
                       kappa.contiguous(), mask, saved=saved)
        ctx.cfg = cfg
        ctx.alpha_shape = alpha.shape
        ctx.learn_beta = beta is not None
        ctx.ws = (saved, scratch)
        ctx.save_for_backward(x, a, xi, zeta, kappa, mask)
        return s

    @staticmethod
    @once_differentiable
    def backward(ctx, gs):
        x, a, xi, zeta, kappa, mask = ctx.saved_tensors
        saved, scratch = ctx.ws
        g = backward(ctx.cfg, x, a, xi, zeta, kappa, mask, gs.contiguous().to(x.dtype),
                     None, saved, scratch, want_beta=ctx.learn_beta)
        ga = g["galpha"].sum_to_size(ctx.alpha_shape)
        gb = g["gbeta"].sum() if ctx.learn_beta else None
        return g["gx"], ga, g["gxi"], g["gzeta"], g["gkappa"], None, None, gb


def _dtype_name(t) -> str:
    names = {torch.float32: "f32", torch.bfloat16: "bf16"}
    if t.dtype not in names:
        raise ValueError(f"dtype must be float32 or bfloat16, got {t.dtype}")
    return names[t.dtype]


def _index_name(t) -> str:
    names = {torch.int32: "i32", torch.int64: "i64"}
    if t.dtype not in names:
        raise ValueError(f"ids and labels must be int32 or int64, got {t.dtype}")
    return names[t.dtype]


class EmbedFunction(torch.autograd.Function):
    """autograd wrapper: scale * table[ids], with the gradient of the table."""

    @staticmethod
    def forward(ctx, table, ids, scale=1.0, padding_id=None):
        ids = ids.contiguous()
        ctx.cfg = make_embed_config(ids.numel(), *table.shape, _dtype_name(table), scale,
                                    padding_id, _index_name(ids))
        ctx.save_for_backward(ids)
        return embed_forward(ctx.cfg, table.contiguous(), ids)

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        ids, = ctx.saved_tensors
        return embed_backward(ctx.cfg, ids, g.contiguous()), None, None, None


class ScanFunction(torch.autograd.Function):
    """autograd wrapper of the gated compartment scan: (h, h_last) of x and gate, [T, B, N] or,
    with layout "batch", [B, T, N]. starts and h0 may be None."""

    @staticmethod
    def forward(ctx, x, gate, starts=None, h0=None, gate_kind="decay", mix="plain",
                layout="time"):
        x, gate = x.contiguous(), gate.contiguous()
        starts = None if starts is None else starts.contiguous()
        h0 = None if h0 is None else h0.contiguous()
        T, B = x.shape[:2] if layout == "time" else (x.shape[1], x.shape[0])
        ctx.cfg = make_scan_config(T, B, x.shape[2], _dtype_name(x), gate_kind, mix, layout)
        ctx.saved = scan_workspace(ctx.cfg, x.device)
        h, last = scan_forward(ctx.cfg, x, gate, starts, h0, ctx.saved, want_last=True)
        ctx.save_for_backward(x, gate, starts, h0)
        return h, last

    @staticmethod
    @once_differentiable
    def backward(ctx, gh, glast):
        x, gate, starts, h0 = ctx.saved_tensors
        g = scan_backward(ctx.cfg, x, gate, gh.contiguous(), starts, h0,
                          None if glast is None else glast.contiguous(), ctx.saved)
        return g["gx"], g["ggate"], None, g.get("gh0"), None, None, None


class XentFunction(torch.autograd.Function):
    """autograd wrapper: the row losses [M] of hidden [M, D] read out by weight [V, D].
    logit_grad as in make_xent_config."""

    @staticmethod
    def forward(ctx, hidden, weight, labels, ignore_index=-100, logit_grad="split"):
        hidden, weight, labels = hidden.contiguous(), weight.contiguous(), labels.contiguous()
        ctx.cfg = make_xent_config(hidden.shape[0], weight.shape[0], hidden.shape[1],
                                   _dtype_name(hidden), ignore_index, _index_name(labels),
                                   logit_grad, "max_sum" if any(ctx.needs_input_grad) else "lse")
        loss, lse = xent_forward(ctx.cfg, hidden, weight, labels)
        ctx.save_for_backward(hidden, weight, labels, lse)
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, gloss):
        hidden, weight, labels, lse = ctx.saved_tensors
        g = xent_backward(ctx.cfg, hidden, weight, labels, lse, gloss.float().contiguous())
        return g["ghidden"], g["gweight"], None, None, None
