"""The gated delta rule on the GPU against the recurrence in float64 (block_reference.py).

Tolerances. With keys of length up to 1, beta in [0, 1] and gates up to 0 a token's step does not lengthen
the state, so errors do not grow along a sequence. Each output is at the end of a chain of at most six
products (k S, the inverse, the state, q S, and the two of the gradient). Three terms leave 2^-24 of a
product. The matrix instruction adds 16 places at a time and cuts the sum off instead of rounding it: half
of 2^-23 on average, always toward zero, so the steps of a product add up: 4 U32 for 64 places, 8 U32 for
128. A state takes in k S (8), the inverse (4) and its own product (4): 16 U32; what is read from it (q S,
or the gradients' sums over v) another 8, the chunk's own square matrices 4 and what three terms leave 4:
32 U32 in norm for a chain. Element by element no value is off by more than 16 times its tensor's share of
that. Half a step more where the output is rounded to bfloat16; and the gradients of bfloat16 q and k come
of factors in two terms (2^-17 each, 2^-16 together).

A gate's gradient is, by definition of how it is formed, a difference of sums over the rest of its chunk:
<D, S'> + sum of (q . gq - v . gv). Each factor in it is off by CHAIN of its own norm, whatever the
difference comes to, so its bound counts the norms of what is summed (at T = 1 the terms are 100 times
their difference)."""
import pytest
import torch

import block_reference as ref
from block_reference import HALF_STEP, U32
from paper_2412_06355_gb300 import DeltaFunction, binding

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
CHAIN = 32 * U32


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def near(name, got, want, chain=CHAIN, summed=None):
    half = HALF_STEP[torch.bfloat16] if got.dtype == torch.bfloat16 else 0.0
    assert got.shape == want.shape, name
    err, want = (got.double() - want).abs(), want.abs()
    assert torch.isfinite(got.float()).all(), name
    norm = float((want if summed is None else want + summed).norm())
    assert float((err - half * want).clamp_min(0).norm()) <= chain * norm, (name, float(err.norm()) / max(norm, 1e-300))
    rms = norm / max(1, want.numel()) ** 0.5
    assert not (err > half * want + 16 * chain * (want + rms)).any(), (name, float(err.max()), rms)


def lead(layout, T, B):
    return {"time": (T, B), "batch": (B, T), "packed": (T,)}[layout]


class Case:
    def __init__(self, layout, T, B, Hk, Hv, Dk, Dv, dtype, lengths=None, behind=0, seed=0, decay=0.05):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 7 * Dk + Dv)
        n = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.layout, self.offsets = layout, None
        offs = None
        if layout == "packed":
            offs = [sum(lengths[:i]) for i in range(len(lengths) + 1)]
            B, T = len(lengths), offs[-1] + behind
            self.offsets = torch.tensor(offs, dtype=torch.int32, device="cuda")
        l = lead(layout, T, B)
        unit = lambda t: t / t.square().sum(-1, keepdim=True).sqrt().clamp_min(1e-6) * 0.999
        self.q, self.k = unit(n(*l, Hk, Dk)).to(DT[dtype]), unit(n(*l, Hk, Dk)).mul(0.99).to(DT[dtype])
        self.v, self.go = n(*l, Hv, Dv).to(DT[dtype]), n(*l, Hv, Dv).to(DT[dtype])
        self.gate, self.beta = -decay * torch.exp(n(*l, Hv)), torch.sigmoid(n(*l, Hv))
        self.s0, self.glast = n(B, Hv, Dk, Dv) * 0.5, n(B, Hv, Dk, Dv) * 0.1
        self.scale = Dk ** -0.5
        self.cfg = binding.make_delta_config(T, B, Hk, Hv, Dk, Dv, dtype, layout, self.scale)
        self.seqs = ref.sequences(layout, T, B, offs)
        self.used = torch.zeros(self.gate.numel() // Hv, dtype=torch.bool, device="cuda")
        self.summed = torch.zeros_like(self.gate)
        self.used[[t for s in self.seqs for t in s]] = True

    def inputs(self):
        return self.q, self.k, self.v, self.gate, self.beta

    def reference(self, grads=True, state=True):
        scale, marks = float(torch.tensor(self.scale)), []
        ins = [t.double().reshape(-1, *t.shape[-d:]) for t, d in zip(self.inputs(), (2, 2, 2, 1, 1))]
        ins.append(self.s0.double() if state else torch.zeros_like(self.s0).double())
        if grads:
            ins = [t.requires_grad_() for t in ins]
        rep = self.cfg.Hv // self.cfg.Hk
        heads = [t.repeat_interleave(rep, 1) for t in ins[:2]]
        o, last = ref.delta(*heads, *ins[2:], self.seqs, scale, marks if grads else None)
        out = {"o": o.detach().view(self.v.shape), "last": last.detach()}
        if grads:
            loss = (o * self.go.double().view_as(o)).sum() + (last * self.glast.double()).sum()
            g = torch.autograd.grad(loss, ins + heads[:1] + [S for _, S in marks], allow_unused=True)
            if self.seqs and marks:
                self.summed = self._summed(heads[0], ins[2], g[len(ins)], g[2], marks, g[len(ins) + 1:])
            for n, t, like in zip(("gq", "gk", "gv", "ggate", "gbeta", "gs0"), g, (*self.inputs(), self.s0)):
                out[n] = torch.zeros_like(like).double() if t is None else t.view(like.shape)
        return out

    def _summed(self, q, v, gq, gv, marks, gmarks):
        """Norms of what a gate's gradient is summed from, for every token and value head."""
        out = torch.zeros_like(v[..., 0])
        for (tokens, S), D in zip(marks, gmarks):
            each = q[tokens].norm(dim=-1) * gq[tokens].norm(dim=-1) + v[tokens].norm(dim=-1) * gv[tokens].norm(dim=-1)
            tail = S.flatten(1).norm(dim=1) * (0.0 if D is None else D.flatten(1).norm(dim=1))
            out[tokens] = each.flip(0).cumsum(0).flip(0) + tail
        return out.detach().view(self.gate.shape)

    def forward(self, **kw):
        return binding.delta_forward(self.cfg, *self.inputs(), self.offsets, self.s0, want_last=True, **kw)

    def both(self):
        saved = binding.delta_workspace(self.cfg)
        o, last = self.forward(saved=saved)
        g = binding.delta_backward(self.cfg, *self.inputs(), self.go, self.offsets, self.s0, self.glast, saved)
        return {"o": o, "last": last, **g}

    def check(self):
        got, want = self.both(), self.reference()
        two = 2.0 ** -16 if self.q.dtype == torch.bfloat16 else 0.0
        for n, t in got.items():
            near(n, t, want[n], CHAIN + two if n in ("gq", "gk") else CHAIN, self.summed if n == "ggate" else None)
        o, last = self.forward()                            # without what the backward needs
        near("o", o, want["o"])
        near("last", last, want["last"])
        again = self.both()
        assert all(torch.equal(got[n], again[n]) for n in got)
        return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["time", "batch"])
@pytest.mark.parametrize("T,B,Hk,Hv,Dk,Dv", [
    (1, 1, 1, 1, 1, 1), (2, 3, 1, 2, 8, 8), (9, 2, 2, 2, 33, 17), (63, 1, 1, 1, 64, 16), (64, 2, 1, 1, 16, 128),
    (65, 1, 2, 4, 65, 40), (129, 2, 1, 3, 128, 128), (200, 1, 1, 1, 40, 72), (191, 1, 1, 1, 127, 121), (70, 3, 3, 3, 7, 3)])
def test_delta(dtype, layout, T, B, Hk, Hv, Dk, Dv):
    Case(layout, T, B, Hk, Hv, Dk, Dv, dtype).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths,behind", [([0], 5), ([1], 0), ([64, 64], 0), ([63, 1, 0, 65], 3), ([0, 0, 130, 0], 0),
                                            ([1] * 40, 7), ([5, 100, 128, 2], 64)])
def test_packed(dtype, lengths, behind):
    c = Case("packed", 0, 0, 1, 2, 40, 24, dtype, lengths, behind)
    got = c.check()                                         # the allocating wrappers give zeros behind the last
    for n in ("o", "gq", "gk", "gv", "ggate", "gbeta"):
        assert not got[n][~c.used].any()


def test_tokens_of_no_sequence_keep_what_was_there():
    c = Case("packed", 0, 0, 1, 2, 16, 24, "bf16", [3, 70], 9)
    c.offsets += 4                                          # none before the first either
    c.offsets.clamp_(max=c.cfg.T)
    free = torch.ones(c.cfg.T, dtype=torch.bool, device="cuda")
    free[int(c.offsets[0]):int(c.offsets[-1])] = False
    assert int(free.sum()) == 9
    saved = binding.delta_workspace(c.cfg)
    scratch = torch.empty(binding.dendsn_delta_workspace_size(c.cfg)[2], dtype=torch.uint8, device="cuda")
    outs = [torch.full_like(t, 7.0) for t in (c.v, *c.inputs())]
    for rest, kept in (("keep", 7.0), ("zero", 0.0)):
        cfg = binding.make_delta_config(c.cfg.T, 2, 1, 2, 16, 24, "bf16", "packed", c.scale, rest)
        binding.dendsn_delta_forward(cfg, *c.inputs(), c.offsets, c.s0, outs[0], None, saved)
        binding.dendsn_delta_backward(cfg, c.go, c.offsets, c.glast, saved, *outs[1:], None, scratch)
        for t in outs:
            assert bool((t[free] == kept).all()) and bool((t[~free] != 7.0).any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,Hk,Hv,Dk,Dv", [(1, 1, 1, 1, 1, 1), (1, 5, 2, 4, 128, 128), (3, 2, 1, 2, 64, 32), (8, 1, 1, 1, 33, 127),
                                             (1, 300, 1, 2, 32, 64), (2, 2, 1, 1, 128, 5), (5, 1, 1, 1, 5, 100)])
def test_single_tokens_with_the_state_in_place(dtype, T, B, Hk, Hv, Dk, Dv):
    c = Case("batch", T, B, Hk, Hv, Dk, Dv, dtype)
    want, state = c.reference(grads=False), c.s0.clone()
    o, last = binding.delta_forward(c.cfg, *c.inputs(), s0=state, last=state)
    assert last is state
    near("o", o, want["o"])
    near("last", last, want["last"])


def test_tokens_one_by_one_and_in_chunks_agree():
    c = Case("batch", 150, 2, 1, 2, 64, 64, "f32")
    o, last = c.forward()
    state = c.s0.clone()
    one = binding.make_delta_config(1, 2, 1, 2, 64, 64, "f32", "batch", c.scale)
    rows = [binding.delta_forward(one, *(t[:, i:i + 1].contiguous() for t in c.inputs()), s0=state, last=state)[0] for i in range(150)]
    near("o", torch.cat(rows, 1), o.double(), 2 * CHAIN)
    near("last", state, last.double(), 2 * CHAIN)


def test_no_state_no_last_and_no_gradient_of_it():
    c = Case("time", 100, 2, 1, 1, 32, 48, "f32")
    want = c.reference(grads=False, state=False)
    saved = binding.delta_workspace(c.cfg)
    o, last = binding.delta_forward(c.cfg, *c.inputs(), saved=saved)
    assert last is None
    near("o", o, want["o"])
    g = binding.delta_backward(c.cfg, *c.inputs(), c.go, saved=saved)
    assert set(g) == {"gq", "gk", "gv", "ggate", "gbeta"}
    c.glast, c.s0 = torch.zeros_like(c.glast), torch.zeros_like(c.s0)
    want = c.reference()
    for n in g:
        near(n, g[n], want[n], 2 * CHAIN)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strong_decays(dtype):
    """Gates far below what float32's exponential has, and minus infinity: the state is forgotten."""
    c = Case("time", 140, 1, 1, 2, 24, 32, dtype)
    c.gate[3::7] = -1e4
    c.gate[5::11] = -float("inf")
    c.gate[70:75] = -150.0
    got = c.both()
    c.gate.clamp_(min=-700.0)                               # 0 in float64 too, where -inf has no gradient
    want = c.reference()
    for n in got:
        near(n, got[n], want[n], (2.0 ** -16 if dtype == "bf16" and n in ("gq", "gk") else 0) + 2 * CHAIN)
    assert not got["ggate"][5::11].any()


def test_no_writing_and_full_writing():
    c = Case("time", 130, 1, 1, 1, 16, 16, "f32")
    c.beta[::3] = 0.0                                       # the key writes nothing; its error still has a gradient
    c.beta[1::5] = 1.0
    c.check()


def test_growing_gates():
    c = Case("time", 130, 1, 1, 1, 32, 16, "f32", decay=-0.002)
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_misaligned_tensors(dtype):
    c = Case("batch", 130, 2, 1, 2, 64, 64, dtype)
    a = c.both()

    def moved(t):
        buf = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        v = buf[1:].view(t.shape)
        v.copy_(t)
        return v

    for n in ("q", "k", "v", "gate", "beta", "go", "s0", "glast"):
        setattr(c, n, moved(getattr(c, n)))
    b = c.both()
    assert all(torch.equal(a[n], b[n]) for n in a)
    c = Case("batch", 2, 2, 1, 2, 64, 64, dtype)
    a = c.forward()
    c.s0 = moved(c.s0)
    near("o", c.forward()[0], a[0].double(), 2 * CHAIN)


def test_a_bad_sequence_stays_alone():
    """A NaN reaches what comes after it, and (products take whole chunks of 64 tokens) its own chunk."""
    c = Case("packed", 0, 0, 1, 1, 32, 32, "f32", [100, 70, 90])
    a, v = c.both(), c.v.clone()
    alone = torch.ones(260, dtype=torch.bool, device="cuda")
    alone[100:170] = False
    for at in (130, 166):
        c.v = v.clone()
        c.v[at] = float("nan")
        b = c.both()
        for n in ("o", "gq", "gk", "gv", "ggate", "gbeta"):
            assert torch.equal(a[n][alone], b[n][alone])
        assert torch.isnan(b["o"][at:170]).all()
    assert torch.equal(a["o"][100:164], b["o"][100:164])    # the chunk before


def test_offsets_out_of_order_stay_within_the_buffers():
    """Results mean nothing then; what lies around the outputs stays (checked on the CPU: slots and rows of
    clamped offsets are below T // 64 + B and T)."""
    c = Case("packed", 0, 0, 1, 1, 16, 16, "f32", [100, 70, 90])
    for bad in ([0, 300, 20, 260], [-5, -7, 2 ** 31 - 1, 10], [260, 100, 0, 0]):
        c.offsets = torch.tensor(bad, dtype=torch.int32, device="cuda")
        pad = torch.full((3, 260, 16), 7.0, device="cuda")
        saved = binding.delta_workspace(c.cfg)
        binding.dendsn_delta_forward(c.cfg, *c.inputs(), c.offsets, c.s0, pad[1].view(260, 1, 16), None, saved)
        torch.cuda.synchronize()
        assert bool((pad[0] == 7).all()) and bool((pad[2] == 7).all())


def test_values_beyond_32_bits():
    """v and o have more than 2^31 elements; the last sequence gives the bits it gives alone."""
    T, B, H, Dk, Dv = 8192, 130, 16, 32, 128
    assert T * B * H * Dv > 2 ** 31
    one = Case("batch", T, 1, H, H, Dk, Dv, "bf16")
    o, last = one.forward()
    z = lambda t: torch.zeros(B, *t.shape[1:], dtype=t.dtype, device="cuda")
    many = [z(t) for t in (*one.inputs(), one.s0)]
    for t, x in zip(many, (*one.inputs(), one.s0)):
        t[-1:] = x
    cfg = binding.make_delta_config(T, B, H, H, Dk, Dv, "bf16", "batch", one.scale)
    all_o, all_last = binding.delta_forward(cfg, *many[:5], None, many[5], want_last=True)
    assert torch.equal(all_o[-1:], o) and torch.equal(all_last[-1:], last)
    assert not all_o[:2].any() and not all_last[:-1].any()


def test_empty():
    for T, B in ((0, 2), (5, 0)):
        cfg = binding.make_delta_config(T, B, 1, 2, 8, 4)
        z = lambda *s: torch.zeros(T, B, *s, device="cuda")
        s0 = torch.randn(B, 2, 8, 4, device="cuda")
        saved = binding.delta_workspace(cfg)
        o, last = binding.delta_forward(cfg, z(1, 8), z(1, 8), z(2, 4), z(2), z(2), None, s0, saved=saved, want_last=True)
        assert o.shape == (T, B, 2, 4) and torch.equal(last, s0)
        if saved is None:
            continue
        g = binding.delta_backward(cfg, z(1, 8), z(1, 8), z(2, 4), z(2), z(2), z(2, 4), None, s0, s0, saved)
        assert torch.equal(g["gs0"], s0)


def test_autograd_against_differences():
    c = Case("batch", 80, 1, 1, 2, 12, 20, "f32")
    leaves = [t.clone().requires_grad_() for t in (*c.inputs(), c.s0)]
    o, last = DeltaFunction.apply(*leaves[:5], leaves[5], None, c.scale, "batch")
    grads = torch.autograd.grad((o * c.go).sum() + (last * c.glast).sum(), leaves)
    flat = lambda ts: [t.double().reshape(-1, *t.shape[-d:]) for t, d in zip(ts[:5], (2, 2, 2, 1, 1))] + [ts[5].double()]

    def loss(ts):
        o, last = ref.delta(*ts, c.seqs, float(torch.tensor(c.scale)))
        return float((o * c.go.double().view_as(o)).sum() + (last * c.glast.double()).sum())

    at = flat([t.detach() for t in leaves])
    torch.manual_seed(1)
    for i, g in enumerate(flat(grads)):
        d = torch.randn_like(at[i])
        d /= d.norm()
        plus, minus = list(at), list(at)
        plus[i], minus[i] = at[i] + 1e-5 * d, at[i] - 1e-5 * d
        slope = (loss(plus) - loss(minus)) / 2e-5
        assert abs(slope - float((g * d).sum())) < 2 * CHAIN * float(g.norm()) + 1e-7 * (1 + abs(slope)), i


def test_autograd_when_nothing_reaches_an_output():
    c = Case("packed", 0, 0, 1, 1, 8, 8, "f32", [5, 70], 2)
    leaves = [t.clone().requires_grad_() for t in c.inputs()]
    _, last = DeltaFunction.apply(*leaves, None, c.offsets, c.scale, "packed")
    g = torch.autograd.grad((last * c.glast).sum(), leaves)
    assert not g[0].any() and not g[1][75:].any() and torch.isfinite(g[1]).all()
    o, _ = DeltaFunction.apply(*leaves, None, c.offsets, c.scale, "packed")
    assert torch.autograd.grad(o.sum(), leaves)[2][:75].any()
