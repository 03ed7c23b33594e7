"""The token-sequence operators on the GPU against float64 references (seq_reference.py):
embedding, gated compartment scan, cross entropy of a linear readout. The tolerances are
first-order bounds of a float32 evaluation, element by element."""
import math

import pytest
import torch

import seq_reference as ref
from paper_2412_06355_gb300 import (EmbedFunction, ScanFunction, XentFunction, binding)
from seq_reference import check

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def offset_copy(t, k):
    """The same values k elements into a buffer: a pointer without the wide alignment."""
    buf = torch.empty(t.numel() + k, dtype=t.dtype, device=t.device)
    v = buf[k:].view(t.shape)
    v.copy_(t)
    return v


# ------------------------------------------------------------------ embedding
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,V,D", [(1, 1, 1), (1, 1000, 384), (7, 5, 3), (64, 32768, 384),
                                   (1000, 50, 251), (4097, 4096, 64), (5000, 300, 8),
                                   (33000, 2, 16), (20000, 70000, 40)])
def test_embed(dtype, n, V, D):
    g = gen(n + V + D)
    table = randn((V, D), g, DT[dtype])
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    ids[::5] = int(ids[0])                               # a frequent token
    grad = randn((n, D), g, DT[dtype])
    for idt, pad, scale in (("i64", None, 1.0), ("i32", int(ids[0]), math.sqrt(D))):
        i = ids if idt == "i64" else ids.int()
        cfg = binding.make_embed_config(n, V, D, dtype, scale, pad, idt)
        out = binding.embed_forward(cfg, table, i)
        want = table[ids].float() * torch.tensor(scale, device="cuda")
        if pad is not None:
            want[ids == pad] = 0
        assert torch.equal(out, want.to(DT[dtype]))
        gt = binding.embed_backward(cfg, i, grad)
        check("gtable", gt, ref.embed_backward(ids, grad, V, torch.tensor(scale).item(), pad))
        again = binding.embed_backward(cfg, i, grad)
        assert torch.equal(gt, again)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_embed_one_token_everywhere_and_misaligned(dtype):
    n, V, D = 9001, 777, 96
    g = gen(3)
    ids = torch.full((n,), 700, device="cuda")
    grad = offset_copy(randn((n, D), g, DT[dtype]), 1)
    table = offset_copy(randn((V, D), g, DT[dtype]), 1)
    cfg = binding.make_embed_config(n, V, D, dtype, 0.5)
    assert torch.equal(binding.embed_forward(cfg, table, ids), (table[ids].float() * 0.5).to(DT[dtype]))
    check("gtable", binding.embed_backward(cfg, ids, grad), ref.embed_backward(ids, grad, V, 0.5, None))


def test_embed_tokens_outside_the_vocabulary():
    V, D = 10, 12
    ids = torch.tensor([3, -1, 10, 3, 2 ** 40, -2 ** 40, 9], device="cuda")
    g = gen(5)
    table, grad = randn((V, D), g), randn((7, D), g)
    cfg = binding.make_embed_config(7, V, D)
    out = binding.embed_forward(cfg, table, ids)
    bad = torch.tensor([False, True, True, False, True, True, False], device="cuda")
    assert torch.isnan(out[bad]).all() and torch.equal(out[~bad], table[ids[~bad]])
    check("gtable", binding.embed_backward(cfg, ids, grad), ref.embed_backward(ids, grad, V, 1.0, None))


def test_embed_nan_of_a_padded_token_stays_out():
    ids = torch.tensor([1, 0, 2, 0], device="cuda")
    grad = torch.ones(4, 8, device="cuda")
    grad[1] = float("nan")
    grad[3] = float("inf")
    cfg = binding.make_embed_config(4, 3, 8, padding_id=0)
    gt = binding.embed_backward(cfg, ids, grad)
    assert torch.equal(gt, torch.tensor([0.0, 1.0, 1.0], device="cuda").unsqueeze(1).expand(3, 8))


def test_embed_empty_and_shapes():
    cfg = binding.make_embed_config(0, 5, 4)
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    table = torch.ones(5, 4, device="cuda")
    assert binding.embed_forward(cfg, table, ids).shape == (0, 4)
    assert torch.count_nonzero(binding.embed_backward(cfg, ids, torch.empty(0, 4, device="cuda"))) == 0
    ids = torch.tensor([[0, 1], [2, 3], [4, 4]], device="cuda")
    cfg = binding.make_embed_config(6, 5, 4)
    assert binding.embed_forward(cfg, table, ids).shape == (3, 2, 4)


def test_embed_offsets_beyond_32_bits():
    n, V, D = 1100000, 3, 2048                            # n * D > 2^31
    g = gen(8)
    table = randn((V, D), g, torch.bfloat16)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    cfg = binding.make_embed_config(n, V, D, "bf16", ids_dtype="i32")
    out = binding.embed_forward(cfg, table, ids)
    tail = slice(n - 1000, n)
    assert torch.equal(out[tail], table[ids[tail].long()])
    gt = binding.embed_backward(cfg, ids, out)
    count = torch.bincount(ids, minlength=V).double()
    want = (count.unsqueeze(1) * table.double())
    bound = (2 * count.unsqueeze(1) * ref.U32 + ref.U16) * want.abs()
    check("gtable", gt, (want, bound))


# ------------------------------------------------------------------ gated scan
def scan_inputs(T, B, N, dtype, kind, layout, starts, seed):
    g = gen(seed)
    shape = (T, B, N) if layout == "time" else (B, T, N)
    x, gh = randn(shape, g, DT[dtype]), randn(shape, g, DT[dtype])
    gate = (torch.randn(shape, generator=g, device="cuda") + 2 if kind == "logit"
            else torch.rand(shape, generator=g, device="cuda")).to(DT[dtype])
    h0, glast = randn((B, N), g), randn((B, N), g)
    st = None
    if starts:
        st = (torch.rand(shape[:2], generator=g, device="cuda") < starts).to(torch.uint8) * 3
    return x, gate, st, h0, gh, glast


def run_scan(T, B, N, dtype="f32", kind="decay", mix="plain", layout="time", starts=0.0, seed=0,
             with_state=True, offset=0):
    x, gate, st, h0, gh, glast = scan_inputs(T, B, N, dtype, kind, layout, starts, seed)
    if not with_state:
        h0 = glast = None
    if offset:
        x, gate, gh = (offset_copy(t, offset) for t in (x, gate, gh))
    cfg = binding.make_scan_config(T, B, N, dtype, kind, mix, layout)
    saved = binding.scan_workspace(cfg)
    h, last = binding.scan_forward(cfg, x, gate, st, h0, saved, want_last=True)
    got = dict(h=h, last=last)
    got.update(binding.scan_backward(cfg, x, gate, gh, st, h0, glast, saved))
    want = ref.scan(x, gate, st, h0, gh, glast, kind, mix, layout)
    for k in got:
        check(k, got[k], want[k])
    # an evaluation without checkpoints gives the same bits, and so does a second backward
    h2, last2 = binding.scan_forward(cfg, x, gate, st, h0, None, want_last=True)
    assert torch.equal(h, h2) and torch.equal(last, last2)
    g2 = binding.scan_backward(cfg, x, gate, gh, st, h0, glast, saved)
    for k in g2:
        assert torch.equal(g2[k], got[k]), k


@pytest.mark.parametrize("layout", ["time", "batch"])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 63, 64, 65, 127, 128, 129, 200, 511, 513, 1000, 4099])
def test_scan_lengths(T, layout):
    run_scan(T, 2, 40, "f32", "logit", "complement", layout, 0.02, seed=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["decay", "logit"])
@pytest.mark.parametrize("mix", ["plain", "complement"])
@pytest.mark.parametrize("B,N", [(1, 1), (3, 33), (2, 128), (5, 1001), (1, 4096)])
def test_scan_forms(dtype, kind, mix, B, N):
    run_scan(150, B, N, dtype, kind, mix, "time", 0.03, seed=N)
    run_scan(75, B, N, dtype, kind, mix, "batch", 0.0, seed=N, with_state=False)


@pytest.mark.parametrize("T,B,N", [(300, 1, 8), (2500, 1, 64), (16384, 1, 24), (3, 700, 36),
                                   (1, 64, 4096), (70, 40, 1024)])
def test_scan_shapes(T, B, N):
    run_scan(T, B, N, "bf16", "logit", "complement", "time", 0.01, seed=T)
    run_scan(T, B, N, "f32", "decay", "plain", "batch", 0.5, seed=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [1, 2, 4])
def test_scan_misaligned_views(dtype, offset):
    run_scan(90, 2, 256, dtype, "logit", "complement", "time", 0.02, offset=offset)


def test_scan_every_step_starts():
    run_scan(100, 2, 64, "f32", "logit", "complement", "time", 1.1)


@pytest.mark.parametrize("T", [5, 100, 700])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_scan_start_cuts_what_is_not_finite(T, value):
    """Steps after a start are those of a scan that begins there, whatever came before."""
    B, N, cut = 2, 40, T // 2
    x, gate, _, h0, gh, glast = scan_inputs(T, B, N, "f32", "logit", "time", 0, 4)
    st = torch.zeros(T, B, dtype=torch.uint8, device="cuda")
    st[cut] = 1
    xb, hb = x.clone(), torch.full_like(h0, value)
    xb[:cut] = value
    cfg = binding.make_scan_config(T, B, N, "f32", "logit", "complement")
    saved = binding.scan_workspace(cfg)
    h, last = binding.scan_forward(cfg, xb, gate, st, hb, saved, want_last=True)
    want = ref.scan(x, gate, st, h0, gh, glast, "logit", "complement", "time")
    check("h", h[cut:], tuple(w[cut:] for w in want["h"]))
    check("last", last, want["last"])
    # and gradients after it that are not finite do not pass back over it
    ghb = gh.clone()
    ghb[cut:] = value
    saved = binding.scan_workspace(cfg)
    binding.scan_forward(cfg, x, gate, st, h0, saved)
    g = binding.scan_backward(cfg, x, gate, ghb, st, h0, torch.full_like(glast, value), saved)
    for k in ("gx", "ggate"):
        check(k, g[k][:cut], tuple(w[:cut] for w in want[k]))
    check("gh0", g["gh0"], want["gh0"])


def test_scan_decays_of_zero_one_and_saturated_gates():
    T, B, N = 130, 1, 64
    g = gen(11)
    x, gh = randn((T, B, N), g), randn((T, B, N), g)
    gate = torch.randint(0, 2, (T, B, N), generator=g, device="cuda").float()
    cfg = binding.make_scan_config(T, B, N)
    saved = binding.scan_workspace(cfg)
    h, _ = binding.scan_forward(cfg, x, gate, saved=saved)
    got = binding.scan_backward(cfg, x, gate, gh, saved=saved)
    want = ref.scan(x, gate, None, None, gh, None, "decay", "plain", "time")
    check("h", h, want["h"])
    check("gx", got["gx"], want["gx"])
    check("ggate", got["ggate"], want["ggate"])
    cfg = binding.make_scan_config(T, B, N, gate="logit", mix="complement")
    gate = (gate * 2 - 1) * 200.0                         # exp overflows on one side
    h, _ = binding.scan_forward(cfg, x, gate, saved=saved)
    got = binding.scan_backward(cfg, x, gate, gh, saved=saved)
    want = ref.scan(x, gate, None, None, gh, None, "logit", "complement", "time")
    check("h", h, want["h"])
    check("gx", got["gx"], want["gx"])
    assert torch.isfinite(got["ggate"]).all()


@pytest.mark.parametrize("B,N", [(2, 64), (3, 17)])
def test_scan_serving_steps_in_place(B, N):
    """T single steps with the state updated in place equal one scan over T."""
    T = 37
    x, gate, _, h0, _, _ = scan_inputs(T, B, N, "f32", "logit", "time", 0, 9)
    whole = ref.scan(x, gate, None, h0, None, None, "logit", "plain", "time")
    cfg = binding.make_scan_config(1, B, N, gate="logit")
    state = h0.clone()
    for t in range(T):
        h = torch.empty_like(x[t:t + 1])
        binding.dendsn_scan_forward(cfg, x[t:t + 1], gate[t:t + 1], None, state, h, state)
        check("h", h[0], tuple(w[t] for w in whole["h"]))
    check("last", state, whole["last"])


def test_scan_long_sequence_with_the_state_in_place():
    """h_last over h0 where several blocks share the sequence."""
    T, B, N = 3000, 1, 32
    x, gate, _, h0, _, _ = scan_inputs(T, B, N, "f32", "logit", "time", 0, 10)
    gate += 6.0                                           # decays near 1: h0 reaches far
    cfg = binding.make_scan_config(T, B, N, gate="logit", mix="complement")
    h, last = binding.scan_forward(cfg, x, gate, None, h0, want_last=True)
    state, h2 = h0.clone(), torch.empty_like(h)
    binding.dendsn_scan_forward(cfg, x, gate, None, state, h2, state)
    assert torch.equal(h, h2) and torch.equal(state, last)


def test_scan_empty():
    h0, glast = torch.ones(2, 3, device="cuda"), torch.full((2, 3), 2.0, device="cuda")
    cfg = binding.make_scan_config(0, 2, 3)
    e = torch.empty(0, 2, 3, device="cuda")
    _, last = binding.scan_forward(cfg, e, e, None, h0, want_last=True)
    assert torch.equal(last, h0)
    assert torch.equal(binding.scan_forward(cfg, e, e, want_last=True)[1], torch.zeros_like(h0))
    assert torch.equal(binding.scan_backward(cfg, e, e, e, None, h0, glast)["gh0"], glast)
    cfg = binding.make_scan_config(4, 0, 3)
    e = torch.empty(4, 0, 3, device="cuda")
    assert binding.scan_forward(cfg, e, e)[0].numel() == 0


def test_scan_offsets_beyond_32_bits():
    T, N = 2 ** 19 + 3, 4100                             # T * N > 2^31
    dt = torch.bfloat16
    x = torch.zeros(T, 1, N, dtype=dt, device="cuda")
    gate = torch.full((T, 1, N), 0.5, dtype=dt, device="cuda")
    tail = 40
    g = gen(2)
    x[-tail:] = randn((tail, 1, N), g, dt)
    cfg = binding.make_scan_config(T, 1, N, "bf16")
    saved = binding.scan_workspace(cfg)
    h, last = binding.scan_forward(cfg, x, gate, saved=saved, want_last=True)
    gh = torch.zeros_like(x)
    gh[-tail:] = randn((tail, 1, N), g, dt)
    got = binding.scan_backward(cfg, x, gate, gh, saved=saved)
    want = ref.scan(x[-tail:], gate[-tail:], None, None, gh[-tail:], None, "decay", "plain", "time")
    check("h", h[-tail:], want["h"])
    check("last", last, want["last"])
    for k in ("gx", "ggate"):
        check(k, got[k][-tail:], want[k])
    assert torch.count_nonzero(h[:-tail]) == 0


def test_scan_rows_far_apart():
    """So many channels that a block's steps lie more than 4 GB apart."""
    M, T = 2 ** 28 + 64, 2
    x = torch.empty(T, 1, M, device="cuda")
    gate = torch.empty_like(x)
    ends = [slice(0, 5000), slice(M - 5000, M)]
    x.fill_(0.5)
    gate.fill_(0.25)
    g = gen(12)
    for e in ends:
        x[..., e], gate[..., e] = randn((T, 1, 5000), g), randn((T, 1, 5000), g)
    cfg = binding.make_scan_config(T, 1, M, "f32", "logit", "complement")
    st = torch.tensor([[0], [1]], dtype=torch.uint8, device="cuda")
    for starts in (None, st):
        h, last = binding.scan_forward(cfg, x, gate, starts, want_last=True)
        got = dict(h=h, last=last)
        got.update(binding.scan_backward(cfg, x, gate, x, starts))
        for e in ends:
            want = ref.scan(x[..., e], gate[..., e], starts, None, x[..., e], None, "logit", "complement", "time")
            for k in got:
                check(k, got[k][..., e], want[k])
        del h, last, got


def test_scan_samples_far_apart():
    """Samples more than 4 GB apart: constant inputs against the recurrence's fixed points."""
    B, T, N = 2, 270000, 4096
    x = torch.full((B, T, N), 0.5, device="cuda")         # h -> 0.5 h + 0.5
    cfg = binding.make_scan_config(T, B, N, layout="batch")
    saved = binding.scan_workspace(cfg)
    h, last = binding.scan_forward(cfg, x, x, saved=saved, want_last=True)
    k = torch.arange(1, 41, dtype=torch.float64, device="cuda")
    first = 1 - 0.5 ** k
    for b in range(B):
        assert torch.equal(h[b, :40].double(), first.unsqueeze(1).expand(40, N).float().double())
        assert bool((h[b, -100:] == 1).all())
    assert bool((last == 1).all())
    got = binding.scan_backward(cfg, x, x, x, saved=saved)
    for b in range(B):                                    # lambda as h, from the end
        assert torch.equal(got["gx"][b, -40:].flip(0).double(), first.unsqueeze(1).expand(40, N).float().double())
        assert bool((got["gx"][b, :100] == 1).all())
        assert bool((got["ggate"][b, 100:-100] == 1).all())


# ------------------------------------------------------------------ cross entropy
def xent_inputs(M, V, D, dtype, seed, ignored=0.2, spread=2.0):
    g = gen(seed)
    H = randn((M, D), g, DT[dtype])
    W = (torch.randn((V, D), generator=g, device="cuda") * (spread / math.sqrt(D))).to(DT[dtype])
    y = torch.randint(0, V, (M,), generator=g, device="cuda")
    y[torch.rand(M, generator=g, device="cuda") < ignored] = -100
    c = torch.rand(M, generator=g, device="cuda") + 0.5
    return H, W, y, c


def run_xent(H, W, y, c, dtype, ignore=-100, norm=True):
    M, D = H.shape
    cfg = binding.make_xent_config(M, W.shape[0], D, dtype, ignore,
                                   "i64" if y.dtype == torch.int64 else "i32")
    loss, lse = binding.xent_forward(cfg, H, W, y)
    got = dict(loss=loss)
    got.update(binding.xent_backward(cfg, H, W, y, lse, c))
    want = ref.xent(H, W, y, ignore, c)
    for k in got:
        check(k, got[k], want[k])
        if norm and k != "loss" and bool(torch.isfinite(want[k][0]).all()):
            # rounding G and the output to bfloat16 are two independent errors of U16 / sqrt(3)
            # on average each; float32 carries about sqrt(depth) roundings
            r, scale = want[k][0], want[k][0].norm()
            if scale > 0:
                assert float((got[k].double() - r).norm() / scale) < (4e-3 if dtype == "bf16" else 3e-6), k
    loss2, lse2 = binding.xent_forward(cfg, H, W, y)
    g2 = binding.xent_backward(cfg, H, W, y, lse, c)
    same = lambda a, b: torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))
    assert same(loss, loss2) and same(lse, lse2)
    for k in g2:
        assert same(g2[k], got[k]), k
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,D", [(1, 1, 1), (1, 1000, 64), (2, 3, 5), (16, 4099, 384),
                                   (63, 257, 72), (127, 128, 128), (128, 256, 64),
                                   (129, 1001, 33), (257, 513, 200), (300, 5000, 520),
                                   (1000, 777, 65), (700, 20001, 96), (640, 12288, 264)])
def test_xent(dtype, M, V, D):
    run_xent(*xent_inputs(M, V, D, dtype, M + V + D), dtype)


@pytest.mark.parametrize("M", [1, 5, 15, 16, 17, 40, 63, 64, 65])
@pytest.mark.parametrize("V,D", [(1, 4), (64, 32), (65, 31), (1000, 100), (4097, 33), (300, 2048)])
def test_xent_few_float32_rows(M, V, D):
    run_xent(*xent_inputs(M, V, D, "f32", M + V + D, ignored=0.2 if M > 1 else 0.0), "f32")


def test_xent_few_float32_rows_ignored_and_out_of_range():
    H, W, y, c = xent_inputs(50, 301, 40, "f32", 11, ignored=0.5)
    H[y == -100] = float("inf")
    y[7] = 301
    run_xent(offset_copy(H, 1), W, y, c, "f32")
    y[:] = -100
    run_xent(H, W, y.int(), c, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_xent_label_types_and_ignore_index(dtype):
    H, W, y, c = xent_inputs(150, 301, 48, dtype, 1, ignored=0.0)
    a = run_xent(H, W, y, c, dtype, ignore=7)
    b = run_xent(H, W, y.int(), c, dtype, ignore=7)
    for k in a:
        assert torch.equal(a[k], b[k])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), torch.finfo(torch.bfloat16).min])
def test_xent_ignored_rows_are_left_out_whatever_they_hold(dtype, value):
    H, W, y, c = xent_inputs(200, 400, 72, dtype, 2, ignored=0.3)
    H[y == -100] = value
    c[y == -100] = float("nan")
    run_xent(H, W, y, c, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_xent_all_rows_ignored(dtype):
    H, W, y, c = xent_inputs(140, 300, 40, dtype, 3)
    y[:] = -100
    got = run_xent(H, W, y, c, dtype)
    for v in got.values():
        assert torch.count_nonzero(v) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_xent_labels_outside_the_vocabulary(dtype):
    H, W, y, c = xent_inputs(140, 300, 40, dtype, 4)
    y[3], y[77], y[139] = 300, -1, 2 ** 35
    got = run_xent(H, W, y, c, dtype)
    assert torch.isnan(got["loss"][[3, 77, 139]]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_xent_no_rows(dtype):
    H, W, y, c = xent_inputs(0, 300, 40, dtype, 5)
    cfg = binding.make_xent_config(0, 300, 40, dtype)
    loss, lse = binding.xent_forward(cfg, H, W, y)
    g = binding.xent_backward(cfg, H, W, y, lse, c)
    assert loss.numel() == 0 and torch.count_nonzero(g["gweight"]) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("spread", [0.0, 60.0, 2000.0])
def test_xent_flat_and_steep_logits(dtype, spread):
    H, W, y, c = xent_inputs(130, 600, 64, dtype, 6, spread=spread)
    run_xent(H, W, y, c, dtype, norm=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_xent_misaligned_operands(dtype):
    H, W, y, c = xent_inputs(130, 600, 64, dtype, 7)
    run_xent(offset_copy(H, 1), offset_copy(W, 3), y, c, dtype)


def test_xent_float32_magnitudes():
    """Values over the whole range of float32 exponents that the products can hold."""
    H, W, y, c = xent_inputs(100, 300, 64, "f32", 8)
    H *= torch.exp2(torch.randint(-40, 40, (100, 1), generator=gen(9), device="cuda").float())
    W *= 2.0 ** -45
    run_xent(H * 2.0 ** 4, W, y, c, "f32", norm=False)
    run_xent(H * 2.0 ** -60, W * 2.0 ** 45, y, c, "f32", norm=False)


def test_xent_offsets_beyond_32_bits():
    M, V, D = 3, 1100000, 2048                            # V * D > 2^31
    H, W, y, c = xent_inputs(M, V, D, "bf16", 10, ignored=0.0)
    y[0] = V - 1
    cfg = binding.make_xent_config(M, V, D, "bf16")
    loss, lse = binding.xent_forward(cfg, H, W, y)
    g = binding.xent_backward(cfg, H, W, y, lse, c)
    logits = torch.cat([H.double() @ w.double().t() for w in W.split(65536)], 1)
    want = torch.logsumexp(logits, 1)
    assert (lse.double() - want).abs().max() < 1e-4
    assert (loss.double() - (want - logits.gather(1, y.unsqueeze(1)).squeeze(1))).abs().max() < 1e-4
    last = slice(V - 500, V)
    G = torch.exp(logits - want.unsqueeze(1))
    G[torch.arange(M, device="cuda"), y] -= 1
    G *= c.double().unsqueeze(1)
    gw = G[:, last].t() @ H.double()
    assert float((g["gweight"][last].double() - gw).norm() / gw.norm()) < 4e-3
    gh = sum(G[:, i:i + 65536] @ W[i:i + 65536].double() for i in range(0, V, 65536))
    assert float((g["ghidden"].double() - gh).norm() / gh.norm()) < 4e-3


# ------------------------------------------------------------------ gradients against differences
def directional(f, params, grads, eps, tol, seed):
    """<grad, d> against the central difference of f along random d, parameter by parameter."""
    g = gen(seed)
    for k, (p, gr) in enumerate(zip(params, grads)):
        d = randn(p.shape, g)
        moved = lambda e: [q if j != k else p + e * d for j, q in enumerate(params)]
        num = (f(*moved(eps)) - f(*moved(-eps))) / (2 * eps)
        ana = float((gr.double() * d.double()).sum())
        scale = float((gr.double().norm() * d.double().norm()) / math.sqrt(p.numel()))
        assert abs(num - ana) < tol * max(scale, abs(ana)), (k, num, ana)


def test_scan_gradient_against_differences():
    T, B, N = 90, 2, 24
    x, gate, st, h0, gh, glast = scan_inputs(T, B, N, "f32", "logit", "time", 0.03, 21)
    cfg = binding.make_scan_config(T, B, N, "f32", "logit", "complement")
    saved = binding.scan_workspace(cfg)

    def f(x_, g_, h_):
        h, last = binding.scan_forward(cfg, x_, g_, st, h_, None, want_last=True)
        return float((h.double() * gh.double()).sum() + (last.double() * glast.double()).sum())

    binding.scan_forward(cfg, x, gate, st, h0, saved)
    g = binding.scan_backward(cfg, x, gate, gh, st, h0, glast, saved)
    # curvature eps^2 / 6 and float32 noise 1e-6 / eps are both below 1e-3 at eps = 1e-2
    directional(f, [x, gate, h0], [g["gx"], g["ggate"], g["gh0"]], 1e-2, 5e-3, 1)


def test_xent_gradient_against_differences():
    H, W, y, c = xent_inputs(60, 150, 32, "f32", 22)
    cfg = binding.make_xent_config(60, 150, 32)

    def f(h_, w_):
        return float((binding.xent_forward(cfg, h_, w_, y)[0].double() * c.double()).sum())

    _, lse = binding.xent_forward(cfg, H, W, y)
    g = binding.xent_backward(cfg, H, W, y, lse, c)
    directional(f, [H, W], [g["ghidden"], g["gweight"]], 1e-2, 5e-3, 2)


def test_embed_gradient_against_differences():
    g = gen(23)
    table, grad = randn((30, 20), g), randn((100, 20), g)
    ids = torch.randint(0, 30, (100,), generator=g, device="cuda")
    cfg = binding.make_embed_config(100, 30, 20, scale=3.0, padding_id=4)
    f = lambda t: float((binding.embed_forward(cfg, t, ids).double() * grad.double()).sum())
    directional(f, [table], [binding.embed_backward(cfg, ids, grad)], 1.0, 1e-4, 3)


# ------------------------------------------------------------------ autograd, streams
def test_autograd_functions_give_the_operators_gradients():
    T, B, N, V = 20, 3, 16, 50
    g = gen(31)
    ids = torch.randint(0, V, (T, B), generator=g, device="cuda")
    table, gates, readout = (randn((V, N), g).requires_grad_() for _ in range(3))
    x = EmbedFunction.apply(table, ids, 2.0, None)
    gate = EmbedFunction.apply(gates, ids)
    h, last = ScanFunction.apply(x, gate, None, None, "logit", "complement")
    y = torch.randint(0, V, (T * B,), generator=g, device="cuda")
    loss = XentFunction.apply(h.reshape(-1, N), readout, y).mean() + last.square().mean()
    loss.backward()
    t64, g64, r64 = (p.detach().double().requires_grad_() for p in (table, gates, readout))
    xs, a = 2 * t64[ids], torch.sigmoid(g64[ids])
    v, hs = torch.zeros(B, N, dtype=torch.float64, device="cuda"), []
    for t in range(T):
        v = a[t] * v + (1 - a[t]) * xs[t]
        hs.append(v)
    l64 = torch.nn.functional.cross_entropy(torch.stack(hs).reshape(-1, N) @ r64.t(), y) + v.square().mean()
    l64.backward()
    assert abs(loss.item() - l64.item()) < 1e-5
    for p, q in ((table, t64), (gates, g64), (readout, r64)):
        assert float((p.grad.double() - q.grad).norm() / q.grad.norm()) < 1e-5


def test_operators_run_on_the_given_stream():
    """On a side stream behind slow work: results are those of a synchronised run."""
    M, V, D = 200, 900, 64
    H, W, y, c = xent_inputs(M, V, D, "bf16", 41)
    cx = binding.make_xent_config(M, V, D, "bf16")
    ce = binding.make_embed_config(M, V, D, "bf16")
    cs = binding.make_scan_config(M, 1, D, "bf16", "logit", "complement")
    ids = y.clamp_min(0)

    def step(src):
        e = binding.embed_forward(ce, src, ids)
        h, _ = binding.scan_forward(cs, e.view(M, 1, D), e.view(M, 1, D))
        loss, lse = binding.xent_forward(cx, h.view(M, D), src, y)
        g = binding.xent_backward(cx, h.view(M, D), src, y, lse, c)
        gt = binding.embed_backward(ce, ids, g["ghidden"])
        return [loss, g["gweight"], gt]

    want = step(W)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(5):
        late = torch.zeros_like(W)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            big = torch.randn(4096, 4096, device="cuda")
            for _ in range(10):
                big = big @ big * 1e-3
            late.copy_(W + (big[0, 0] * 0).nan_to_num().to(W.dtype))
            got = step(late)
        s.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_operators_in_a_cuda_graph():
    """A step captured once gives, replayed on new inputs, the bits of the calls themselves."""
    M, V, D = 700, 900, 64
    H, W, y, c = xent_inputs(M, V, D, "bf16", 42)
    cx, ce = binding.make_xent_config(M, V, D, "bf16"), binding.make_embed_config(M, V, D, "bf16")
    cs = binding.make_scan_config(M, 1, D, "bf16", "logit", "complement")
    ids, x = y.clamp_min(0), H.view(M, 1, D)
    saved = binding.scan_workspace(cs)

    def step():
        h, _ = binding.scan_forward(cs, x, x, saved=saved)
        loss, lse = binding.xent_forward(cx, h.view(M, D), W, y)
        g = binding.xent_backward(cx, h.view(M, D), W, y, lse, c)
        gs = binding.scan_backward(cs, x, x, g["ghidden"].view(M, 1, D), saved=saved)
        return [loss, g["gweight"], gs["gx"], gs["ggate"], binding.embed_backward(ce, ids, gs["gx"].view(M, D))]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for seed in (43, 44):
        H.copy_(xent_inputs(M, V, D, "bf16", seed)[0])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, step()):
            assert torch.equal(a, b)


def test_operators_count_their_launches():
    n0 = binding.launch_count()
    cfg = binding.make_scan_config(3, 2, 8)
    x = torch.ones(3, 2, 8, device="cuda")
    binding.scan_forward(cfg, x, x)
    assert binding.launch_count() - n0 == 1
