"""The operators of a token block together, as a program uses them, and how they are called: a block's
training step against float64, streams, graphs, host threads, serving token by token."""
import threading

import pytest
import torch

import block_reference as ref
from block_reference import U32
from paper_2412_06355_gb300 import AdamW, DeltaFunction, EmbedFunction, NormFunction, XentFunction, binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    binding.load()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


V, D, H, DK, DV, T, B = 50, 24, 2, 8, 12, 70, 2
SHAPES = dict(table=(V, D), n1=(D,), n2=(D,), wq=(D, DK), wk=(D, DK), wv=(D, H * DV), wg=(D, H), wb=(D, H), wo=(H * DV, D), readout=(V, D))


def parameters():
    g = gen(0)
    p = {n: torch.randn(s, generator=g, device="cuda") * (1.0 if n == "table" else s[0] ** -0.5) for n, s in SHAPES.items()}
    p["n1"], p["n2"] = 1 + 0.1 * p["n1"], 1 + 0.1 * p["n2"]
    return p


def block(p, ids, embed, norm, delta):
    """Rows of the readout's inputs: embedding, norm, delta rule over what it projects, norm of the sum."""
    x = embed(p["table"], ids)
    y, total = norm(x, None, p["n1"])
    k = y @ p["wk"]
    k = (k / (1.0 + k.square().sum(-1, keepdim=True)).sqrt()).unsqueeze(2)
    q, v = (y @ p["wq"]).unsqueeze(2), (y @ p["wv"]).view(T, B, H, DV)
    o = delta(q, k, v, -torch.nn.functional.softplus(y @ p["wg"]), torch.sigmoid(y @ p["wb"]))
    z, _ = norm(o.reshape(T, B, H * DV) @ p["wo"], total, p["n2"])
    return z.reshape(T * B, D)


def test_a_training_step_of_a_block():
    """Gradients of all parameters against float64, then AdamW's step on them.

    Each of the some twenty operators on a gradient's way is off by at most 32 U32 of its norm (the delta rule;
    the others, products of 24 to 70 places among them, by less): 640 U32 for the way, and what each hands on
    to the others is not more than 4 times larger than itself here (weights of length about 1)."""
    ids = torch.randint(0, V, (T, B), generator=gen(1), device="cuda")
    labels = torch.randint(0, V, (T * B,), generator=gen(2), device="cuda")
    p = {n: t.requires_grad_() for n, t in parameters().items()}
    scale = DK ** -0.5
    z = block(p, ids, EmbedFunction.apply, lambda x, r, w: NormFunction.apply(x, r, w, 1e-5),
              lambda *a: DeltaFunction.apply(*a, None, None, scale, "time")[0])
    loss = XentFunction.apply(z, p["readout"], labels).sum()
    loss.backward()

    d = {n: t.detach().double().requires_grad_() for n, t in p.items()}
    eps = float(torch.tensor(1e-5))

    def norm(x, r, w):
        s = x if r is None else x + r
        return s / torch.sqrt(s.square().mean(-1, keepdim=True) + eps) * w, s

    def delta(q, k, v, gate, beta):
        flat = [t.reshape(T * B, *t.shape[2:]) for t in (q, k, v, gate, beta)]
        s0 = torch.zeros(B, H, DK, DV, dtype=torch.float64, device="cuda")
        return ref.delta(*flat, s0, ref.sequences("time", T, B, None), float(torch.tensor(scale)))[0].view(T, B, H, DV)

    logits = block(d, ids, lambda w, i: w[i], norm, delta) @ d["readout"].t()
    want = (torch.logsumexp(logits, 1) - logits.gather(1, labels[:, None])[:, 0]).sum()
    want.backward()
    assert abs(float(loss) - float(want)) < 640 * U32 * abs(float(want))
    for n in p:
        assert float((p[n].grad.double() - d[n].grad).norm()) < 4 * 640 * U32 * float(d[n].grad.norm()), n

    before = {n: t.detach().clone() for n, t in p.items()}
    opt = AdamW(p.values(), lr=1e-2, weight_decay=0.1, max_norm=0.5)
    opt.step()
    total = float(torch.stack([t.grad.double().square().sum() for t in p.values()]).sum().sqrt())
    assert total > 0.5 and abs(float(opt.grad_norm) - total) < 20 * U32 * total
    for n, t in p.items():
        m = v = torch.zeros_like(t, dtype=torch.float64)
        q, _, _ = ref.adamw(before[n], t.grad, m, v, 1, 1e-2, (0.9, 0.999), 1e-8, 0.1, 0.5 / total)
        # a first step moves by lr g / (|g| + eps sqrt(1 - beta2)): 64 U32 of it, and rounding of p
        assert float((t.detach().double() - q).abs().max()) < 1e-2 * 64 * U32 + 4 * U32 * float(before[n].abs().max()), n


def step_of(dtype, seed, layout="batch", T=130, B=3):
    """Inputs of norm -> delta -> gradients, and the calls."""
    g = gen(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    unit = lambda t: (t / t.square().sum(-1, keepdim=True).sqrt()).to(dt)
    x = dict(x=r(B * T, 64).to(dt), res=r(B * T, 64).to(dt), w=1 + 0.1 * r(64), q=unit(r(B, T, 1, 32)), k=unit(r(B, T, 1, 32)),
             gate=-r(B, T, 2).exp() * 0.1, beta=torch.sigmoid(r(B, T, 2)), s0=r(B, 2, 32, 32), go=r(B, T, 2, 32).to(dt), glast=r(B, 2, 32, 32))
    cn = binding.make_norm_config(B * T, 64, dtype)
    cd = binding.make_delta_config(T, B, 1, 2, 32, 32, dtype, layout, 32 ** -0.5)

    def run(x, saved, between=lambda: None, **kw):
        y, total, _ = binding.norm_forward(cn, x["x"], x["w"], x["res"], **kw)
        between()
        o, last = binding.delta_forward(cd, x["q"], x["k"], y.view(B, T, 2, 32), x["gate"], x["beta"], None, x["s0"], saved=saved, want_last=True, **kw)
        between()
        g = binding.delta_backward(cd, x["q"], x["k"], y.view(B, T, 2, 32), x["gate"], x["beta"], x["go"], None, x["s0"], x["glast"], saved=saved, **kw)
        between()
        gn = binding.norm_backward(cn, total, x["w"], g["gv"].view(B * T, 64), x["x"], **kw)
        between()
        return [y, total, o, last, *g.values(), *gn.values()]

    return x, cd, run


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_on_a_stream_that_is_not_current(dtype, raw):
    x, cfg, run = step_of(dtype, 3)
    saved = binding.delta_workspace(cfg)
    want = run(x, saved)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    sizes = [*binding.dendsn_delta_workspace_size(cfg), x["x"].numel() * 2, x["x"].numel() * 4, x["s0"].numel() * 4]

    def fill():                                             # takes whatever memory looks free, and writes it
        for s in sizes:
            for _ in range(3):
                torch.full((s,), 255, dtype=torch.uint8, device="cuda")

    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            big = big @ big * 1e-3
    got = run(x, saved, fill, stream=side.cuda_stream if raw else side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_replayed_on_other_inputs(dtype):
    """Two graphs, each with buffers of its own, replayed in turn."""
    graphs = []
    for seed in (5, 6):
        x, cfg, run = step_of(dtype, seed)
        saved = binding.delta_workspace(cfg)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run(x, saved)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run(x, saved)
        graphs.append((graph, x, out, run, cfg))
    for seed in (7, 8):
        news = []
        for i, (graph, x, out, run, cfg) in enumerate(graphs):
            new, _, _ = step_of(dtype, seed + 10 * i)
            for n in x:
                x[n].copy_(new[n])
            news.append(new)
        for graph, *_ in graphs:
            graph.replay()
        for (graph, x, out, run, cfg), new in zip(graphs, news):
            want = run(new, binding.delta_workspace(cfg))
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_autograd_captured():
    """Forward and backward of both functions in one graph, its leaves not used eagerly before."""
    x, cfg, _ = step_of("f32", 9)
    leaves = [x[n].clone().requires_grad_() for n in ("x", "w", "q", "k", "gate", "beta")]

    def step():
        y, _ = NormFunction.apply(leaves[0], None, leaves[1])
        o, _ = DeltaFunction.apply(*leaves[2:4], y.view(3, 130, 2, 32), *leaves[4:], None, None, 0.2, "batch")
        return torch.autograd.grad((o * x["go"]).sum(), leaves)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    with torch.no_grad():
        leaves[0].mul_(0.5).add_(0.1)
    graph.replay()
    torch.cuda.synchronize()
    kept = [t.clone() for t in got]
    assert all(torch.equal(a, b) for a, b in zip(kept, step()))


def test_two_host_threads_on_their_own_streams():
    cases = [step_of("bf16", 11), step_of("f32", 12)]
    want = [run(x, binding.delta_workspace(cfg)) for x, cfg, run in cases]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        try:
            x, cfg, run = cases[i]
            with torch.cuda.stream(torch.cuda.Stream()):
                saved = binding.delta_workspace(cfg)
                for _ in range(20):
                    got = run(x, saved)
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                        wrong.append(i)
        except Exception as e:                              # noqa: BLE001
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_a_prompt_then_token_by_token():
    """Serving: a packed prefill hands its states to single tokens, as the whole sequences at once give them."""
    lens, more, Hk, Hv, Dk, Dv = [65, 3, 128], 4, 1, 2, 64, 32
    g = gen(20)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    unit = lambda t: t / t.square().sum(-1, keepdim=True).sqrt()
    whole = [n + more for n in lens]
    N = sum(whole)
    q, k, v = unit(r(N, Hk, Dk)).bfloat16(), unit(r(N, Hk, Dk)).bfloat16(), r(N, Hv, Dv).bfloat16()
    gate, beta = -r(N, Hv).exp() * 0.05, torch.sigmoid(r(N, Hv))
    offs = lambda ls: torch.tensor([sum(ls[:i]) for i in range(len(ls) + 1)], dtype=torch.int32, device="cuda")
    cfg = binding.make_delta_config(N, 3, Hk, Hv, Dk, Dv, "bf16", "packed", 0.1)
    o, last = binding.delta_forward(cfg, q, k, v, gate, beta, offs(whole), want_last=True)
    starts = [sum(whole[:i]) for i in range(3)]
    prompt = torch.tensor([s + i for s, n in zip(starts, lens) for i in range(n)], device="cuda")
    pre = binding.make_delta_config(sum(lens), 3, Hk, Hv, Dk, Dv, "bf16", "packed", 0.1)
    _, state = binding.delta_forward(pre, *(t[prompt] for t in (q, k, v, gate, beta)), offs(lens), want_last=True)
    one = binding.make_delta_config(1, 3, Hk, Hv, Dk, Dv, "bf16", "batch", 0.1)
    for i in range(more):
        at = torch.tensor([s + n + i for s, n in zip(starts, lens)], device="cuda")
        row, _ = binding.delta_forward(one, *(t[at].unsqueeze(1) for t in (q, k, v, gate, beta)), s0=state, last=state)
        # both are within 32 U32 of the recurrence before they are rounded: half a bfloat16 step each, and that
        err = (row[:, 0].float() - o[at].float()).abs()
        assert bool((err <= o[at].float().abs() * 2.0 ** -7 + 2.0 ** -16).all())
    assert float((state - last).norm()) < 64 * U32 * float(last.norm())
