"""How the token-sequence operators are called on the GPU: other streams than the current one,
several host threads, graphs, and the sizes at which other kernels take over."""

import threading

import pytest
import torch

import seq_reference as ref
from paper_2412_06355_gb300 import binding

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


@pytest.mark.parametrize("raw", [False, True])
def test_wrappers_on_a_stream_that_is_not_current(raw):
    """The current stream allocates and fills memory right after each call, while the kernels
    still wait behind slow work on their own stream."""
    n, V, D = 3000, 900, 64
    g = gen(1)
    W = torch.randn((V, D), generator=g, device="cuda").bfloat16()
    y = torch.randint(0, V, (n,), generator=g, device="cuda")
    c = torch.rand(n, generator=g, device="cuda")
    ce = binding.make_embed_config(n, V, D, "bf16")
    cs = binding.make_scan_config(n, 1, D, "bf16", "logit", "complement")
    cx = binding.make_xent_config(n, V, D, "bf16")
    saved = binding.scan_workspace(cs)

    def step(stream, between):
        kw = {} if stream is None else dict(stream=stream)
        e = binding.embed_forward(ce, W, y, **kw).view(n, 1, D)
        between()
        h, last = binding.scan_forward(cs, e, e, saved=saved, want_last=True, **kw)
        between()
        loss, lse = binding.xent_forward(cx, h.view(n, D), W, y, **kw)
        between()
        gx = binding.xent_backward(cx, h.view(n, D), W, y, lse, c, **kw)
        between()
        gs = binding.scan_backward(cs, e, e, gx["ghidden"].view(n, 1, D), saved=saved, **kw)
        between()
        gt = binding.embed_backward(ce, y, gs["gx"].view(n, D), **kw)
        between()
        return [e, h, last, loss, gx["gweight"], gs["gx"], gs["ggate"], gt]

    want = step(None, lambda: None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    sizes = [s for c_ in (cx,) for s in binding.dendsn_xent_workspace_size(c_)]
    sizes += [binding.dendsn_embed_workspace_size(ce), n * D * 2, n * 4, V * D * 2]

    def fill():                                       # takes whatever memory looks free, and writes it
        for s in sizes:
            for _ in range(3):
                torch.full((s,), 255, dtype=torch.uint8, device="cuda")

    for _ in range(3):
        big = torch.randn(4096, 4096, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(20):
                big = big @ big * 1e-3
        got = step(side.cuda_stream if raw else side, fill)
        side.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_embedding_gradients_from_two_host_threads():
    """Two sizes whose index kernels want different amounts of shared memory, called at once."""
    V, D = 50, 8
    cases, errors = [], []
    for n in (300000, 1100000):
        g = gen(n)
        ids = torch.randint(0, V, (n,), generator=g, device="cuda")
        grad = torch.ones((n, D), device="cuda")
        cfg = binding.make_embed_config(n, V, D)
        scratch = torch.empty(binding.dendsn_embed_workspace_size(cfg), dtype=torch.uint8, device="cuda")
        cases.append((cfg, ids, grad, torch.empty(V, D, device="cuda"), scratch,
                      torch.bincount(ids, minlength=V).float()))
    torch.cuda.synchronize()
    go = threading.Barrier(2)

    def work(cfg, ids, grad, out, scratch, _):
        go.wait()
        try:
            for _ in range(1500):
                binding.dendsn_embed_backward(cfg, ids, grad, out, scratch)
        except Exception as e:              # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=c) for c in cases]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for _, _, _, out, _, count in cases:
        assert torch.equal(out, count.unsqueeze(1).expand(V, D))


def test_the_cooperative_index_in_a_cuda_graph():
    """More than 8192 tokens: captured once, replayed on other tokens and gradients."""
    n, V, D = 20000, 3000, 40
    cfg = binding.make_embed_config(n, V, D)
    scratch = torch.empty(binding.dendsn_embed_workspace_size(cfg), dtype=torch.uint8, device="cuda")

    def inputs(seed):
        g = gen(seed)
        ids = torch.randint(0, V, (n,), generator=g, device="cuda")
        ids[::3] = 7
        return ids, torch.randn((n, D), generator=g, device="cuda")

    ids, grad = inputs(1)
    out = torch.empty(V, D, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.dendsn_embed_backward(cfg, ids, grad, out, scratch)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.dendsn_embed_backward(cfg, ids, grad, out, scratch)
    for seed in (2, 3):
        new = inputs(seed)
        ids.copy_(new[0])
        grad.copy_(new[1])
        graph.replay()
        torch.cuda.synchronize()
        ref.check("gtable", out, ref.embed_backward(ids, grad, V, 1.0, None))


def test_operators_from_two_host_threads_on_their_own_streams():
    """Each thread gets the bits of a run alone."""
    def inputs(M, seed):
        g = gen(seed)
        V, D = 900, 64
        W = torch.randn((V, D), generator=g, device="cuda").bfloat16()
        y = torch.randint(0, V, (M,), generator=g, device="cuda")
        return (M, V, D, W, y, torch.rand(M, generator=g, device="cuda"))

    def step(M, V, D, W, y, c):
        cx = binding.make_xent_config(M, V, D, "bf16")
        ce = binding.make_embed_config(M, V, D, "bf16")
        cs = binding.make_scan_config(M, 1, D, "bf16", "logit", "complement")
        e = binding.embed_forward(ce, W, y).view(M, 1, D)
        saved = binding.scan_workspace(cs)
        h, _ = binding.scan_forward(cs, e, e, saved=saved)
        loss, lse = binding.xent_forward(cx, h.view(M, D), W, y)
        g = binding.xent_backward(cx, h.view(M, D), W, y, lse, c)
        gs = binding.scan_backward(cs, e, e, g["ghidden"].view(M, 1, D), saved=saved)
        return [loss, g["gweight"], binding.embed_backward(ce, y, gs["gx"].view(M, D))]

    data = [inputs(700, 1), inputs(3000, 2)]
    want = [step(*d) for d in data]
    torch.cuda.synchronize()
    go, errors = threading.Barrier(2), []

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                go.wait()
                for _ in range(100):
                    got = step(*data[k])
                torch.cuda.current_stream().synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, want[k]))
        except Exception as e:              # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


@pytest.mark.parametrize("handle", [0, 1, 2])
def test_the_drivers_own_stream_handles(handle):
    """0 and 1 are the default stream, 2 the calling thread's."""
    g = gen(4)
    table = torch.randn((50, 16), generator=g, device="cuda")
    ids = torch.randint(0, 50, (300,), generator=g, device="cuda")
    cfg = binding.make_embed_config(300, 50, 16)
    torch.cuda.synchronize()
    before = torch.cuda.current_stream()
    out = binding.embed_forward(cfg, table, ids, stream=handle)
    grad = binding.embed_backward(cfg, ids, out, stream=handle)
    assert torch.cuda.current_stream() == before
    torch.cuda.synchronize()
    assert torch.equal(out, table[ids])
    ref.check("gtable", grad, ref.embed_backward(ids, out, 50, 1.0, None))
