"""The token-sequence operators, as measured cases: embedding, gated compartment scan, and
softmax cross entropy of a linear readout.

Each case is one pass a training step or a serving step makes through one operator. `run`
computes it with the library's kernels where `own` is true, and otherwise in plain form:
elementary torch operations in float32, rounded once at the end to the inputs' dtype.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one serving step of 64 sequences: latency of a small gather
        dict(name="embed_step", op="embed", n=64, V=32768, D=384, dtype="bf16", train=False),
        # an odd vocabulary and an odd width, float32: nothing is a multiple of a vector
        dict(name="embed_odd_f32", op="embed", n=5001, V=10007, D=251, dtype="f32", train=True),
        # an ordinary training batch: 16 sequences of 1024 tokens
        dict(name="embed_train", op="embed", n=16384, V=50000, D=1024, dtype="bf16", train=True),
        # the largest: 64 sequences of 2048 tokens over a large vocabulary
        dict(name="embed_large", op="embed", n=131072, V=131072, D=2048, dtype="bf16", train=True),
        # one serving step: one token for each of 64 sequences, state in and out
        dict(name="scan_step", op="scan", T=1, B=64, N=4096, dtype="bf16", gate="logit",
             mix="complement", layout="time", starts=False, train=False),
        # one long sequence on few channels: parallelism has to come from the time axis
        dict(name="scan_long", op="scan", T=16384, B=1, N=1024, dtype="f32", gate="decay",
             mix="plain", layout="time", starts=False, train=True),
        # odd sizes, batch first, packed sequences
        dict(name="scan_odd", op="scan", T=1009, B=3, N=1001, dtype="f32", gate="logit",
             mix="complement", layout="batch", starts=True, train=True),
        # the long-horizon layer (T = 2048, 16 x 4096 neurons) with packed sequences
        dict(name="scan_train", op="scan", T=2048, B=16, N=4096, dtype="bf16", gate="logit",
             mix="complement", layout="time", starts=True, train=True),
        # scoring one token of each of 16 sequences: bound by reading the readout weights
        dict(name="xent_score", op="xent", M=16, V=32768, D=384, dtype="bf16", ignored=0.0,
             train=False),
        # float32 with an odd vocabulary, a third of the rows ignored
        dict(name="xent_odd_f32", op="xent", M=1001, V=10007, D=384, dtype="f32", ignored=0.33,
             train=True),
        # an ordinary training batch
        dict(name="xent_train", op="xent", M=4096, V=50000, D=1024, dtype="bf16", ignored=0.1,
             train=True),
        # the largest: 8192 tokens over a large vocabulary
        dict(name="xent_large", op="xent", M=8192, V=131072, D=2048, dtype="bf16", ignored=0.02,
             train=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _even(rng, v, to):
    """Half of the sizes are multiples of `to`, the others as drawn."""
    return max(to, v // to * to) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(("embed", "scan", "xent"))
    dtype = rng.choice(("f32", "bf16"))
    if op == "embed":
        n = _log_int(rng, 1, 131072)
        return dict(op=op, n=n, V=_even(rng, _log_int(rng, 1000, 131072), 64),
                    D=_even(rng, _log_int(rng, 64, 1024 if dtype == "f32" else 2048), 64),
                    dtype=dtype, train=n > 256)
    if op == "scan":
        T = _log_int(rng, 1, 16384)
        most = (2 ** 26 if dtype == "f32" else 2 ** 27) // T
        B = _log_int(rng, 1, min(64, most))
        N = _even(rng, _log_int(rng, 16, max(16, min(8192, most // B))), 16)
        return dict(op=op, T=T, B=B, N=N, dtype=dtype, gate=rng.choice(("decay", "logit")),
                    mix=rng.choice(("plain", "complement")),
                    layout=rng.choice(("time", "batch")),
                    starts=T > 4 and rng.random() < 0.5, train=T > 1)
    M = _log_int(rng, 1, 8192 if dtype == "bf16" else 4096)
    return dict(op=op, M=M, V=_even(rng, _log_int(rng, 1000, 131072 if dtype == "bf16" else 65536), 64),
                D=_even(rng, _log_int(rng, 64, 2048 if dtype == "bf16" else 1024), 64), dtype=dtype,
                ignored=rng.choice((0.0, 0.1, 0.5)), train=M > 64)


# ------------------------------------------------------------------ inputs
def _zipf(n, V, g, device):
    """Token ids as text has them: rank r with a weight of about 1 / (r + 3), ranks spread over
    the vocabulary."""
    u = torch.rand(n, generator=g, device=device, dtype=torch.float64)
    rank = (torch.exp(u * math.log((V + 3) / 3.0)) * 3.0 - 3.0).long().clamp_(0, V - 1)
    step = 7919
    while math.gcd(step, V) != 1:
        step += 2
    return (rank * step) % V


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(shape, std=1.0):
        return torch.randn(shape, generator=g, device=dev).mul_(std).to(dt)

    s = {"case": case}
    if case["op"] == "embed":
        n, V, D = case["n"], case["V"], case["D"]
        s["table"] = normal((V, D), 1.0 / math.sqrt(D))
        s["ids"] = _zipf(n, V, g, dev)
        s["scale"] = math.sqrt(D)
        s["padding_id"] = 0
        if case["train"]:
            s["grad"] = normal((n, D))
    elif case["op"] == "scan":
        T, B, N = case["T"], case["B"], case["N"]
        shape = (T, B, N) if case["layout"] == "time" else (B, T, N)
        s["x"] = normal(shape)
        if case["gate"] == "logit":     # decays around 0.9
            s["gate"] = torch.randn(shape, generator=g, device=dev).add_(2.0).to(dt)
        else:                           # decays of compartments: U(0.5, 0.95), as the layers draw them
            s["gate"] = torch.rand(shape, generator=g, device=dev).mul_(0.45).add_(0.5).to(dt)
        s["h0"] = torch.randn((B, N), generator=g, device=dev)
        s["starts"] = None
        if case["starts"]:              # packed sequences of about 200 tokens
            s["starts"] = (torch.rand(shape[:2], generator=g, device=dev) < 0.005).to(torch.uint8)
        if case["train"]:
            s["gh"] = normal(shape)
            s["glast"] = torch.randn((B, N), generator=g, device=dev)
    else:
        M, V, D = case["M"], case["V"], case["D"]
        s["hidden"] = normal((M, D))
        s["weight"] = normal((V, D), 2.0 / math.sqrt(D))
        s["labels"] = _zipf(M, V, g, dev)
        drop = torch.rand(M, generator=g, device=dev) < case["ignored"]
        s["labels"][drop] = -100
        if case["train"]:               # a mean over the batch, each row with a weight of its own
            s["gloss"] = torch.rand(M, generator=g, device=dev).add_(0.5).div_(M)
    return s


# ------------------------------------------------------------------ the library's operators
def _run_own(s):
    from paper_2412_06355_gb300 import binding as b
    c = s["case"]
    if c["op"] == "embed":
        cfg = b.make_embed_config(c["n"], c["V"], c["D"], c["dtype"], scale=s["scale"],
                                  padding_id=s["padding_id"])
        out = {"out": b.embed_forward(cfg, s["table"], s["ids"])}
        if c["train"]:
            out["gtable"] = b.embed_backward(cfg, s["ids"], s["grad"])
        return out
    if c["op"] == "scan":
        cfg = b.make_scan_config(c["T"], c["B"], c["N"], c["dtype"], gate=c["gate"],
                                 mix=c["mix"], layout=c["layout"])
        saved = b.scan_workspace(cfg) if c["train"] else None
        h, last = b.scan_forward(cfg, s["x"], s["gate"], s["starts"], s["h0"], saved=saved,
                                 want_last=True)
        out = {"h": h, "last": last}
        if c["train"]:
            out.update(b.scan_backward(cfg, s["x"], s["gate"], s["gh"], s["starts"], s["h0"],
                                       grad_last=s["glast"], saved=saved))
        return out
    cfg = b.make_xent_config(c["M"], c["V"], c["D"], c["dtype"], ignore_index=-100)
    loss, lse = b.xent_forward(cfg, s["hidden"], s["weight"], s["labels"])
    out = {"loss": loss}
    if c["train"]:
        out.update(b.xent_backward(cfg, s["hidden"], s["weight"], s["labels"], lse, s["gloss"]))
    return out


# ------------------------------------------------------------------ the plain forms
def _plain_embed(s):
    c = s["case"]
    dt, ids = s["table"].dtype, s["ids"]
    keep = (ids != s["padding_id"]).unsqueeze(1)
    out = {"out": (s["table"][ids].float() * s["scale"] * keep).to(dt)}
    if c["train"]:
        g = torch.zeros((c["V"], c["D"]), device=ids.device)
        g.index_add_(0, ids, s["grad"].float() * keep)
        out["gtable"] = (g * s["scale"]).to(dt)
    return out


def _double(a, b):
    """b_t <- a_t b_{t-1} + b_t along the first axis, by doubling the reach log2(T) times."""
    T, reach = a.shape[0], 1
    while reach < T:
        b = torch.cat([b[:reach], torch.addcmul(b[reach:], a[reach:], b[:-reach])])
        a = torch.cat([a[:reach], a[reach:] * a[:-reach]])
        reach *= 2
    return b


def _plain_scan(s):
    c = s["case"]
    dt = s["x"].dtype

    def time_first(v):
        return v.transpose(0, 1) if c["layout"] == "batch" else v

    x, g = time_first(s["x"]).float(), time_first(s["gate"]).float()
    a = 1.0 / (1.0 + torch.exp(-g)) if c["gate"] == "logit" else g
    na = 1.0 / (1.0 + torch.exp(g)) if c["gate"] == "logit" else 1.0 - g
    m = a if s["starts"] is None else a * (time_first(s["starts"]) == 0).unsqueeze(2)
    u = x * na if c["mix"] == "complement" else x.clone()
    u[0] += m[0] * s["h0"]
    h = _double(m, u)
    out = {"h": time_first(h).to(dt), "last": h[-1].clone()}
    if c["train"]:
        gh = time_first(s["gh"]).float().clone()
        gh[-1] += s["glast"]
        nxt = torch.cat([m[1:], torch.zeros_like(m[:1])])
        lam = _double(nxt.flip(0), gh.flip(0)).flip(0)
        before = torch.cat([s["h0"].unsqueeze(0), h[:-1]])
        if s["starts"] is not None:
            before = before * (time_first(s["starts"]) == 0).unsqueeze(2)
        ga = lam * (before - x) if c["mix"] == "complement" else lam * before
        out["gx"] = time_first(lam * na if c["mix"] == "complement" else lam).to(dt)
        out["ggate"] = time_first(ga * a * na if c["gate"] == "logit" else ga).to(dt)
        out["gh0"] = m[0] * lam[0]
    return out


def _plain_xent(s):
    c = s["case"]
    dt = s["hidden"].dtype
    H, W, y = s["hidden"].float(), s["weight"].float(), s["labels"]
    keep = y != -100
    at = torch.where(keep, y, torch.zeros_like(y)).unsqueeze(1)
    logits = H @ W.t()
    top = logits.max(1, keepdim=True).values
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    loss = (top + torch.log(total) - logits.gather(1, at)).squeeze(1)
    out = {"loss": torch.where(keep, loss, torch.zeros_like(loss))}
    if c["train"]:
        del logits
        g = e.div_(total)
        g.scatter_add_(1, at, torch.full_like(total, -1.0))
        g.mul_((s["gloss"] * keep).unsqueeze(1))
        out["ghidden"] = (g @ W).to(dt)
        out["gweight"] = (g.t() @ H).to(dt)
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"embed": _plain_embed, "scan": _plain_scan, "xent": _plain_xent}[state["case"]["op"]](state)


# ------------------------------------------------------------------ floors
def work(case):
    b = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "embed":
        n, V, D = case["n"], case["V"], case["D"]
        moved = n * 8 + min(n, V) * D * b + n * D * b
        if case["train"]:
            moved += n * D * b + V * D * b
        return {"bytes": moved, "flops": n * D * (2 if case["train"] else 1)}
    if case["op"] == "scan":
        T, M = case["T"], case["B"] * case["N"]
        flags = T * case["B"] if case["starts"] else 0
        arrays, states = (6, 4) if case["train"] else (3, 2)
        return {"bytes": arrays * T * M * b + flags + states * M * 4,
                "flops": (8 if case["train"] else 2) * T * M}
    M, V, D = case["M"], case["V"], case["D"]
    rows = M * (1.0 - case["ignored"])
    return {"bytes": (M + V) * D * b * (2 if case["train"] else 1) + M * 16,
            "flops": (6.0 if case["train"] else 2.0) * rows * V * D}


# ------------------------------------------------------------------ 64 bits
def _as(t):
    return t.detach().cpu().double().numpy()


def _exact_embed(s):
    ids = s["ids"].cpu().numpy()
    kept = ids != s["padding_id"]
    out = {"out": _as(s["table"])[ids] * s["scale"] * kept[:, None]}
    if s["case"]["train"]:
        order = np.argsort(ids, kind="stable")
        rows, first = np.unique(ids[order], return_index=True)
        g = np.zeros((s["case"]["V"], s["case"]["D"]))
        g[rows] = np.add.reduceat(_as(s["grad"])[order], first, axis=0) * s["scale"]
        g[s["padding_id"]] = 0.0
        out["gtable"] = g
    return out


def _exact_scan(s):
    """The recurrence step by step, in float64 on the GPU."""
    c = s["case"]
    batch_first = c["layout"] == "batch"
    shape = s["x"].shape
    T = c["T"]
    step = [(slice(None), t) if batch_first else (t,) for t in range(T)]
    x, raw = s["x"].double(), s["gate"].double()
    a = torch.sigmoid(raw) if c["gate"] == "logit" else raw
    first = torch.zeros(shape[:2], dtype=torch.bool, device=x.device) if s["starts"] is None else s["starts"].bool()
    carry = a.masked_fill(first.unsqueeze(2), 0.0)
    weight = 1.0 - a if c["mix"] == "complement" else torch.ones_like(a)
    h, prev = torch.empty_like(x), torch.empty_like(x)
    state = s["h0"].double()
    for at in step:
        prev[at] = state
        state = carry[at] * state + weight[at] * x[at]
        h[at] = state
    out = {"h": h, "last": state}
    if c["train"]:
        gx, ga = torch.empty_like(x), torch.empty_like(x)
        gh = s["gh"].double()
        back = s["glast"].double()
        live = (~first).unsqueeze(2).double()
        for at in reversed(step):
            lam = gh[at] + back
            gx[at] = lam * weight[at]
            ga[at] = lam * (live[at] * prev[at] - (x[at] if c["mix"] == "complement" else 0.0))
            back = carry[at] * lam
        out.update(gx=gx, ggate=ga * a * (1.0 - a) if c["gate"] == "logit" else ga, gh0=back)
    return out


def _exact_xent(s):
    """Row by row of logits, in float64 on the GPU, in blocks of rows."""
    c = s["case"]
    H, W, y = s["hidden"].double(), s["weight"].double(), s["labels"]
    loss = torch.zeros(c["M"], dtype=torch.float64, device=H.device)
    gw = torch.zeros_like(W) if c["train"] else None
    gh = torch.zeros_like(H) if c["train"] else None
    rows = torch.nonzero(y != -100).squeeze(1)
    for r in rows.split(512):
        logits = torch.mm(H[r], W.t())
        lse = torch.logsumexp(logits, 1)
        loss[r] = lse - logits[torch.arange(len(r), device=r.device), y[r]]
        if c["train"]:
            p = torch.exp(logits - lse.unsqueeze(1))
            p[torch.arange(len(r), device=r.device), y[r]] -= 1.0
            p *= s["gloss"][r].double().unsqueeze(1)
            gh[r] = p @ W
            gw += p.t() @ H[r]
    return {"loss": loss, "ghidden": gh, "gweight": gw} if c["train"] else {"loss": loss}


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "scan": _exact_scan, "xent": _exact_xent}[case["op"]](s)
