"""The operators of a stack of token blocks and of its training step, as measured cases: the
root-mean-square norm with the residual's addition, the gated delta rule, and the AdamW step over
many tensors.

Each case is one pass a training step or a serving step makes through one operator. `run`
computes it with the library's kernels where `own` is true, and otherwise in plain form:
elementary torch operations in float32, rounded once at the end.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
BLOCK = 256          # elements that share a scale of the 8-bit optimizer states
BETAS, EPS, LR, DECAY, SEED = (0.9, 0.999), 1e-8, 1e-3, 0.01, 1234


def listed():
    return [
        # one serving step of 64 sequences: latency of a small norm
        dict(name="norm_step", op="norm", M=64, D=384, dtype="bf16", residual=True, out="same",
             train=False),
        # odd rows and an odd width, float32: nothing is a multiple of a vector
        dict(name="norm_odd_f32", op="norm", M=1009, D=1001, dtype="f32", residual=True, out="same",
             train=True),
        # an ordinary training batch: 16 sequences of 1024 tokens
        dict(name="norm_train", op="norm", M=16384, D=1024, dtype="bf16", residual=True, out="same",
             train=True),
        # the largest: a long prefill whose next product takes 8-bit operands
        dict(name="norm_large8", op="norm", M=32768, D=8192, dtype="bf16", residual=True,
             out="e4m3_128", train=False),
        # one serving step: one token for each of 64 sequences, states updated in place
        dict(name="delta_step", op="delta", T=1, B=64, Hk=4, Hv=8, Dk=128, Dv=128, dtype="bf16",
             layout="batch", train=False),
        # odd sizes, time first, two value heads on a key head, float32
        dict(name="delta_odd_f32", op="delta", T=509, B=3, Hk=3, Hv=6, Dk=40, Dv=72, dtype="f32",
             layout="time", train=True),
        # packed sequences of very different lengths, one of them empty, on few heads
        dict(name="delta_packed", op="delta", T=16384, B=24, Hk=4, Hv=8, Dk=64, Dv=128, dtype="bf16",
             layout="packed", train=True),
        # the largest: a training batch of 8 sequences of 2048 tokens, 16 heads
        dict(name="delta_train", op="delta", T=2048, B=8, Hk=16, Hv=16, Dk=128, Dv=128, dtype="bf16",
             layout="batch", train=True),
        # the parameters of a one-layer token model (512 tokens, 256 neurons of 4 compartments)
        dict(name="adamw_example", op="adamw", count=7, total=1183744, param="f32", grad="f32",
             copy=False, state="f32", clip=False, odd=False),
        # many tensors of odd sizes at odd addresses, bfloat16, clipped
        dict(name="adamw_odd", op="adamw", count=37, total=2000003, param="bf16", grad="bf16",
             copy=False, state="f32", clip=True, odd=True),
        # float32 parameters, bfloat16 gradients and bfloat16 copies for the next forward, clipped
        dict(name="adamw_train", op="adamw", count=150, total=134217728, param="f32", grad="bf16",
             copy=True, state="f32", clip=True, odd=False),
        # the largest: bfloat16 parameters with states in 8 bits
        dict(name="adamw_large8", op="adamw", count=200, total=536870912, param="bf16", grad="bf16",
             copy=False, state="e4m3", clip=False, odd=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _even(rng, v, to):
    """Half of the sizes are multiples of `to`, the others as drawn."""
    return max(to, v // to * to) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(("norm", "delta", "adamw"))
    dtype = rng.choice(("f32", "bf16"))
    if op == "norm":
        D = _even(rng, _log_int(rng, 16, 16384), 16)
        out = rng.choice(("same", "same", "e4m3_row", "e4m3_128"))
        return dict(op=op, M=_log_int(rng, 1, min(65536, 2 ** 26 // D)), D=D, dtype=dtype,
                    residual=rng.random() < 0.7, out=out, train=out == "same" and rng.random() < 0.7)
    if op == "delta":
        layout = rng.choice(("time", "batch", "packed"))
        Hk = rng.choice((1, 2, 3, 4, 8))
        Hv = Hk * rng.choice((1, 1, 2))
        if rng.random() < 0.3:          # a serving step
            return dict(op=op, T=1, B=_log_int(rng, 1, 256), Hk=Hk, Hv=Hv,
                        Dk=rng.choice((32, 64, 128)), Dv=rng.choice((32, 64, 128)), dtype=dtype,
                        layout=rng.choice(("time", "batch")), train=False)
        T = _log_int(rng, 16, 8192)
        B = _log_int(rng, 1, max(1, min(32, 131072 // (T * Hv))))
        return dict(op=op, T=T * B if layout == "packed" else T, B=B, Hk=Hk, Hv=Hv,
                    Dk=_even(rng, _log_int(rng, 8, 128), 16), Dv=_even(rng, _log_int(rng, 8, 128), 16),
                    dtype=dtype, layout=layout, train=rng.random() < 0.8)
    state = rng.choice(("f32", "e4m3"))
    total = _log_int(rng, 10000, 2 ** 27)
    return dict(op=op, count=min(_log_int(rng, 1, 200), total // 1000), total=total, param=dtype,
                grad=rng.choice(("f32", "bf16")), copy=dtype == "f32" and rng.random() < 0.4,
                state=state, clip=rng.random() < 0.5, odd=rng.random() < 0.3)


# ------------------------------------------------------------------ inputs
def _lengths(case, seed):
    """Lengths of the packed sequences: log-normal, the second one empty, tokens left behind the last."""
    r = random.Random(seed)
    T, B = case["T"], case["B"]
    share = [math.exp(r.gauss(0.0, 1.0)) for _ in range(B)]
    if B > 2:
        share[1] = 0.0
    use = T - min(7, T // 8)
    lens = [int(use * v / sum(share)) for v in share]
    lens[0] += use - sum(lens)
    return lens


def _sizes(case):
    """Element counts of the tensors: a few large ones hold most, as in a model."""
    n, total = case["count"], case["total"]
    r = random.Random(n * 1000003 + total)
    share = [math.exp(r.gauss(0.0, 1.5)) for _ in range(n)]
    sizes = [max(1, int(total * v / sum(share))) for v in share]
    if not case["odd"]:
        sizes = [max(8, v // 8 * 8) for v in sizes]
    return sizes


def _places(sizes, odd):
    """Where each tensor lies in its flat buffer: 256-element boundaries, or end to end."""
    at, places = 0, []
    for n in sizes:
        places.append(at)
        at += n if odd else (n + 255) // 256 * 256
    return places, at


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(shape, std=1.0, dt=torch.float32):
        return torch.randn(shape, generator=g, device=dev).mul_(std).to(dt)

    s = {"case": case}
    if case["op"] == "norm":
        M, D, dt = case["M"], case["D"], DTYPES[case["dtype"]]
        s["x"] = normal((M, D), 1.0, dt)
        s["residual"] = normal((M, D), 2.0, dt) if case["residual"] else None
        s["weight"] = normal((D,), 0.2).add_(1.0)
        if case["train"]:
            s["gy"] = normal((M, D), 1.0, dt)
            s["gsum"] = normal((M, D), 1.0, dt) if case["residual"] else None
    elif case["op"] == "delta":
        T, B, Hk, Hv, Dk, Dv = (case[k] for k in ("T", "B", "Hk", "Hv", "Dk", "Dv"))
        dt = DTYPES[case["dtype"]]
        lead = {"time": (T, B), "batch": (B, T), "packed": (T,)}[case["layout"]]
        q, k = normal((*lead, Hk, Dk)), normal((*lead, Hk, Dk))
        # keys and queries of unit length, as a model hands them over
        s["q"] = (q / q.square().sum(-1, keepdim=True).sqrt()).to(dt)
        s["k"] = (k / k.square().sum(-1, keepdim=True).sqrt()).to(dt)
        s["v"] = normal((*lead, Hv, Dv), 1.0, dt)
        s["gate"] = -0.05 * torch.exp(normal((*lead, Hv)))
        s["beta"] = torch.sigmoid(normal((*lead, Hv)))
        s["s0"] = normal((B, Hv, Dk, Dv), 0.5)
        s["scale"] = 1.0 / math.sqrt(Dk)
        s["offsets"], s["longest"] = None, T
        if case["layout"] == "packed":
            lens = _lengths(case, seed)
            s["offsets"] = torch.tensor([sum(lens[:i]) for i in range(B + 1)], dtype=torch.int32, device=dev)
            s["longest"] = max(lens)
        if case["train"]:
            s["go"] = normal((*lead, Hv, Dv), 1.0, dt)
            s["glast"] = normal((B, Hv, Dk, Dv), 0.1)
    else:
        sizes = _sizes(case)
        places, n = _places(sizes, case["odd"])
        s["sizes"], s["places"] = sizes, places
        s["p"] = normal(n, 0.05, DTYPES[case["param"]])
        s["g"] = normal(n, 0.01, DTYPES[case["grad"]])
        s["copy"] = torch.zeros(n, dtype=torch.bfloat16, device=dev) if case["copy"] else None
        s["step"] = torch.full((1,), 100, dtype=torch.int64, device=dev)
        if case["state"] == "f32":
            s["m"] = normal(n, 0.003)
            s["v"] = normal(n, 0.01).square_()
        else:       # codes of values around a third of their block's largest
            s["m"] = normal(n, 150.0).clamp_(-448.0, 448.0).to(E4M3)
            s["v"] = normal(n, 150.0).abs_().clamp_(1.0, 448.0).to(E4M3)
            blocks = sum((v + BLOCK - 1) // BLOCK for v in sizes)
            s["scales"] = torch.rand((blocks, 2), generator=g, device=dev).add_(0.5).mul_(
                torch.tensor([2e-5, 6e-5], device=dev))
    return s


def _views(s, name):
    return [s[name][a:a + n] for a, n in zip(s["places"], s["sizes"])]


def _scale_views(s):
    out, at = [], 0
    for n in s["sizes"]:
        b = (n + BLOCK - 1) // BLOCK
        out.append(s["scales"][at:at + b])
        at += b
    return out


def _adamw_out(s, norm):
    out = {"p": s["p"], "m": s["m"], "v": s["v"], "step": s["step"]}
    if s["copy"] is not None:
        out["copy"] = s["copy"]
    if s["case"]["state"] != "f32":
        out["scales"] = s["scales"]
    if s["case"]["clip"]:
        out["norm"] = norm
    return out


# ------------------------------------------------------------------ the library's operators
def _run_own(s):
    from paper_2412_06355_gb300 import binding as b
    c = s["case"]
    if c["op"] == "norm":
        group = {"same": None, "e4m3_row": 0, "e4m3_128": 128}[c["out"]]
        cfg = b.make_norm_config(c["M"], c["D"], c["dtype"], eps=1e-6,
                                 out="same" if group is None else "e4m3", group=group or 0)
        y, total, scale = b.norm_forward(cfg, s["x"], s["weight"], s["residual"])
        out = {"y": y, "sum": total if c["residual"] else None, "scale": scale}
        if c["train"]:
            out.update(b.norm_backward(cfg, total, s["weight"], s["gy"], s["gsum"]))
        return out
    if c["op"] == "delta":
        cfg = b.make_delta_config(c["T"], c["B"], c["Hk"], c["Hv"], c["Dk"], c["Dv"], c["dtype"],
                                  layout=c["layout"], scale=s["scale"])
        if not c["train"]:
            o, last = b.delta_forward(cfg, s["q"], s["k"], s["v"], s["gate"], s["beta"],
                                      s["offsets"], s["s0"], last=s["s0"])
            return {"o": _used(s, o), "last": last}
        saved = b.delta_workspace(cfg)
        o, last = b.delta_forward(cfg, s["q"], s["k"], s["v"], s["gate"], s["beta"], s["offsets"],
                                  s["s0"], saved=saved, want_last=True)
        g = b.delta_backward(cfg, s["q"], s["k"], s["v"], s["gate"], s["beta"], s["go"], s["offsets"],
                             s["s0"], s["glast"], saved=saved)
        return {"o": _used(s, o), "last": last, "gs0": g.pop("gs0"),
                **{n: _used(s, t) for n, t in g.items()}}
    if "plan" not in s:     # an optimizer keeps it
        s["cfg"] = b.make_adamw_config(lr=LR, betas=BETAS, eps=EPS, state=c["state"],
                                       max_norm=1.0 if c["clip"] else 0.0, seed=SEED)
        s["plan"] = b.adamw_plan(s["cfg"], _views(s, "p"), _views(s, "m"), _views(s, "v"),
                                 scales=None if c["state"] == "f32" else _scale_views(s),
                                 copies=_views(s, "copy") if c["copy"] else None,
                                 weight_decay=DECAY)
        s["grads"] = _views(s, "g")
    return _adamw_out(s, b.adamw_step(s["cfg"], s["plan"], s["grads"], s["step"]))


# ------------------------------------------------------------------ the plain forms
def _quantize(y, group):
    """(e4m3 values, scales): the largest of each group of columns becomes 448."""
    M, D = y.shape
    group = group or D
    n = (D + group - 1) // group
    pad = torch.nn.functional.pad(y, (0, n * group - D)).view(M, n, group)
    top = pad.abs().amax(2)
    scale = torch.where(top > 0, top / 448.0, torch.ones_like(top))
    return (pad / scale.unsqueeze(2)).view(M, n * group)[:, :D].to(E4M3), scale


def _plain_norm(s):
    c = s["case"]
    dt = s["x"].dtype
    total = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dt)
    z, w = total.float(), s["weight"]
    r = 1.0 / torch.sqrt(z.square().mean(1, keepdim=True) + 1e-6)
    y = z * r * w
    out = {"sum": total if c["residual"] else None}
    if c["out"] == "same":
        out["y"] = y.to(dt)
    else:
        out["y"], out["scale"] = _quantize(y, 0 if c["out"] == "e4m3_row" else 128)
    if c["train"]:
        g = s["gy"].float()
        h = g * w
        gx = r * (h - z * r.square() * (h * z).mean(1, keepdim=True))
        if s["gsum"] is not None:
            gx = gx + s["gsum"].float()
        out["gx"] = gx.to(dt)
        out["gweight"] = (g * z * r).sum(0)
    return out


def _used(s, t):
    """Rows of a packed tensor behind the last sequence hold nothing."""
    return t if s["offsets"] is None else t[:s["case"]["T"] - min(7, s["case"]["T"] // 8)]


def _token_index(s, pad):
    """[B, L] positions in the flat tokens, and which of them are there; L a multiple of pad."""
    c = s["case"]
    T, B, dev = c["T"], c["B"], s["q"].device
    t = torch.arange((s["longest"] + pad - 1) // pad * pad, device=dev).unsqueeze(0)
    b = torch.arange(B, device=dev).unsqueeze(1)
    if c["layout"] == "packed":
        off = s["offsets"].long()
        return (off[:-1].unsqueeze(1) + t).clamp_max(T - 1), t < (off[1:] - off[:-1]).unsqueeze(1)
    at = t * B + b if c["layout"] == "time" else b * T + t
    return at.clamp_max(T * B - 1), (t < T).expand(B, -1)


def _unit_lower_inverse(A):
    """(I + A)^-1 of strictly lower triangular A, blocks joined by pairs."""
    n = A.shape[-1]
    X = torch.ones((*A.shape[:-2], n, 1, 1), device=A.device, dtype=A.dtype)
    h = 1
    while h < n:
        m = n // (2 * h)
        blocks = A.reshape(*A.shape[:-2], m, 2 * h, m, 2 * h)
        low = torch.diagonal(blocks[..., h:, :, :h], dim1=-4, dim2=-2).movedim(-1, -3)
        X1, X2 = X[..., 0::2, :, :], X[..., 1::2, :, :]
        corner = -(X2 @ (low @ X1))
        X = torch.cat([torch.cat([X1, torch.zeros_like(X1)], -1), torch.cat([corner, X2], -1)], -2)
        h *= 2
    return X.squeeze(-3)


def _delta_chunks(s, q, k, v, gate, beta, s0):
    """o and the last state, in chunks of 64 tokens (of one where a step has one)."""
    c = s["case"]
    C = 64 if s["longest"] > 1 else 1
    Hv, rep = c["Hv"], c["Hv"] // c["Hk"]
    at, there = _token_index(s, C)
    B, L = at.shape
    N = L // C

    def chunks(t):      # [B, H, N, C, ...] with zeros where no token is
        x = t[at] * there.reshape(B, L, *([1] * (t.dim() - 1)))
        return x.transpose(1, 2).reshape(B, x.shape[2], N, C, *x.shape[3:])

    q, k = chunks(q.reshape(-1, c["Hk"], c["Dk"])), chunks(k.reshape(-1, c["Hk"], c["Dk"]))
    q, k = q.repeat_interleave(rep, 1), k.repeat_interleave(rep, 1)
    v = chunks(v.reshape(-1, Hv, c["Dv"]))
    gate, beta = chunks(gate.reshape(-1, Hv)), chunks(beta.reshape(-1, Hv))
    G = gate.double().cumsum(-1)
    lower = torch.ones(C, C, device=q.device, dtype=torch.bool).tril()
    lam = torch.exp((G.unsqueeze(-1) - G.unsqueeze(-2)).masked_fill(~lower, -1e30)).float()
    first, rest = torch.exp(G).float().unsqueeze(-1), torch.exp(G[..., -1:] - G).float().unsqueeze(-1)
    keep = torch.exp(G[..., -1]).float().unsqueeze(-1).unsqueeze(-1)
    kk = (k @ k.transpose(-1, -2)) * lam * beta.unsqueeze(-2)
    X = _unit_lower_inverse(kk.tril(-1))
    P = (q @ k.transpose(-1, -2)) * lam
    E0, W = X @ v, X @ (first * k)
    S, out = s0, []
    for n in range(N):
        u = beta[:, :, n].unsqueeze(-1) * (E0[:, :, n] - W[:, :, n] @ S)
        out.append((first[:, :, n] * q[:, :, n]) @ S + P[:, :, n] @ u)
        S = keep[:, :, n] * S + (rest[:, :, n] * k[:, :, n]).transpose(-1, -2) @ u
    o = (torch.stack(out, 2) * s["scale"]).reshape(B, Hv, L, c["Dv"]).transpose(1, 2)
    return o[there], at[there], S


def _plain_delta(s):
    c = s["case"]
    dt = s["q"].dtype
    ins = [s[n].float().detach() for n in ("q", "k", "v", "gate", "beta", "s0")]
    if c["train"]:
        ins = [t.clone().requires_grad_() for t in ins]
    rows, at, last = _delta_chunks(s, *ins)
    o = torch.zeros((s["v"].numel() // (c["Hv"] * c["Dv"]), c["Hv"], c["Dv"]), device=rows.device)
    o = o.index_copy(0, at, rows).reshape(s["v"].shape)
    out = {"o": _used(s, o.detach().to(dt)), "last": last.detach()}
    if not c["train"]:
        s["s0"].copy_(out["last"])
        out["last"] = s["s0"]
        return out
    upstream = _used(s, s["go"]).float()
    g = torch.autograd.grad((_used(s, o), last), ins, (upstream, s["glast"]))
    out.update({n: _used(s, t.to(dt)) for n, t in zip(("gq", "gk", "gv"), g)})
    out.update(ggate=_used(s, g[3]), gbeta=_used(s, g[4]), gs0=g[5])
    return out


def _mix(h):
    """Scrambles 32-bit integers held in 64 bits: shifts and products with odd digits of sqrt(2) and e."""
    h = ((h ^ (h >> 16)) * 0x6A09E667) & 0xFFFFFFFF
    h = ((h ^ (h >> 15)) * 0xADF85459) & 0xFFFFFFFF
    return h ^ (h >> 16)


def _dither(index, step, n, device):
    """Two uniform numbers in (0, 1) for each element of a tensor, from seed, step and place."""
    start = _mix((_mix((step * 0x9E3779B1 + SEED) & 0xFFFFFFFF) + index) & 0xFFFFFFFF)
    h = _mix((torch.arange(n, device=device) * 0x9E3779B1 + start) & 0xFFFFFFFF)
    return ((h & 0xFFFF).float() + 0.5) / 65536.0, ((h >> 16).float() + 0.5) / 65536.0


def _to_codes(value, u, squared):
    """e4m3 values around value (0 to 448), the upper one where u is below the share that makes
    the expectation of value (or of its square) right."""
    step = torch.exp2((torch.frexp(value.clamp_min(2.0 ** -6)).exponent - 4).float())
    low = torch.floor(value / step) * step
    share = (value - low) * (value + low) / (step * (2.0 * low + step)) if squared else (value - low) / step
    return torch.where(u < share, low + step, low).clamp_max(448.0)


def _encode(x, u, squared):
    n = x.numel()
    blocks = (n + BLOCK - 1) // BLOCK
    pad = torch.nn.functional.pad(x, (0, blocks * BLOCK - n)).view(blocks, BLOCK)
    top = pad.abs().amax(1, keepdim=True)
    scale = top / 448.0
    inverse = torch.where(top > 0, 448.0 / top, torch.zeros_like(top))
    value = (pad * inverse).abs().clamp_max(448.0).view(-1)[:n]
    return (torch.copysign(_to_codes(value, u, squared), x)).to(E4M3), scale.squeeze(1)


def _decode(code, scale):
    return code.float() * scale.repeat_interleave(BLOCK)[:code.numel()]


def _plain_adamw(s):
    c = s["case"]
    norm, factor = None, 1.0
    if c["clip"]:
        squares = torch.stack([g.float().square().sum() for g in _views(s, "g")])
        norm = squares.sum().sqrt().reshape(1)
        factor = torch.where(norm > 1.0, 1.0 / norm, torch.ones_like(norm))
    s["step"] += 1
    t = s["step"].double()
    first, second = -torch.expm1(t * math.log(BETAS[0])), -torch.expm1(t * math.log(BETAS[1]))
    rate, root = (LR / first).float(), second.sqrt().float()
    eight = c["state"] != "f32"
    scales = _scale_views(s) if eight else s["sizes"]
    copies = _views(s, "copy") if c["copy"] else s["sizes"]
    for i, (p, g, m, v, sc, cp) in enumerate(zip(*(_views(s, n) for n in "pgmv"), scales, copies)):
        grad = g.float() * factor
        old_m = _decode(m, sc[:, 0]) if eight else m
        old_v = _decode(v, sc[:, 1]).square() if eight else v
        new_m = old_m + (1.0 - BETAS[0]) * (grad - old_m)
        new_v = old_v + (1.0 - BETAS[1]) * (grad.square() - old_v)
        new_p = p.float() * (1.0 - LR * DECAY) - rate * new_m / (new_v.sqrt() / root + EPS)
        p.copy_(new_p)
        if c["copy"]:
            cp.copy_(new_p)
        if eight:
            um, uv = _dither(i, s["step"], p.numel(), p.device)
            code_m, scale_m = _encode(new_m, um, False)
            code_v, scale_v = _encode(new_v.sqrt(), uv, True)
            m.copy_(code_m)
            v.copy_(code_v)
            sc.copy_(torch.stack([scale_m, scale_v], 1))
        else:
            m.copy_(new_m)
            v.copy_(new_v)
    return _adamw_out(s, norm)


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _plain_norm, "delta": _plain_delta, "adamw": _plain_adamw}[state["case"]["op"]](state)


# ------------------------------------------------------------------ floors
def work(case):
    if case["op"] == "norm":
        n, b = case["M"] * case["D"], 2 if case["dtype"] == "bf16" else 4
        moved = n * b * (3 if case["residual"] else 1) + n * (b if case["out"] == "same" else 1)
        if case["train"]:
            moved += n * b * (4 if case["residual"] else 3)
        return {"bytes": moved, "flops": n * (12 if case["train"] else 4)}
    if case["op"] == "delta":
        b = 2 if case["dtype"] == "bf16" else 4
        tokens = case["T"] * (1 if case["layout"] == "packed" else case["B"])
        qk, vo = 2 * tokens * case["Hk"] * case["Dk"], 2 * tokens * case["Hv"] * case["Dv"]
        states = case["B"] * case["Hv"] * case["Dk"] * case["Dv"] * 4
        gates = tokens * case["Hv"] * 8
        one = tokens * case["Hv"] * case["Dk"] * case["Dv"]
        if not case["train"]:
            return {"bytes": (qk + vo) * b + gates + 2 * states, "flops": 6 * one}
        return {"bytes": 2 * (qk + vo) * b + 2 * gates + 4 * states, "flops": 18 * one}
    n = sum(_sizes(case))
    size = {"f32": 4, "bf16": 2, "e4m3": 1}
    moved = n * (2 * size[case["param"]] + size[case["grad"]] + 4 * size[case["state"]] + (2 if case["copy"] else 0))
    return {"bytes": moved + (n * 16 // BLOCK if case["state"] != "f32" else 0), "flops": 14 * n}


# ------------------------------------------------------------------ 64 bits
def _exact_norm(s):
    c = s["case"]
    z = s["x"].double()
    if c["residual"]:       # the norm is that of the sum as it is handed on, in the inputs' type
        z = (z + s["residual"].double()).to(s["x"].dtype).double()
    w = s["weight"].double()
    power = torch.einsum("md,md->m", z, z) / c["D"] + 1e-6
    unit = z / torch.sqrt(power)[:, None]
    y = unit * w
    out = {"sum": (s["x"].double() + s["residual"].double()) if c["residual"] else None}
    if c["out"] == "same":
        out["y"] = y
    else:
        group = c["D"] if c["out"] == "e4m3_row" else 128
        parts = [(p / (p.abs().amax(1, keepdim=True) / 448.0), p.abs().amax(1) / 448.0)
                 for p in y.split(group, dim=1)]
        out["y"], out["scale"] = torch.cat([p[0] for p in parts], 1), torch.stack([p[1] for p in parts], 1)
    if c["train"]:
        g = s["gy"].double()
        along = torch.einsum("md,d,md->m", g, w, unit) / c["D"]
        gx = (g * w - unit * along[:, None]) / torch.sqrt(power)[:, None]
        out["gx"] = gx + s["gsum"].double() if c["residual"] else gx
        out["gweight"] = torch.einsum("md,md->d", g, unit)
    return out


def _exact_delta(s):
    """The recurrence token by token in float64, states kept every 64 tokens for the way back."""
    c = s["case"]
    at, there = _token_index(s, 1)
    rep = c["Hv"] // c["Hk"]
    L = at.shape[1]

    def by_step(t, d):      # [L, B, H(, d)]
        t = t.reshape(-1, t.shape[-1]) if d is None else t.reshape(-1, t.shape[-2], d)
        return t.double()[at].transpose(0, 1)

    q, k = (by_step(s[n], c["Dk"]).repeat_interleave(rep, 2) for n in ("q", "k"))
    v, gate, beta = by_step(s["v"], c["Dv"]), by_step(s["gate"], None), by_step(s["beta"], None)
    live = there.transpose(0, 1)[..., None].double()            # [L, B, 1]
    decay = torch.exp(gate * live)
    beta = beta * live
    S = s["s0"].double()
    o, err, marks = torch.zeros_like(v), torch.zeros_like(v), []

    def step(S, t):
        S = S * decay[t][..., None, None]
        e = v[t] - torch.einsum("bhk,bhkv->bhv", k[t], S)
        return S + torch.einsum("bhk,bhv->bhkv", k[t], beta[t][..., None] * e), e

    for t in range(L):
        if t % 64 == 0:
            marks.append(S)
        S, err[t] = step(S, t)
        o[t] = s["scale"] * torch.einsum("bhk,bhkv->bhv", q[t], S)

    def back_to_tokens(t, like):
        flat = torch.zeros((like.numel() // t[0, 0].numel(), *t.shape[2:]), dtype=torch.float64, device=t.device)
        flat[at[there]] = t.transpose(0, 1)[there]
        return _used(s, flat.reshape(like.shape))

    out = {"o": back_to_tokens(o, s["v"]), "last": S}
    if not c["train"]:
        return out
    go = by_step(s["go"], c["Dv"]) * live[..., None] * s["scale"]
    gq, gk, gv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    ggate, gbeta = torch.zeros_like(gate), torch.zeros_like(beta)
    D = s["glast"].double()
    for n in range(len(marks) - 1, -1, -1):
        states, S = [], marks[n]
        for t in range(64 * n, min(L, 64 * n + 64)):
            states.append(S)
            S, _ = step(S, t)
        for t in range(min(L, 64 * n + 64) - 1, 64 * n - 1, -1):
            before = states[t - 64 * n]
            gq[t] = torch.einsum("bhkv,bhv->bhk", S, go[t])
            D = D + torch.einsum("bhk,bhv->bhkv", q[t], go[t])
            y = torch.einsum("bhk,bhkv->bhv", k[t], D)
            faded = before * decay[t][..., None, None]
            by = beta[t][..., None] * y
            gk[t] = torch.einsum("bhkv,bhv->bhk", D, beta[t][..., None] * err[t]) - torch.einsum("bhkv,bhv->bhk", faded, by)
            gv[t] = by
            gbeta[t] = (err[t] * y).sum(-1)
            D = D - torch.einsum("bhk,bhv->bhkv", k[t], by)
            ggate[t] = (D * faded).sum((-1, -2))
            D = D * decay[t][..., None, None]
            S = before
    shared = q.shape[:2] + (c["Hk"], rep, c["Dk"])
    out.update(gq=back_to_tokens(gq.reshape(shared).sum(3), s["q"]), gk=back_to_tokens(gk.reshape(shared).sum(3), s["k"]),
               gv=back_to_tokens(gv, s["v"]), ggate=back_to_tokens(ggate, s["gate"]),
               gbeta=back_to_tokens(gbeta * live, s["beta"]), gs0=D)
    return out


def _exact_adamw(s):
    c = s["case"]
    norm, factor = None, 1.0
    if c["clip"]:
        total = 0.0
        for g in _views(s, "g"):
            total += float(torch.linalg.vector_norm(g.double())) ** 2
        norm = torch.tensor([math.sqrt(total)], dtype=torch.float64)
        factor = min(1.0, 1.0 / math.sqrt(total))
    t = int(s["step"]) + 1
    eight = c["state"] != "f32"
    out = {n: s[n].double() for n in "pmv"}     # what lies between the tensors stays
    if c["copy"]:
        out["copy"] = s["copy"].double()
    scales, at = [], 0
    for a, n in zip(s["places"], s["sizes"]):
        g, m, v, p = (s[w][a:a + n].double() for w in "gmvp")
        if eight:
            sc = s["scales"][at:at + (n + BLOCK - 1) // BLOCK].double()
            at += len(sc)
            m, v = m * sc[:, 0].repeat_interleave(BLOCK)[:n], (v * sc[:, 1].repeat_interleave(BLOCK)[:n]) ** 2
        g = g * factor
        m = BETAS[0] * m + (1.0 - BETAS[0]) * g
        v = BETAS[1] * v + (1.0 - BETAS[1]) * g * g
        unit = (m / (1.0 - BETAS[0] ** t)) / (torch.sqrt(v / (1.0 - BETAS[1] ** t)) + EPS)
        out["p"][a:a + n] = p - LR * DECAY * p - LR * unit
        if c["copy"]:
            out["copy"][a:a + n] = out["p"][a:a + n]
        if eight:
            both = []
            for w, x in (("m", m), ("v", v.sqrt())):
                top = torch.stack([y.abs().max() for y in x.split(BLOCK)]) if n < 4096 else torch.cat(
                    [x[:n // BLOCK * BLOCK].view(-1, BLOCK).abs().amax(1)] + ([x[n // BLOCK * BLOCK:].abs().amax()[None]] if n % BLOCK else []))
                both.append(top / 448.0)
                out[w][a:a + n] = x / both[-1].repeat_interleave(BLOCK)[:n]
            scales.append(torch.stack(both, 1))
        else:
            out["m"][a:a + n], out["v"][a:a + n] = m, v
    out["step"] = s["step"] + 1
    if eight:
        out["scales"] = torch.cat(scales)
    if c["clip"]:
        out["norm"] = norm
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "delta": _exact_delta, "adamw": _exact_adamw}[case["op"]](s)
