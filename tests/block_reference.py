"""Plain float64 references of the operators of a token block: norm with residual, gated delta rule,
AdamW over many tensors. Nothing here is shared with the library."""
import math

import torch

U32 = 2.0 ** -24           # half a step of float32, relative
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}


def within(name, got, want, bound):
    """Element by element; the outputs' own rounding is part of `bound`."""
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / bound.clamp_min(1e-300)).max()):.3g} of the bound"


# ------------------------------------------------------------------ norm
def norm(x, residual, w, eps):
    """(sum as handed on, y before its rounding, r) in float64."""
    z = x if residual is None else (x.double() + residual.double()).to(x.dtype)
    # the sum of two float32 (or bfloat16) values is exact in float64, so this rounds once as the library does
    r = 1.0 / torch.sqrt(z.double().square().mean(-1, keepdim=True) + eps)
    return z, z.double() * r * w.double(), r


def norm_backward(z, w, gy, gsum, eps):
    """(gx, gweight) in float64 with bounds of their float32 evaluation (without the output's rounding)."""
    z, w, g = z.double(), w.double(), gy.double()
    D = z.shape[-1]
    r = 1.0 / torch.sqrt(z.square().mean(-1, keepdim=True) + eps)
    h = g * w
    along = (h * z).mean(-1, keepdim=True)
    gx = r * (h - z * r.square() * along)
    # a sum of D products is off by at most (D + 1) U32 of their magnitudes; r carries half of that
    c = (D + 16) * U32
    mag = (h * z).abs().mean(-1, keepdim=True)
    bound = r * (h.abs() * c + z.abs() * r.square() * (mag + along.abs() * 2) * c)
    if gsum is not None:
        gx = gx + gsum.double()
        bound = bound + gsum.double().abs() * 2 * U32
    rows = g.numel() // D
    gw = (g * z * r).reshape(-1, D).sum(0)
    gw_bound = (g * z * r).abs().reshape(-1, D).sum(0) * (c + rows * U32)
    return gx, bound, gw, gw_bound


# ------------------------------------------------------------------ gated delta rule
def sequences(layout, T, B, offsets):
    """Flat token indices of every sequence."""
    if layout == "packed":
        return [list(range(offsets[b], offsets[b + 1])) for b in range(B)]
    return [[t * B + b if layout == "time" else b * T + t for t in range(T)] for b in range(B)]


def delta(q, k, v, gate, beta, s0, seqs, scale, marks=None):
    """(o, last) token by token, differentiable; q, k [N, Hk, Dk], v [N, Hv, Dv], gate, beta [N, Hv],
    s0 [B, Hv, Dk, Dv]. Tokens of no sequence have o = 0. marks: a list that receives (tokens, state as
    the tokens behind them take it) of every 64 tokens of a sequence."""
    rep = v.shape[1] // k.shape[1]
    q, k = q.repeat_interleave(rep, 1), k.repeat_interleave(rep, 1)
    rows, lasts = {}, []
    for b, seq in enumerate(seqs):
        S = s0[b]
        for i, t in enumerate(seq):
            S = S * torch.exp(gate[t])[:, None, None]
            u = beta[t][:, None] * (v[t] - torch.einsum("hk,hkv->hv", k[t], S))
            S = S + torch.einsum("hk,hv->hkv", k[t], u)
            rows[t] = scale * torch.einsum("hk,hkv->hv", q[t], S)
            if marks is not None and (i % 64 == 63 or i + 1 == len(seq)):
                S = S * 1.0
                marks.append((seq[i // 64 * 64:i + 1], S))
        lasts.append(S)
    zero = torch.zeros_like(v[0]) if v.shape[0] else v
    o = torch.stack([rows.get(t, zero) for t in range(v.shape[0])]) if v.shape[0] else v
    return o, torch.stack(lasts)


# ------------------------------------------------------------------ AdamW
def adamw(p, g, m, v, t, lr, betas, eps, decay, factor=1.0):
    """(p, m, v) after step t, in float64."""
    g = g.double() * factor
    m = betas[0] * m.double() + (1.0 - betas[0]) * g
    v = betas[1] * v.double() + (1.0 - betas[1]) * g * g
    unit = (m / (1.0 - betas[0] ** t)) / (torch.sqrt(v / (1.0 - betas[1] ** t)) + eps)
    return p.double() * (1.0 - lr * decay) - lr * unit, m, v


def decoded(codes, scale):
    """Values of e4m3 codes with a scale for each 256."""
    return codes.double() * scale.double().repeat_interleave(256)[:codes.numel()]


def spacing(value):
    """Distance of the e4m3 neighbours around value (0 to 448)."""
    return torch.exp2(torch.floor(torch.log2(value.clamp_min(2.0 ** -6))) - 3)


def log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
