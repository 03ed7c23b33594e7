"""Plain float64 references of the token-sequence operators, and first-order error bounds of
their float32 evaluation. Nothing here is shared with the library."""
import torch

U32 = 2.0 ** -24           # unit roundoff of float32
U16 = 2.0 ** -8            # unit roundoff of bfloat16 (8 bits of significand)


def rounding(dtype, ref):
    """Bound of the one rounding to the output's dtype."""
    return (U16 if dtype == torch.bfloat16 else U32) * ref.abs()


# ------------------------------------------------------------------ embedding
def embed_backward(ids, grad, V, scale, padding_id):
    """(grad_table, bound): a sum of c terms in float32, in any order, is off by at most c U32
    times the sum of magnitudes; one more rounding for the scale, twice that for safety."""
    D = grad.shape[-1]
    ids, g = ids.reshape(-1).long(), grad.reshape(-1, D).double()
    ok = (ids >= 0) & (ids < V)
    if padding_id is not None:
        ok &= ids != padding_id
    out = torch.zeros(V, D, dtype=torch.float64, device=g.device).index_add_(0, ids[ok], g[ok])
    mag = torch.zeros_like(out).index_add_(0, ids[ok], g[ok].abs())
    c = torch.bincount(ids[ok], minlength=V).double().unsqueeze(1)
    return out * scale, 2 * (c + 1) * U32 * mag * abs(scale) + rounding(grad.dtype, out * scale)


# ------------------------------------------------------------------ gated scan
def scan(x, gate, starts, h0, gh, glast, kind, mix, layout):
    """Forward and backward step by step in float64, with bounds. Returns dict name ->
    (value, bound). Every step's decay, complement and products are off by a few roundings of
    their own (exp, the sum, the quotient, the product: at most 8 U32 in all, 16 with safety),
    which the recurrence carries on like the values' magnitudes."""
    if layout == "batch":
        f = lambda t: None if t is None else t.transpose(0, 1)
        out = scan(f(x), f(gate), f(starts), h0, f(gh), glast, kind, mix, "time")
        return {k: (f(v), f(b)) if k in ("h", "gx", "ggate") else (v, b)
                for k, (v, b) in out.items()}
    T, B, N = x.shape
    dt = x.dtype
    x, g = x.double(), gate.double()
    a = torch.sigmoid(g) if kind == "logit" else g
    na = torch.sigmoid(-g) if kind == "logit" else 1 - g
    na_abs = na.abs() + (0 if kind == "logit" else U32 * (1 + g.abs()))
    live = torch.ones(T, B, 1, dtype=torch.bool, device=x.device)
    if starts is not None:
        live = (starts == 0).unsqueeze(2)
    comp = mix == "complement"
    v = torch.zeros(B, N, dtype=torch.float64, device=x.device) if h0 is None else h0.double()
    mag, err = v.abs(), torch.zeros_like(v)
    h, prev, pmag, perr, herr = (torch.empty_like(x) for _ in range(5))
    c = 16 * U32
    for t in range(T):
        prev[t] = torch.where(live[t], v, 0.0)
        pmag[t] = torch.where(live[t], mag, 0.0)
        perr[t] = torch.where(live[t], err, 0.0)
        u = na[t] * x[t] if comp else x[t]
        v = torch.where(live[t], a[t] * prev[t] + u, u)
        mag = a[t].abs() * pmag[t] + u.abs()
        err = a[t].abs() * perr[t] + c * mag
        h[t], herr[t] = v, err
    out = {"h": (h, herr + rounding(dt, h)), "last": (v, err + U32 * v.abs())}
    if gh is None:
        return out
    gx, gg, gxe, gge = (torch.empty_like(x) for _ in range(4))
    mu = torch.zeros_like(v) if glast is None else glast.double()
    mmag, merr = mu.abs(), torch.zeros_like(mu)
    for t in reversed(range(T)):
        lam = gh[t].double() + mu
        lmag = gh[t].double().abs() + mmag
        lerr = merr + c * lmag
        w = na[t] if comp else torch.ones_like(lam)
        hp = prev[t] - x[t] if comp else prev[t]
        hpm = pmag[t] + (x[t].abs() if comp else 0)
        d = a[t] * na[t] if kind == "logit" else torch.ones_like(lam)
        gx[t] = lam * w
        gxe[t] = (lerr + c * lmag) * (na_abs[t] if comp else 1)
        gg[t] = lam * hp * d
        gge[t] = (lerr * hpm + lmag * (perr[t] + c * hpm) + c * lmag * hpm) * d.abs()
        mu = torch.where(live[t], a[t] * lam, 0.0)
        mmag = torch.where(live[t], a[t].abs() * lmag, 0.0)
        merr = torch.where(live[t], a[t].abs() * lerr, 0.0) + c * mmag
    out.update(gx=(gx, gxe + rounding(dt, gx)), ggate=(gg, gge + rounding(dt, gg)),
               gh0=(mu, merr + U32 * mu.abs()))
    return out


# ------------------------------------------------------------------ cross entropy
def xent(hidden, weight, labels, ignore, gloss=None):
    """Loss and gradients in float64, with bounds. Returns dict name -> (value, bound).

    A logit is a float32 sum of D exact (bfloat16) or 2^-22-accurate (float32) products; its
    roundings, of at most 2^-23 of the running magnitude each, are independent in sign, so
    4 sqrt(D) of them bound the sum (16 sigma / 4). G is rounded to bfloat16 for bfloat16
    inputs. exp, the sum of exponentials and the logarithm add 2^-19 of the magnitudes."""
    dt = hidden.dtype
    M, D = hidden.shape
    V = weight.shape[0]
    keep = (labels != ignore) & (labels >= 0) & (labels < V)
    H = torch.where(keep.unsqueeze(1), hidden.double(), 0.0)
    W = weight.double()
    y = torch.where(keep, labels.long(), 0).unsqueeze(1)
    logits = H @ W.t()
    e_l = 4 * (D ** 0.5 + 1) * 2.0 ** -23 * (H.abs() @ W.abs().t())
    lse = torch.logsumexp(logits, 1)
    e_lse = e_l.max(1).values + 2.0 ** -19 * (1 + lse.abs())
    picked = logits.gather(1, y).squeeze(1)
    loss = torch.where(keep, lse - picked, 0.0)
    bad = ~keep & (labels != ignore)
    loss[bad] = float("nan")
    out = {"loss": (loss, torch.where(keep, e_lse + e_l.gather(1, y).squeeze(1) + 2 * U32 * picked.abs(), 0.0))}
    if gloss is None:
        return out
    c = torch.where(keep, gloss.double(), 0.0).unsqueeze(1)
    p = torch.exp(logits - lse.unsqueeze(1))
    rel = e_l + e_lse.unsqueeze(1) + 2.0 ** -21 * (1 + (logits - lse.unsqueeze(1)).abs())
    G = p.scatter_add(1, y, torch.full_like(p[:, :1], -1.0)) * c
    e_G = c.abs() * (p * rel + U32) + (U16 * G.abs() if dt == torch.bfloat16 else 4 * U32 * G.abs())
    e_G = torch.where(keep.unsqueeze(1), e_G, 0.0)
    gh, gw = G @ W, G.t() @ H
    acc_h = 4 * (V ** 0.5 + 1) * 2.0 ** -23 * (G.abs() @ W.abs())
    acc_w = 4 * (M ** 0.5 + 1) * 2.0 ** -23 * (G.abs().t() @ H.abs())
    b_h = e_G @ W.abs() + acc_h + rounding(dt, gh)
    b_w = e_G.t() @ H.abs() + acc_w + rounding(dt, gw)
    gh[bad] = float("nan")
    out.update(ghidden=(gh, b_h), gweight=(gw, b_w))
    return out


def check(name, got, want):
    """Every element within its bound; NaN exactly where the reference has NaN."""
    ref, bound = want
    got = got.double().to(ref.device)
    assert got.shape == ref.shape, name
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(got), nan), f"{name}: NaN in other places"
    off = torch.where(nan, 0.0, (got - ref).abs() - bound)
    tiny = 1e-37               # a subnormal that is flushed, or 0 against 0
    assert bool((off <= tiny).all()), \
        f"{name}: off by {(got - ref).abs()[off > tiny].max():.3e}, worst excess {off.max():.3e}"
