"""The language-model operators written out from their definitions in 64 bits on the CPU, with the error that a result
may have where the operator computes in 32 bits (`tol_*`: first-order bounds, see each)."""

import torch

D = torch.float64
U32 = 2.0 ** -24            # half a unit in the last place of 1.0, fp32 (24 significant bits); bf16 has 8: 2^-8 (1 + 2^-8 becomes 1)
ROUND = {torch.float32: U32, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126}


def d(t):
    return None if t is None else t.detach().cpu().to(D)


def rows_logp(z, y):
    """(logp [T], softmax [T, V], live [T]); live: the label is in range and some logit is above -inf."""
    z = d(z)
    y = y.cpu().long()
    V = z.shape[1]
    live = (y >= 0) & (y < V) & ~(z == float("-inf")).all(1)
    safe = torch.where(live[:, None], z, torch.zeros((), dtype=D))
    ls = torch.log_softmax(safe, 1)
    logp = ls.gather(1, y.clamp(0, V - 1)[:, None])[:, 0]
    return torch.where(live, logp, torch.zeros((), dtype=D)), ls.exp(), live


def policy(z, y, old, adv, w, ref=None, lo=0.2, hi=0.2, kl_coef=0.0):
    logp, p, live = rows_logp(z, y)
    old, A, w, ref = d(old), d(adv), d(w), d(ref)
    live = live & (w != 0)
    zero = torch.zeros((), dtype=D)
    logp = torch.where(live, logp, zero)
    r = (logp - old).exp()
    lo, hi = 1.0 - float(torch.tensor(lo)), 1.0 + float(torch.tensor(hi))
    up, down = (A > 0) & (r > hi), (A < 0) & (r < lo)
    loss = torch.where(up, -hi * A, torch.where(down, -lo * A, torch.where(A == 0, zero, -r * A)))
    slope = torch.where(up | down | (A == 0), zero, -r * A)
    size = torch.where(up | down, A.abs() * hi, torch.where(A == 0, zero, r * A.abs()))     # what the terms' errors are relative to
    kl = torch.zeros_like(A)
    if ref is not None:
        x = ref - logp
        kl = x.exp() - x - 1.0
        loss, slope, size = loss + kl_coef * kl, slope + kl_coef * (1.0 - x.exp()), size + kl_coef * (x.exp() + x.abs() + 1.0)
    keep = lambda v: torch.where(live, v, zero)  # noqa: E731
    g = keep(w * slope)
    grad = torch.where(live[:, None], -g[:, None] * p, zero)
    yy = y.cpu().long().clamp(0, p.shape[1] - 1)
    grad[torch.arange(len(yy)), yy] += g
    return {"loss": (keep(w * loss)).sum(), "kl": keep(w * kl).sum(), "clipped": keep(w * (up | down)).sum(), "logp": logp, "dlogits": grad,
            "live": live, "size": keep(w.abs() * size), "kl_size": keep(w.abs() * (torch.ones_like(A) if ref is None else x.exp() + x.abs() + 1.0))}


def logp_error(z, logp):
    """Bound of the error of an fp32 logp: the exponentials' relative error (1e-6 covers the base-2 exponential's 2^-22 and
    the roundings of its argument, each term weighted by its share) and that of their sum (a thread adds at most some 64 pieces,
    then a tree: 100 roundings), which the logarithm turns into an absolute one, and two roundings of numbers of logp's size."""
    z = d(z)
    span = torch.where(torch.isfinite(z), z, torch.zeros((), dtype=D)).abs().amax(1)
    return 1e-6 + 100 * U32 + 4 * U32 * (logp.abs() + span)


def preference(z, y, offsets, ref, beta=0.1, smoothing=0.0, scale=None):
    T = z.shape[0]
    logp, p, live = rows_logp(z, y)
    at = offsets.cpu().long().clamp(0, T).tolist()
    n = len(at) // 2
    scale = (1.0 / n if n else 0.0) if scale is None else scale
    beta, smoothing, scale = (float(torch.tensor(v)) for v in (beta, smoothing, scale))
    s = torch.stack([logp[a:max(a, b)].sum() for a, b in zip(at[:-1], at[1:])]) if n else torch.zeros(0, dtype=D)
    m = s - d(ref)
    h = beta * (m[0::2] - m[1::2])
    ls = torch.nn.functional.logsigmoid
    pair = -(1 - smoothing) * ls(h) - smoothing * ls(-h)
    c = scale * beta * (torch.sigmoid(h) - (1 - smoothing))
    g = torch.zeros(T, dtype=D)
    for q in range(2 * n):
        g[at[q]:max(at[q], at[q + 1])] = c[q // 2] if q % 2 == 0 else -c[q // 2]
    g = torch.where(live, g, torch.zeros((), dtype=D))
    grad = torch.where(live[:, None], -g[:, None] * p, torch.zeros((), dtype=D))
    grad[torch.arange(T), y.cpu().long().clamp(0, p.shape[1] - 1)] += g
    return {"loss": scale * pair.sum(), "pair_loss": pair, "seq_logp": s, "dlogits": grad, "logp": logp, "h": h, "at": at, "g": g}


def gate_of(gate):
    return None if gate is None else d(gate) if gate.dim() == 1 else torch.sigmoid(d(gate))


def residual(x, h, w_pre, w_post=None, gate=None, scale=1.0, eps=1e-6):
    x, h, w_pre, w_post, G = d(x), d(h), d(w_pre), d(w_post), gate_of(gate)
    rms = lambda v: (v.square().mean(1, keepdim=True) + eps).sqrt()  # noqa: E731
    u = h if w_post is None else h / rms(h) * w_post
    gu = u if G is None else G * u
    y = scale * x + gu
    n = y / rms(y) * w_pre
    # relative error of each factor: the mean of squares adds about width / 256 + 16 numbers one after the other (at most
    # 80 roundings), the rest a handful; sigmoid's exponential 2e-7.  2e-5 covers 160 roundings and twice the exponential.
    e = 2e-5
    tol_y = e * ((scale * x).abs() + gu.abs())
    tol_n = e * n.abs() + tol_y / rms(y) * w_pre.abs() + n.abs() * (tol_y * y.abs()).mean(1, keepdim=True) / rms(y) ** 2
    return y, n, tol_y, tol_n


def residual_backward(dn, dy, y, h, w_pre, w_post=None, gate=None, scale=1.0, eps=1e-6):
    dn, dy, y, h, w_pre, w_post, G = d(dn), d(dy), d(y), d(h), d(w_pre), d(w_post), gate_of(gate)
    mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    rms = lambda v: (mean(v.square()) + eps).sqrt()  # noqa: E731
    e = 2e-5                                        # as in residual()
    ry = 1 / rms(y)
    a, yn = dn * w_pre, y * ry
    dY = ry * (a - yn * mean(a * yn))
    t = ry * (a.abs() + yn.abs() * mean((a * yn).abs()))
    if dy is not None:
        dY, t = dY + dy, t + dy.abs()
    t = e * t
    out, tol = {"dx": scale * dY}, {"dx": abs(scale) * t}
    out["dw_pre"], tol["dw_pre"] = (dn * yn).sum(0), e * (dn * yn).abs().sum(0)
    hn = h / rms(h)
    u = h if w_post is None else hn * w_post
    if G is not None and G.dim() == 1:
        out["dgate"], tol["dgate"] = (dY * u).sum(0), (t * u.abs() + e * (dY * u).abs()).sum(0)
    elif G is not None:
        k = u * G * (1 - G)
        # 1 - sigmoid is a difference: its error is that of 1
        out["dgate"], tol["dgate"] = dY * k, t * k.abs() + e * (dY * u * G).abs()
    dU, tU = (dY, t) if G is None else (dY * G, t * G.abs() + e * (dY * G).abs())
    if w_post is None:
        out["dh"], tol["dh"] = dU, tU
    else:
        out["dw_post"], tol["dw_post"] = (dU * hn).sum(0), (tU * hn.abs() + e * (dU * hn).abs()).sum(0)
        b, tb, rh = dU * w_post, tU * w_post.abs(), 1 / rms(h)
        out["dh"] = rh * (b - hn * mean(b * hn))
        tol["dh"] = rh * (tb + hn.abs() * mean(tb * hn.abs())) + e * rh * (b.abs() + hn.abs() * mean((b * hn).abs()))
    return out, tol


def pack(x):
    """(q [T, W], e [T, W / 32]) as integers, from the definition: e by search over the powers of two."""
    x = d(x)
    T, width = x.shape
    W = (width + 31) // 32 * 32
    full = torch.zeros(T, W, dtype=D)
    full[:, :width] = x
    b = full.view(T, W // 32, 32)
    top = b.abs().amax(2)
    bad = ~torch.isfinite(b).all(2)
    top = torch.where(bad, torch.zeros((), dtype=D), top)
    powers = torch.tensor([127.0 * 2.0 ** (e - 127) for e in range(255)], dtype=D)
    e = torch.searchsorted(powers, top.contiguous())       # the first power that is at least top
    e = torch.where(bad, torch.full_like(e, 255), e)
    q = torch.round(torch.where(bad[..., None], torch.zeros((), dtype=D), b) * torch.exp2(127.0 - torch.where(bad, torch.zeros_like(e), e).to(D))[..., None])
    return q.view(T, W), e


def unpack(q, e, width):
    s = torch.exp2(e.to(D) - 127.0)
    s = torch.where(e == 255, torch.full_like(s, float("nan")), s)
    return (q.to(D).view(q.shape[0], -1, 32) * s[..., None]).view(q.shape[0], -1)[:, :width]


def close(got, want, tol, name=""):
    """|got - want| <= tol + the rounding of got's type, element by element; infinities and NaN in the same places."""
    g, r = d(got), ROUND[got.dtype]
    assert g.shape == want.shape, (name, g.shape, want.shape)
    tol = torch.as_tensor(tol, dtype=D).expand(want.shape)
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(g[odd]), torch.isnan(want[odd])), f"{name}: NaN in other places"
    err = (g - want)[~odd].abs()
    bound = (tol + (want.abs() + tol) * r + TINY[got.dtype] * 2)[~odd]
    if err.numel():
        worst = float((err / bound).max())
        assert worst <= 1.0, f"{name}: {worst:.3g} times the bound (largest error {float(err.max()):.3g})"
