"""Embedding, layer norm, linear layer and gated recurrence written out from their definitions in 64 bits on the CPU, with the
error that a result may have where the operator computes in 32 bits (first-order bounds, see each)."""

import math

import torch

from tests.llm_reference import ROUND, U32, d

D = torch.float64


def embed(ids, table, scale):
    ids, table = ids.cpu().long(), d(table)
    known = (ids >= 0) & (ids < table.shape[0])
    return torch.where(known[:, None], scale * table[ids.clamp(0, table.shape[0] - 1)], torch.zeros((), dtype=D))


def embed_backward(dy, ids, vocab, scale):
    """The gradient, and its error: a row's sum has at most as many additions as tokens, and one product."""
    ids, dy = ids.cpu().long(), d(dy)
    at = torch.where((ids >= 0) & (ids < vocab), ids, torch.full_like(ids, vocab))
    out, size = torch.zeros(vocab + 1, dy.shape[1], dtype=D), torch.zeros(vocab + 1, dy.shape[1], dtype=D)
    live = torch.where((at < vocab)[:, None], dy, torch.zeros((), dtype=D))
    out.index_add_(0, at, live)
    size.index_add_(0, at, live.abs())
    count = torch.bincount(at, minlength=vocab + 1)[:-1, None]
    return scale * out[:-1], (count + 2) * U32 * abs(scale) * size[:-1]


E = 160 * U32            # a sum over a row: at most 32 numbers one after the other in a thread, then trees; 160 roundings cover it


def layer_norm(x, w, b, eps):
    x, w, b = d(x), d(w), d(b)
    mean = x.mean(1, keepdim=True)
    c = x - mean
    r = 1 / (c.square().mean(1, keepdim=True) + eps).sqrt()
    off = E * x.abs().mean(1, keepdim=True) + U32 * x.abs()                    # of c
    er = E + (c.abs() * off).mean(1, keepdim=True) * r ** 2                    # of r, relative
    n = c * r * w
    tol = (off * r * w.abs()) + n.abs() * (er + 4 * U32)
    if b is not None:
        n = n + b
        tol = tol + U32 * n.abs()
    return n, tol, (c, r, off, er)


def layer_norm_backward(dn, x, w, skip, eps):
    _, _, (c, r, off, er) = layer_norm(x, w, None, eps)
    dn, w, skip = d(dn), d(w), d(skip)
    mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    a, xh = dn * w, c * r
    dx = r * (a - mean(a) - xh * mean(a * xh))
    size = r * (a.abs() + mean(a.abs()) + xh.abs() * mean((a * xh).abs()))
    tol = (3 * er + 2 * E) * size + r * (off * r * mean((a * xh).abs()) + xh.abs() * mean(a.abs() * off * r))
    if skip is not None:
        dx, tol = dx + skip, tol + U32 * skip.abs() + U32 * dx.abs()
    rows = x.shape[0] / 148 + 200                                             # additions of a column sum, one after the other
    out = {"dx": dx, "dw": (dn * xh).sum(0), "db": dn.sum(0)}
    tols = {"dx": tol, "dw": (dn.abs() * (off * r + xh.abs() * (er + 4 * U32))).sum(0) + rows * U32 * (dn * xh).abs().sum(0),
            "db": rows * U32 * dn.abs().sum(0)}
    return out, tols


def phi(z):
    return 0.5 * torch.erfc(-z * math.sqrt(0.5))          # keeps its precision in the lower tail


def act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros((), dtype=D))
    if name == "gelu":
        return z * phi(z)
    return z * torch.sigmoid(z) if name == "silu" else z


def slope(name, z):
    if name == "relu":
        return (z > 0).to(D)
    if name == "gelu":
        return phi(z) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(z)
    return s * (1 + z * torch.sigmoid(-z)) if name == "silu" else torch.ones_like(z)


# A product of bf16 numbers is exact in fp32.  The tensor core drops the bits below the 24 of an accumulator at each of its additions,
# 16 products at a time, 48 times until the sum is taken over: 64 steps of 2^-23 of the terms' sum cover that and the additions after it.
SUM = 64 * 2.0 ** -23
ACT = 1e-5               # of an activation or slope, of |z| <= 20: the fast exponential's 2 + 1.2 |z| units in the last place, and a few


def product(a, b):
    """a b with its error."""
    a, b = d(a), d(b)
    return a @ b, SUM * (a.abs() @ b.abs())


def linear(x, w, b, name, res):
    z, tol = product(x, w)
    if b is not None:
        z, tol = z + d(b), tol + U32 * (z + d(b)).abs()
    y = act(name, z)
    ty = 1.2 * tol + ACT * (y.abs() + (z.abs() < 20) * 1e-3 if name != "none" else 0 * z)
    if res is not None:
        y, ty = y + d(res), ty + U32 * (y + d(res)).abs()
    return y, ty, z, tol


def dgrad(dy, w, name, z, res):
    v, tol = product(dy, d(w).t())
    if name != "none":
        s = slope(name, d(z))
        # gelu's and silu's slopes are sums of terms of up to one half of opposite signs: 1e-6 of the size that the product has
        v, tol = v * s, tol * s.abs() + ACT * (v * s).abs() + 1e-6 * v.abs()
    if res is not None:
        v, tol = v + d(res), tol + U32 * (v + d(res)).abs()
    return v, tol


GATE = 2e-6              # of a and of 1 - a, |g| <= 12: the exponential's 2^-22 and its argument's rounding, |g| 2^-24, and the division


def scan(a, b, s):
    """Rows of s_t = a_t s_{t-1} + b_t, and of its error: every row's factors and sums are right to GATE."""
    out, err, e = torch.empty_like(b), torch.empty_like(b), torch.zeros_like(s)
    size = s.abs()
    for t in range(a.shape[0]):
        s, size = a[t] * s + b[t], a[t] * size + b[t].abs()
        e = a[t] * e + GATE * size
        out[t], err[t] = s, e
    return out, err


def bounds(offsets, T, seqs):
    at = [0, T] if offsets is None else offsets.cpu().clamp(0, T).tolist()
    return [(at[q], max(at[q], at[q + 1])) for q in range(seqs)]


def recurrence(x, g, offsets, h0, kind):
    x, g, h0 = d(x), d(g), d(h0)
    T, W = x.shape
    seqs = 1 if offsets is None else offsets.numel() - 1
    a, rest = torch.sigmoid(g), torch.sigmoid(-g)
    b = x * rest if kind == "blend" else x
    y, ey = torch.zeros(T, W, dtype=D), torch.zeros(T, W, dtype=D)
    last, el = torch.zeros(seqs, W, dtype=D), torch.zeros(seqs, W, dtype=D)
    for q, (i, j) in enumerate(bounds(offsets, T, seqs)):
        s = torch.zeros(W, dtype=D) if h0 is None else h0[q]
        last[q] = s
        if j > i:
            y[i:j], ey[i:j] = scan(a[i:j], b[i:j], s)
            last[q], el[q] = y[j - 1], ey[j - 1]
    return y, ey, last, el


def recurrence_backward(dy, x, g, y, offsets, h0, dlast, kind):
    dy, x, g, y, h0, dlast = d(dy), d(x), d(g), d(y), d(h0), d(dlast)
    T, W = x.shape
    seqs = 1 if offsets is None else offsets.numel() - 1
    a, rest = torch.sigmoid(g), torch.sigmoid(-g)
    zero = lambda n: torch.zeros(n, W, dtype=D)  # noqa: E731
    out, tol = {"dx": zero(T), "dg": zero(T), "dh0": zero(seqs)}, {"dx": zero(T), "dg": zero(T), "dh0": zero(seqs)}
    for q, (i, j) in enumerate(bounds(offsets, T, seqs)):
        behind = torch.zeros(W, dtype=D) if dlast is None else dlast[q]
        out["dh0"][q] = behind
        if j == i:
            continue
        # e_t = a_t (dy_t + e_{t+1}) from the end
        e, ee = scan(a[i:j].flip(0), (a[i:j] * dy[i:j]).flip(0), behind)
        e, ee = e.flip(0), ee.flip(0)
        dd = dy[i:j] + torch.cat((e[1:], behind[None]))
        ed = torch.cat((ee[1:], torch.zeros(1, W, dtype=D))) + U32 * (dy[i:j].abs() + (dd - dy[i:j]).abs())
        before = torch.cat((torch.zeros(1, W, dtype=D) if h0 is None else h0[q:q + 1], y[i:j - 1]))
        k, z = a[i:j], rest[i:j]
        diff = before - x[i:j] if kind == "blend" else before
        out["dx"][i:j] = dd * z if kind == "blend" else dd
        tol["dx"][i:j] = (ed * z + 2 * GATE * (dd * z).abs()) if kind == "blend" else ed
        out["dg"][i:j] = dd * diff * k * z
        tol["dg"][i:j] = k * z * (ed * diff.abs() + dd.abs() * (6 * GATE * diff.abs() + U32 * (before.abs() + x[i:j].abs())))
        out["dh0"][q], tol["dh0"][q] = e[0], ee[0]
    return out, tol


def close(got, want, tol, name=""):
    """got (rounded once to its type from a number within tol of want) against want."""
    r = ROUND[got.dtype]
    err = (d(got) - want).abs()
    lim = tol + r * (want.abs() + tol) * (0 if got.dtype == torch.float32 else 1) + 2 * U32 * want.abs() + 2.0 ** -126
    bad = ~(err <= lim)
    assert not bad.any(), (name, int(bad.sum()), float((err / lim.clamp(min=1e-300)).nan_to_num(1e9).max()))
