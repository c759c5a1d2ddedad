"""Linear layer, its gradients and the activations against their definitions in 64 bits."""

import pytest
import torch

from tests import llm_layers_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def normal(*s, seed, dtype=BF, scale=1.0):
    return (scale * torch.randn(*s, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)).to(dtype)


# one token to several tiles; widths that are no multiple of 8, of 64, of 256; a K of one, of part of a run, of more than twelve and of many
# runs (cut along K where there are few tiles); more tiles than pairs of SMs
SIZES = [(1, 1, 1), (1, 8, 8), (2, 16, 40), (3, 5, 7), (17, 64, 64), (7, 100, 24), (64, 65, 33), (100, 200, 300), (129, 768, 257), (255, 1000, 130), (256, 256, 256), (257, 264, 520),
         (515, 1000, 1111), (16, 4096, 512), (40, 1600, 1000), (5, 8200, 70), (300, 832, 1024), (3000, 72, 2600), (2500, 1608, 2064)]


@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("act,dtype,extras", [("none", BF, True), ("gelu", BF, True), ("silu", torch.float32, True), ("relu", torch.float32, False), ("none", torch.float32, False)])
def test_forward(llm, T, K, N, act, dtype, extras):
    x, w = normal(T, K, seed=1), normal(K, N, seed=2, scale=K ** -0.5)
    b = normal(N, seed=3, dtype=torch.float32) if extras else None
    res = normal(T, N, seed=4, dtype=dtype) if extras else None
    y, ty, z, tz = R.linear(x, w, b, act, res)
    r = llm.linear(x, w, b, act=act, residual=res, keep=True, dtype=dtype)
    assert r.y.dtype == dtype and r.z.dtype == BF
    R.close(r.y, y, ty, "y")
    R.close(r.z, z, tz, "z")
    again = llm.linear(x, w, b, act=act, residual=res, dtype=dtype)
    assert again.z is None and torch.equal(again.y, r.y)
    if res is not None:
        spare = res.clone()
        assert torch.equal(llm.linear(x, w, b, act=act, residual=spare, dtype=dtype, y=spare).y, r.y)
    llm.check()


@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("act,dtype,extras", [("none", BF, False), ("gelu", BF, True), ("silu", torch.float32, True), ("relu", BF, False)])
def test_dgrad(llm, T, K, N, act, dtype, extras):
    dy, w = normal(T, N, seed=1), normal(K, N, seed=2, scale=N ** -0.5)
    z = None if act == "none" else normal(T, K, seed=3, scale=2.0)
    res = normal(T, K, seed=4, dtype=dtype) if extras else None
    want, tol = R.dgrad(dy, w, act, z, res)
    dx = llm.linear_dgrad(dy, w, act=act, z=z, residual=res, dtype=dtype)
    assert dx.dtype == dtype
    R.close(dx, want, tol)
    if z is not None and dtype == BF:
        spare = z.clone()
        assert torch.equal(llm.linear_dgrad(dy, w, act=act, z=spare, residual=res, dx=spare), dx)
    llm.check()


@pytest.mark.parametrize("T,K,N", SIZES)
def test_wgrad(llm, T, K, N):
    x, dy = normal(T, K, seed=1), normal(T, N, seed=2)
    want, tol = R.product(x.t(), dy)
    r = llm.linear_wgrad(x, dy, bias=True)
    R.close(r.dw, want, tol, "dw")
    if want.norm() > 0:      # the same accumulations measured 1.6e-7 of the norm in the 8-bit weight gradient
        assert float((R.d(r.dw) - want).norm() / want.norm()) < 1e-6
    db, tb = R.d(dy).sum(0), (T / 8 + 64) * R.U32 * R.d(dy).abs().sum(0)
    R.close(r.db, db, tb, "db")
    only = llm.linear_wgrad(x, dy)
    assert only.db is None and torch.equal(only.dw, r.dw)
    base, vec = normal(K, N, seed=5, dtype=torch.float32), normal(N, seed=6, dtype=torch.float32)
    acc, accb = base.clone(), vec.clone()
    llm.linear_wgrad(x, dy, bias=True, dw=acc, db=accb, accumulate=True)
    R.close(acc, R.d(base) + want, tol + R.U32 * (R.d(base).abs() + want.abs()), "dw +=")
    R.close(accb, R.d(vec) + db, tb + R.U32 * (R.d(vec).abs() + db.abs()), "db +=")
    llm.check()


@pytest.mark.parametrize("place", [(0, 0, 0, 0), (1, 3, 5, 2), (8, 16, 8, 8), (8, 8, 1, 8)])
@pytest.mark.parametrize("T,K,N,pad", [(70, 136, 200, 8), (33, 65, 77, 3), (300, 264, 512, 16)])
def test_slices(llm, place, T, K, N, pad):
    """Operands and outputs inside wider buffers, at addresses that TMA cannot or can start at; what lies beside stays."""
    def at(rows, cols, shift, dtype=BF, values=None):
        buf = torch.full((rows * (cols + pad) + 32,), 9.0, device=DEV, dtype=dtype)
        v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        if values is not None:
            v.copy_(values)
        return buf, v

    x = at(T, K, place[0], values=normal(T, K, seed=1))[1]
    w = at(K, N, place[1], values=normal(K, N, seed=2, scale=K ** -0.5))[1]
    res = at(T, N, place[2], values=normal(T, N, seed=3))[1]
    b = normal(N + 1, seed=4, dtype=torch.float32)[1:]
    y, ty, z, tz = R.linear(x, w, b, "gelu", res)
    (by, oy), (bz, oz) = at(T, N, place[3]), at(T, N, place[2])
    llm.linear(x, w, b, act="gelu", residual=res, keep=True, y=oy, z=oz)
    R.close(oy, y, ty, "y")
    R.close(oz, z, tz, "z")
    dy = at(T, N, place[0], values=normal(T, N, seed=5))[1]
    zin = at(T, K, place[3], values=normal(T, K, seed=6))[1]
    bx, ox = at(T, K, place[1])
    llm.linear_dgrad(dy, w, act="silu", z=zin, dx=ox)
    R.close(ox, *R.dgrad(dy, w, "silu", zin, None), "dx")
    bw, ow = at(K, N, place[2], torch.float32)
    llm.linear_wgrad(x, dy, dw=ow)
    R.close(ow, *R.product(x.t(), dy), "dw")
    for buf, v in ((by, oy), (bz, oz), (bx, ox), (bw, ow)):
        v.fill_(9.0)
        assert (buf == 9).all()
    llm.check()


def test_columns_of_one_buffer(llm):
    """Input and output as columns of one buffer: rows that interleave, elements that do not."""
    T, K, N = 90, 128, 64
    buf = normal(T, K + N, seed=1)
    w = normal(K, N, seed=2, scale=K ** -0.5)
    y, ty, *_ = R.linear(buf[:, :K], w, None, "none", None)
    llm.linear(buf[:, :K], w, y=buf[:, K:])
    R.close(buf[:, K:], y, ty)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu", "none"])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("T,W,shift", [(1, 1, 0), (5, 7, 0), (33, 64, 0), (40, 129, 1), (300, 1000, 0), (64, 256, 8)])
def test_activation_backward(llm, act, dtype, T, W, shift):
    dy = normal(T * W + shift, seed=1, dtype=dtype)[shift:].view(T, W)
    z = normal(T * W + shift, seed=2, scale=3.0)[shift:].view(T, W)
    want = R.d(dy) * R.slope(act, R.d(z))
    got = llm.activation_backward(dy, z, act)
    R.close(got, want, R.ACT * R.d(dy).abs() * (1 + R.slope(act, R.d(z)).abs()))
    spare = z.clone()
    assert torch.equal(llm.activation_backward(dy, spare, act, dz=spare), got)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_tails_of_the_activations(llm, act):
    """Values from -20 to 20 through the layer (weight 1), relative to themselves where the definition is small."""
    z = torch.linspace(-20, 20, 801, device=DEV).bfloat16()[:, None]
    one = torch.ones(1, 1, device=DEV, dtype=BF)
    y = llm.linear(z, one, act=act, dtype=torch.float32).y
    want = R.act(act, R.d(z))
    assert ((R.d(y) - want).abs() <= 1e-5 * want.abs() + 2.0 ** -126).all()
    s = llm.linear_dgrad(torch.ones_like(z), one, act=act, z=z, dtype=torch.float32)
    sl = R.slope(act, R.d(z))
    # a slope is a sum of two terms of opposite signs below zero: relative to the terms
    size = sl.abs() if act != "gelu" else R.phi(R.d(z)) + R.d(z).abs() * torch.exp(-0.5 * R.d(z) ** 2)
    size = size if act != "silu" else torch.sigmoid(R.d(z)) * (1 + R.d(z).abs())
    assert ((R.d(s) - sl).abs() <= 3e-5 * size + 2.0 ** -126).all()


def test_what_is_no_number_stays_in_its_row_or_column(llm):
    T, K, N = 70, 200, 300
    x, w, dy = normal(T, K, seed=1), normal(K, N, seed=2), normal(T, N, seed=3)
    y, dx = llm.linear(x, w).y, llm.linear_dgrad(dy, w)
    bad = x.clone()
    bad[11, 5] = float("nan")
    got = llm.linear(bad, w).y
    keep = torch.arange(T, device=DEV) != 11
    assert got[11].isnan().all() and torch.equal(got[keep], y[keep])
    worse = dy.clone()
    worse[3, 7] = float("inf")
    got = llm.linear_dgrad(worse, w)
    keep = torch.arange(T, device=DEV) != 3
    assert not got[3].isfinite().any() and torch.equal(got[keep], dx[keep])


def test_no_tokens(llm):
    none, w = torch.zeros(0, 16, device=DEV, dtype=BF), normal(16, 24, seed=1)
    assert llm.linear(none, w, keep=True).z.shape == (0, 24)
    assert llm.linear_dgrad(torch.zeros(0, 24, device=DEV, dtype=BF), w).shape == (0, 16)
    r = llm.linear_wgrad(none, torch.zeros(0, 24, device=DEV, dtype=BF), bias=True)
    assert (r.dw == 0).all() and (r.db == 0).all()


def test_layer_against_differences(llm):
    """Gradients of sum(y c) through two layers, by differences of the definitions in 64 bits."""
    T, K, H, N = 6, 5, 9, 4
    x, w1, w2 = normal(T, K, seed=1), normal(K, H, seed=2, scale=0.5), normal(H, N, seed=3, scale=0.5)
    b1, b2, c = normal(H, seed=4, dtype=torch.float32), normal(N, seed=5, dtype=torch.float32), normal(T, N, seed=6)
    first = llm.linear(x, w1, b1, act="gelu", keep=True)
    dz = llm.linear_dgrad(c, w2, act="gelu", z=first.z)
    g1, g2, dx = llm.linear_wgrad(x, dz, bias=True), llm.linear_wgrad(first.y, c, bias=True), llm.linear_dgrad(dz, w1)
    v = [R.d(t) for t in (x, w1, b1, w2, b2)]

    def loss():
        h = R.act("gelu", v[0] @ v[1] + v[2])
        return ((h @ v[3] + v[4]) * R.d(c)).sum()

    for t, grad in zip(v, (dx, g1.dw, g1.db, g2.dw, g2.db)):
        flat, out = t.view(-1), R.d(grad).view(-1)
        for i in range(flat.numel()):
            keep = float(flat[i])
            flat[i] = keep + 1e-5
            up = loss()
            flat[i] = keep - 1e-5
            down = loss()
            flat[i] = keep
            # z, y and dz are bf16: three roundings of 2^-8 on the way, of gradients that add up at most nine terms of about two
            assert abs(float(up - down) / 2e-5 - float(out[i])) < 3 * 2.0 ** -8 * 18
