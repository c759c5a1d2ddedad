"""Layer norm and its gradients against their definitions in 64 bits."""

import pytest
import torch

from tests import llm_layers_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = float(torch.tensor(1e-5))


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rows(T, W, dtype, seed, mean=0.5):
    x = 3.0 * torch.randn(T, W, generator=gen(seed), device=DEV) + mean
    x[:, :: max(1, W // 8)] *= 12.0
    return x.to(DT[dtype])


def weights(W):
    return 1.0 + 0.1 * torch.randn(W, generator=gen(70), device=DEV), 0.1 * torch.randn(W, generator=gen(71), device=DEV)


SIZES = [(1, 1), (1, 2), (2, 7), (5, 8), (3, 31), (9, 100), (17, 256), (33, 300), (9, 384), (700, 40), (40, 385), (7, 1024), (300, 1000), (11, 1537), (400, 2048), (20, 4096),
         (10, 8192), (6, 8200), (5, 10000), (4, 16384), (4, 16392), (3, 20001), (2, 32768), (5000, 64), (1500, 520)]


@pytest.mark.parametrize("T,W", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bias", [True, False])
def test_forward(llm, T, W, dtype, bias):
    x, (w, b) = rows(T, W, dtype, T + W), weights(W)
    b = b if bias else None
    n = llm.layer_norm(x, w, b)
    want, tol, _ = R.layer_norm(x, w, b, EPS)
    R.close(n, want, tol)


@pytest.mark.parametrize("T,W", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("skip", [True, False])
def test_backward(llm, T, W, dtype, skip):
    x, (w, _) = rows(T, W, dtype, T + W), weights(W)
    dn = torch.randn(T, W, generator=gen(3), device=DEV).to(DT[dtype])
    sk = torch.randn(T, W, generator=gen(4), device=DEV).to(DT[dtype]) if skip else None
    got = llm.layer_norm_backward(dn, x, w, dskip=sk)
    want, tol = R.layer_norm_backward(dn, x, w, sk, EPS)
    for k in want:
        R.close(getattr(got, k), want[k], tol[k], k)
    again = llm.layer_norm_backward(dn, x, w, dskip=sk, bias=False)
    assert again.db is None and torch.equal(again.dx, got.dx) and torch.equal(again.dw, got.dw)
    base = torch.randn(2, W, generator=gen(5), device=DEV)
    acc = base.clone()
    llm.layer_norm_backward(dn, x, w, dskip=sk, dw=acc[0], db=acc[1], accumulate=True)
    for i, k in enumerate(("dw", "db")):
        R.close(acc[i], R.d(base[i]) + want[k], tol[k] + R.U32 * (R.d(base[i]).abs() + want[k].abs()), k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("W", [40, 130, 1000, 1537])
@pytest.mark.parametrize("place", [(0, 0, 0, 0), (1, 1, 1, 1), (3, 3, 3, 3), (0, 1, 0, 0), (2, 0, 4, 1), (8, 8, 8, 8)])
def test_rows_at_any_alignment(llm, dtype, W, place):
    """x, dn, dskip and the output start at these elements of rows that are 11 elements longer than needed."""
    T, L = 50, W + 11
    dt = DT[dtype]
    w, b = weights(W)

    def at(shift, values=None):
        buf = torch.full((T * L + 16,), 9.0, device=DEV, dtype=dt)
        v = buf[shift:shift + T * L].view(T, L)[:, :W]
        if values is not None:
            v.copy_(values)
        return buf, v

    x = at(place[0], rows(T, W, dtype, 5))[1]
    dn = at(place[1], torch.randn(T, W, generator=gen(6), device=DEV))[1]
    sk = at(place[2], torch.randn(T, W, generator=gen(7), device=DEV))[1]
    buf, n = at(place[3])
    llm.layer_norm(x, w, b, n=n)
    want, tol, _ = R.layer_norm(x, w, b, EPS)
    R.close(n, want, tol)
    got = llm.layer_norm_backward(dn, x, w, dskip=sk, dx=n)
    want, tol = R.layer_norm_backward(dn, x, w, sk, EPS)
    for k in want:
        R.close(getattr(got, k), want[k], tol[k], k)
    n.fill_(9.0)
    assert (buf == 9).all()                                   # nothing beside the rows was written


@pytest.mark.parametrize("W", [96, 1000, 8200])
def test_in_place(llm, W):
    T = 30
    x, (w, b) = rows(T, W, "bf16", 1), weights(W)
    dn, sk = (torch.randn(T, W, generator=gen(i), device=DEV).bfloat16() for i in (2, 3))
    n, g = llm.layer_norm(x, w, b), llm.layer_norm_backward(dn, x, w, dskip=sk)
    y = x.clone()
    assert torch.equal(llm.layer_norm(y, w, b, n=y), n)
    for i in range(3):
        a = [dn.clone(), x.clone(), sk.clone()]
        r = llm.layer_norm_backward(a[0], a[1], w, dskip=a[2], dx=a[i])
        assert torch.equal(r.dx, g.dx) and torch.equal(r.dw, g.dw) and torch.equal(r.db, g.db)


@pytest.mark.parametrize("W", [200, 1024, 20000])
def test_a_large_common_offset(llm, W):
    """Rows around 300 with a spread of 1: x^2 - mean^2 would leave three digits of the variance."""
    x = (300.0 + torch.randn(8, W, generator=gen(2), device=DEV))
    w, b = weights(W)
    want, tol, _ = R.layer_norm(x, w, b, EPS)
    R.close(llm.layer_norm(x, w, b), want, tol)


@pytest.mark.parametrize("W", [300, 512, 1000, 4096, 4100, 8192])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_whose_samples_are_far_from_the_rest(llm, W, dtype):
    """32 elements at equal distances far above the others, every start of the pattern, and rows that are zero but for one element."""
    T = 2 * (W // 32) if W <= 1000 else 150
    x = torch.randn(T, W, generator=gen(8), device=DEV)
    for t in range(T):
        x[t, t % (W // 32):: W // 32] += 3000.0
    x[3] = 0.0
    x[3, W // 2] = 100.0
    x = x.to(DT[dtype])
    w, b = weights(W)
    want, tol, _ = R.layer_norm(x, w, b, EPS)
    R.close(llm.layer_norm(x, w, b), want, tol)
    dn = torch.randn(T, W, generator=gen(9), device=DEV).to(DT[dtype])
    want, tol = R.layer_norm_backward(dn, x, w, None, EPS)
    got = llm.layer_norm_backward(dn, x, w)
    for k in want:
        R.close(getattr(got, k), want[k], tol[k], k)


def test_rows_with_what_is_no_number(llm):
    """A NaN or an infinity spoils its own row and the column sums, no other row."""
    T, W = 40, 512
    x, (w, b) = rows(T, W, "f32", 1), weights(W)
    dn = torch.randn(T, W, generator=gen(2), device=DEV)
    clean, back = llm.layer_norm(x, w, b), llm.layer_norm_backward(dn, x, w)
    x[7, 3], x[20, 500] = float("nan"), float("inf")
    n, g = llm.layer_norm(x, w, b), llm.layer_norm_backward(dn, x, w)
    bad = torch.zeros(T, dtype=torch.bool, device=DEV)
    bad[[7, 20]] = True
    assert n[7].isnan().all() and n[20].isnan().any()
    assert torch.equal(n[~bad], clean[~bad]) and torch.equal(g.dx[~bad], back.dx[~bad])
    assert torch.equal(g.db, back.db)


def test_constant_rows_and_no_rows(llm):
    w, b = weights(300)
    n = llm.layer_norm(torch.full((3, 300), 2.5, device=DEV), w, b)
    # the mean is right to a rounding of 2.5 (E of it), which 1 / sqrt(eps) = 316 enlarges
    assert (n - b).abs().max() <= 2.5 * R.E * 317 * 1.5
    none = torch.zeros(0, 300, device=DEV)
    assert llm.layer_norm(none, w, b).shape == (0, 300)
    g = llm.layer_norm_backward(none, none, w)
    assert (g.dw == 0).all() and (g.db == 0).all()
    kept = torch.ones(300, device=DEV)
    llm.layer_norm_backward(none, none, w, bias=False, dw=kept, accumulate=True)
    assert (kept == 1).all()


def test_against_differences(llm):
    T, W = 3, 12
    x, (w, b) = torch.randn(T, W, generator=gen(1), device=DEV, dtype=torch.float64), weights(W)
    dn, sk = (torch.randn(T, W, generator=gen(i), device=DEV) for i in (2, 3))
    g = llm.layer_norm_backward(dn, x.float(), w, dskip=sk)

    def loss(x, w, b):
        return (R.layer_norm(x, w, b, EPS)[0] * R.d(dn)).sum() + (R.d(x) * R.d(sk)).sum()

    x, w, b = R.d(x.float()), R.d(w), R.d(b)
    for name, at, grad in (("x", x, g.dx), ("w", w, g.dw), ("b", b, g.db)):
        flat, out = at.view(-1), R.d(grad).view(-1)
        for i in range(flat.numel()):
            keep = float(flat[i])
            flat[i] = keep + 1e-5
            up = loss(x, w, b)
            flat[i] = keep - 1e-5
            down = loss(x, w, b)
            flat[i] = keep
            assert abs(float(up - down) / 2e-5 - float(out[i])) < 2e-5, name      # the kernel's fp32 error; the differences' is 1e-9
