"""Gated linear recurrence, its gradients and its single step against their definitions in 64 bits."""

import pytest
import torch

from tests import llm_layers_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def normal(*s, seed, dtype="f32", scale=1.0, mean=0.0):
    return (mean + scale * torch.randn(*s, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)).to(DT[dtype])


def offs(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def check(llm, x, g, offsets, h0, kind, dtype, dlast=True, llm_kw=None):
    seqs = 1 if offsets is None else offsets.numel() - 1
    T, W = x.shape
    r = llm.gated_recurrence(x, g, offsets, h0=h0, kind=kind)
    y, ey, last, el = R.recurrence(x, g, offsets, h0, kind)
    R.close(r.y, y, ey, "y")
    R.close(r.last, last, el, "last")
    dy = normal(T, W, seed=90, dtype=dtype)
    dl = normal(seqs, W, seed=91) if dlast else None
    b = llm.gated_recurrence_backward(dy, x, g, r.y, offsets, h0=h0, dlast=dl, kind=kind, dh0=torch.empty(seqs, W, device=DEV))
    want, tol = R.recurrence_backward(dy, x, g, r.y, offsets, h0, dl, kind)
    for k in want:
        R.close(getattr(b, k), want[k], tol[k], k)
    again = llm.gated_recurrence_backward(dy, x, g, r.y, offsets, h0=h0, dlast=dl, kind=kind)
    assert torch.equal(again.dx, b.dx) and torch.equal(again.dg, b.dg) and (again.dh0 is None) == (h0 is None)
    llm.check()
    return r, b


# around a warp's rows, a tile, a group of tiles; columns around a lane's pair and a strip
@pytest.mark.parametrize("T,W", [(1, 1), (1, 64), (2, 3), (15, 2), (16, 31), (17, 64), (127, 65), (128, 33), (129, 130), (300, 7), (1000, 66), (4096, 20), (4097, 64), (5000, 3),
                                 (9000, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["blend", "add"])
def test_one_sequence(llm, T, W, dtype, kind):
    x, g = normal(T, W, seed=1, dtype=dtype), normal(T, W, seed=2, dtype=dtype, scale=1.5, mean=2.0)
    check(llm, x, g, None, None, kind, dtype, dlast=False)
    check(llm, x, g, None, normal(1, W, seed=3), kind, dtype)


CUTS = [(300, (0, 300)), (300, (0, 1, 2, 300)), (300, (0, 16, 32, 128, 129, 299, 300)), (300, (5, 40, 40, 40, 250)), (300, (0, 0, 0, 300, 300, 300)), (300, (7, 7, 7)),
        (300, (-4, 100, 400)), (300, (300, 300)), (64, tuple(range(65))), (6000, (0, 4500, 4600, 6000)), (6000, (100, 101, 5999)), (5000, (0,) + tuple(range(3, 5000, 37)))]


@pytest.mark.parametrize("T,cuts", CUTS, ids=[f"{t}-{len(c) - 1}" for t, c in CUTS])
@pytest.mark.parametrize("dtype,kind,W,state", [("bf16", "blend", 66, True), ("f32", "add", 5, True), ("bf16", "add", 33, False)])
def test_packed_sequences(llm, T, cuts, dtype, kind, W, state):
    """Short, empty and long sequences, rows in front of the first and behind the last."""
    offsets = offs(*cuts)
    x, g = normal(T, W, seed=T, dtype=dtype), normal(T, W, seed=2, dtype=dtype, scale=1.5, mean=2.0)
    h0 = normal(len(cuts) - 1, W, seed=3) if state else None
    lo, hi = max(0, min(T, cuts[0])), max(0, min(T, cuts[-1]))
    outside = torch.ones(T, dtype=torch.bool, device=DEV)
    outside[lo:max(lo, hi)] = False
    x[outside], g[outside] = float("nan"), float("inf")            # rows of no sequence are not read
    clean_x, clean_g = x.clone(), g.clone()
    clean_x[outside], clean_g[outside] = 0, 0
    r, b = check(llm, clean_x, clean_g, offsets, h0, kind, dtype)
    got = llm.gated_recurrence(x, g, offsets, h0=h0, kind=kind)
    assert torch.equal(got.y, r.y) and torch.equal(got.last, r.last) and (got.y[outside] == 0).all()
    spoiled = r.y.clone()
    spoiled[outside] = float("nan")
    dy, dl = normal(T, W, seed=90, dtype=dtype), normal(len(cuts) - 1, W, seed=91)
    dy[outside] = float("nan")
    back = llm.gated_recurrence_backward(dy, x, g, spoiled, offsets, h0=h0, dlast=dl, kind=kind)
    assert torch.equal(back.dx, b.dx) and torch.equal(back.dg, b.dg)


@pytest.mark.parametrize("kind", ["blend", "add"])
def test_no_sequence_reaches_the_next(llm, kind):
    """NaN and infinities of one sequence, also across tiles and groups, leave the others as they are."""
    T, W = 9500, 34
    offsets = offs(0, 200, 5000, 5001, 5130, 9500)
    x, g = normal(T, W, seed=1), normal(T, W, seed=2, mean=2.0)
    h0 = normal(5, W, seed=3)
    clean = llm.gated_recurrence(x, g, offsets, h0=h0, kind=kind)
    dy, dl = normal(T, W, seed=4), normal(5, W, seed=5)
    back = llm.gated_recurrence_backward(dy, x, g, clean.y, offsets, h0=h0, dlast=dl, kind=kind)
    bx, bg, bh = x.clone(), g.clone(), h0.clone()
    bx[300, 3], bg[301, 4], bh[1, 5], bx[210, 6], bg[5000, 7] = float("nan"), float("nan"), float("inf"), float("-inf"), float("nan")
    got = llm.gated_recurrence(bx, bg, offsets, h0=bh, kind=kind)
    keep = torch.ones(T, dtype=torch.bool, device=DEV)
    keep[200:5001] = False
    assert torch.equal(got.y[keep], clean.y[keep]) and torch.equal(got.last[[0, 3, 4]], clean.last[[0, 3, 4]])
    assert got.y[4999, 3].isnan() and got.y[4999, 4].isnan() and not got.last[1, 3:7].isfinite().any() and got.last[2, 7].isnan()
    bd, bl = dy.clone(), dl.clone()
    bd[4000, 3], bl[1, 5] = float("nan"), float("inf")
    b = llm.gated_recurrence_backward(bd, bx, bg, got.y, offsets, h0=bh, dlast=bl, kind=kind)
    assert torch.equal(b.dx[keep], back.dx[keep]) and torch.equal(b.dg[keep], back.dg[keep]) and torch.equal(b.dh0[[0, 3, 4]], back.dh0[[0, 3, 4]])
    assert b.dx[200, 3].isnan()


@pytest.mark.parametrize("mean", [-30.0, -100.0, 30.0, 100.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gates_that_are_shut_or_open(llm, mean, dtype):
    """Gates near 0 and 1: the state forgets at once, or keeps all; 1 - a stays right to its own size."""
    T, W = 500, 40
    x, g = normal(T, W, seed=1, dtype=dtype), normal(T, W, seed=2, dtype=dtype, mean=mean)
    r = llm.gated_recurrence(x, g, None, h0=normal(1, W, seed=3))
    a = torch.sigmoid(R.d(g))
    h, want = R.d(normal(1, W, seed=3))[0], []
    for t in range(T):
        h = a[t] * h + torch.sigmoid(-R.d(g[t])) * R.d(x[t])
        want.append(h)
    # 500 roundings of the state where nothing is forgotten; the exponential of an argument of 100 is right to 100 2^-24 + 2^-22
    R.close(r.y, torch.stack(want), torch.tensor(500 * 5 * R.U32 + 1e-5 * 5 * 2.0 ** -20).double() + 1e-5 * torch.sigmoid(-R.d(g)) * R.d(x).abs())
    assert r.y.isfinite().all()
    shut = torch.full((T, W), float("-inf"), device=DEV)
    assert torch.allclose(llm.gated_recurrence(x.float(), shut).y, x.float(), rtol=1e-6, atol=1e-30)
    assert torch.equal(llm.gated_recurrence(x.float(), -shut, None, h0=torch.ones(1, W, device=DEV)).y, torch.ones(T, W, device=DEV))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift,pad", [(0, 6), (1, 0), (1, 5), (2, 2), (0, 3)])
def test_slices(llm, dtype, shift, pad):
    T, W = 400, 70
    offsets = offs(3, 150, 390)

    def at(values=None):
        buf = torch.full((T * (W + pad) + shift + 8,), 9.0, device=DEV, dtype=DT[dtype])
        v = buf[shift:shift + T * (W + pad)].view(T, W + pad)[:, :W]
        if values is not None:
            v.copy_(values)
        return buf, v

    x, g, dy = (at(normal(T, W, seed=i))[1] for i in (1, 2, 3))
    by, y = at()
    llm.gated_recurrence(x, g, offsets, y=y)
    R.close(y, *R.recurrence(x, g, offsets, None, "blend")[:2])
    (bx, dx), (bg, dg) = at(), at()
    kept = y.clone()
    llm.gated_recurrence_backward(dy, x, g, y, offsets, dx=dx, dg=dg)
    want, tol = R.recurrence_backward(dy, x, g, kept, offsets, None, None, "blend")
    R.close(dx, want["dx"], tol["dx"])
    R.close(dg, want["dg"], tol["dg"])
    for b, v in ((by, y), (bx, dx), (bg, dg)):
        v.fill_(9.0)
        assert (b == 9).all()


@pytest.mark.parametrize("T", [100, 5000])
def test_in_place(llm, T):
    W, offsets = 66, offs(0, T // 3, T // 3, T)
    x, g, dy = (normal(T, W, seed=i, dtype="bf16") for i in (1, 2, 3))
    h0, dl = normal(3, W, seed=4), normal(3, W, seed=5)
    r = llm.gated_recurrence(x, g, offsets, h0=h0)
    for i in range(2):
        a = [x.clone(), g.clone()]
        q = llm.gated_recurrence(a[0], a[1], offsets, h0=h0, y=a[i])
        assert torch.equal(a[i], r.y) and torch.equal(q.last, r.last)
    b = llm.gated_recurrence_backward(dy, x, g, r.y, offsets, h0=h0, dlast=dl)
    for i, j in ((0, 1), (1, 0), (0, 2), (1, 2), (2, 0), (2, 1)):
        a = [dy.clone(), x.clone(), g.clone()]
        q = llm.gated_recurrence_backward(a[0], a[1], a[2], r.y, offsets, h0=h0, dlast=dl, dx=a[i], dg=a[j])
        assert torch.equal(a[i], b.dx) and torch.equal(a[j], b.dg) and torch.equal(q.dh0, b.dh0)


@pytest.mark.parametrize("kind", ["blend", "add"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,W", [(1, 1), (3, 7), (16, 2048), (5, 257), (40000, 2)])
def test_step(llm, kind, dtype, S, W):
    """One row for each sequence is what the packed form makes of sequences of one row."""
    x, g, h = normal(S, W, seed=1, dtype=dtype), normal(S, W, seed=2, dtype=dtype, mean=2.0), normal(S, W, seed=3)
    r = llm.gated_recurrence_step(x, g, h, kind=kind)
    y, ey, last, el = R.recurrence(x.view(1, -1), g.view(1, -1), None, h.view(1, -1), kind)
    R.close(r.y.view(1, -1), y, ey)
    R.close(r.last.view(1, -1), last, el)
    spare = h.clone()
    q = llm.gated_recurrence_step(x, g, spare, kind=kind, out=spare)
    assert torch.equal(spare, r.last) and torch.equal(q.y, r.y)


def test_steps_continue_a_sequence(llm):
    T, W = 40, 96
    x, g = normal(T, W, seed=1), normal(T, W, seed=2, mean=1.0)
    whole = llm.gated_recurrence(x, g)
    h = llm.gated_recurrence(x[:30], g[:30]).last
    for t in range(30, T):
        r = llm.gated_recurrence_step(x[t:t + 1], g[t:t + 1], h, out=h)
        # the same ten steps from states that differ by their roundings
        assert (r.y[0] - whole.y[t]).abs().max() <= 1e-5
    halves = llm.gated_recurrence(torch.cat((x, x)), torch.cat((g, g)), offs(0, T, 2 * T))
    assert torch.equal(halves.y[:T], whole.y)


def test_nothing_at_all(llm):
    none = torch.zeros(0, 6, device=DEV)
    h0 = normal(2, 6, seed=1)
    r = llm.gated_recurrence(none, none, offs(0, 0, 0), h0=h0)
    assert r.y.shape == (0, 6) and torch.equal(r.last, h0)
    assert (llm.gated_recurrence(none, none).last == 0).all()
    assert llm.gated_recurrence(none, none, offs(0)).last.shape == (0, 6)
    b = llm.gated_recurrence_backward(none, none, none, none, offs(0, 0, 0), h0=h0, dlast=h0)
    assert torch.equal(b.dh0, h0)
    x = normal(10, 6, seed=2)
    assert (llm.gated_recurrence(x, x, offs(0)).y == 0).all()


def test_against_differences(llm):
    T, W, offsets = 11, 3, offs(1, 5, 5, 10)
    x, g, dy = (normal(T, W, seed=i) for i in (1, 2, 3))
    h0, dl = normal(3, W, seed=4), normal(3, W, seed=5)
    for kind in ("blend", "add"):
        y = llm.gated_recurrence(x, g, offsets, h0=h0, kind=kind).y
        b = llm.gated_recurrence_backward(dy, x, g, y, offsets, h0=h0, dlast=dl, kind=kind)
        v = [R.d(t) for t in (x, g, h0)]

        def loss():
            y, _, last, _ = R.recurrence(v[0], v[1], offsets, v[2], kind)
            return (y * R.d(dy)).sum() + (last * R.d(dl)).sum()

        for t, grad in zip(v, (b.dx, b.dg, b.dh0)):
            flat, out = t.view(-1), R.d(grad).view(-1)
            for i in range(flat.numel()):
                keep = float(flat[i])
                flat[i] = keep + 1e-5
                up = loss()
                flat[i] = keep - 1e-5
                down = loss()
                flat[i] = keep
                assert abs(float(up - down) / 2e-5 - float(out[i])) < 2e-5          # the kernel's fp32 error; the differences' is 1e-9
