"""A gated recurrence whose state is infinite: no gate is zero, so it stays infinite, however many rows lie behind, and the other sequences
and channels do not see it."""

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
INF = float("inf")


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def normal(*s, seed, dtype):
    return torch.randn(*s, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(DT[dtype])


# rows inside a warp's, of a tile, of several tiles and segments; gates whose product falls below the smallest number after some 150 and 30 rows
@pytest.mark.parametrize("T,W", [(40, 64), (600, 64), (2000, 130), (20000, 20), (3000, 7)])
@pytest.mark.parametrize("gate", [0.0, -5.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["blend", "add"])
def test_an_infinite_state_stays(llm, T, W, gate, dtype, kind):
    x, g = normal(2 * T + 9, W, seed=1, dtype=dtype), (gate + 0.1 * normal(2 * T + 9, W, seed=2, dtype="f32")).to(DT[dtype])
    offsets = torch.tensor([0, T, T + 9, 2 * T + 9], dtype=torch.int32, device=DEV)
    h0 = torch.zeros(3, W, device=DEV)
    clean = llm.gated_recurrence(x, g, offsets, h0=h0, kind=kind)
    bad = h0.clone()
    bad[0, ::2] = INF
    bad[2, 1::3] = -INF
    r = llm.gated_recurrence(x, g, offsets, h0=bad, kind=kind)
    assert (r.y[:T, ::2] == INF).all() and (r.last[0, ::2] == INF).all()
    assert (r.y[T + 9:, 1::3] == -INF).all() and (r.last[2, 1::3] == -INF).all()
    keep = torch.ones(2 * T + 9, W, dtype=torch.bool, device=DEV)
    keep[:T, ::2] = False
    keep[T + 9:, 1::3] = False
    assert torch.equal(r.y[keep], clean.y[keep])
    # an input that is infinite: from its row on
    late = x.clone()
    late[T // 3, 0] = INF
    r = llm.gated_recurrence(late, g, offsets, h0=h0, kind=kind)
    assert (r.y[T // 3:T, 0] == INF).all() and torch.equal(r.y[:T // 3], clean.y[:T // 3]) and torch.equal(r.y[T:], clean.y[T:])


@pytest.mark.parametrize("T,W", [(40, 64), (600, 64), (2000, 130), (20000, 20), (3000, 7)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["blend", "add"])
def test_an_infinite_gradient_stays(llm, T, W, dtype, kind):
    x, g, dy = (normal(T + 9, W, seed=i, dtype=dtype) for i in (1, 2, 3))
    g = (0.1 * g.float()).to(DT[dtype])
    offsets = torch.tensor([0, 9, T + 9], dtype=torch.int32, device=DEV)
    h0 = torch.zeros(2, W, device=DEV)
    y = llm.gated_recurrence(x, g, offsets, h0=h0, kind=kind).y
    clean = llm.gated_recurrence_backward(dy, x, g, y, offsets, h0=h0, dlast=torch.zeros_like(h0), kind=kind)
    dlast = torch.zeros_like(h0)
    dlast[1, ::2] = -INF
    r = llm.gated_recurrence_backward(dy, x, g, y, offsets, h0=h0, dlast=dlast, kind=kind)
    assert (r.dx[9:, ::2] == -INF).all() and (r.dh0[1, ::2] == -INF).all()
    for k in ("dx", "dg"):
        a, b = getattr(r, k), getattr(clean, k)
        assert torch.equal(a[:9], b[:9]) and torch.equal(a[:, 1::2], b[:, 1::2]), k
    assert torch.equal(r.dh0[0], clean.dh0[0]) and torch.equal(r.dh0[:, 1::2], clean.dh0[:, 1::2])
