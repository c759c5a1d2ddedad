"""Gates of fp32 sequences are as exact as fp32 arithmetic makes them."""

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


@pytest.mark.parametrize("how", ["step", "rows"])
def test_gates_near_one(llm, how):
    """a = 1 / (1 + e) with e = exp(-g) < 0.007: 1 + e is off by 2^-24 at most (and what e is off by, two units of 2^-23 of it), the quotient, which
    is between 1/2 and 1, by 2^-25; a state of 1 with nothing added to it is the gate."""
    W = 1 << 18
    g = torch.linspace(5.0, 18.0, W, device=DEV)[None].contiguous()
    one, zero = torch.ones_like(g), torch.zeros_like(g)
    if how == "step":
        a = llm.gated_recurrence_step(zero, g, one, kind="add").last
    else:
        a = llm.gated_recurrence(zero, g, h0=one, kind="add").last
    e = torch.exp(-g.double())
    err = (a.double() - 1 / (1 + e)).abs()
    assert bool((err <= 2.0 ** -24 + 2.0 ** -25 + e * 2.0 ** -22).all()), float(err.max() * 2 ** 24)


def test_a_state_behind_many_gates(llm):
    """16384 rows that keep 0.9991 of the state each and add nothing: every row is off by what its gate is (1.5 units of 2^-24) and a rounding."""
    T, W = 16384, 64
    g = (7.0 + 0.3 * torch.randn(T, W, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)).contiguous()
    h0 = torch.ones(1, W, device=DEV)
    last = llm.gated_recurrence(torch.zeros_like(g), g, h0=h0, kind="add").last
    want = torch.sigmoid(g.double()).log().sum(0).exp()
    assert bool(((last[0].double() - want).abs() <= T * (1.6 + 1.0) * 2.0 ** -24 * want).all())
