"""The linear layer's activations and their slopes over everything that bfloat16 holds."""

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


def every_number():
    """All finite bf16 numbers, in both signs."""
    z = torch.arange(0, 1 << 16, dtype=torch.int32).to(torch.int16).view(BF)
    return z[z.isfinite()].to(DEV)[:, None].contiguous()


def value(llm, z, act, dtype=torch.float32):
    return llm.linear(z, torch.ones(1, 1, device=DEV, dtype=BF), act=act, dtype=dtype).y


def slopes(llm, z, act):
    """As the product's epilogue and as the call of its own form it."""
    one = torch.ones_like(z)
    return llm.linear_dgrad(one, torch.ones(1, 1, device=DEV, dtype=BF), act=act, z=z, dtype=torch.float32), llm.activation_backward(one, z, act)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_far_from_zero(llm, act):
    """z itself far above zero and nothing far below, out to the largest numbers: where e^-|z| falls below 2^-126 it counts as zero, which is
    |z| 2^-126 of SiLU's value and slope there, |z| < 88 (and less of GELU's)."""
    z = every_number()
    z = z[z.abs() > 20][:, None]
    least = 90 * 2.0 ** -126
    for dtype in (torch.float32, BF):
        y, want = R.d(value(llm, z, act, dtype)), R.act(act, R.d(z))
        r = 0 if dtype == torch.float32 else 2.0 ** -8
        assert ((y - want).abs() <= (1e-5 + r) * want.abs() + least).all()
    s, b = slopes(llm, z, act)
    # below zero a slope is about z times the value's factor
    want, size = R.slope(act, R.d(z)), (R.d(z) < 0) * (1 + R.d(z).abs()) * torch.exp(R.d(z).clamp(max=0))
    for got, r in ((s, 0.0), (b, 2.0 ** -8)):
        assert ((R.d(got) - want).abs() <= 3e-5 * size + (r + 1e-5) * want.abs() + least).all()


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_infinities_and_what_is_no_number(llm, act):
    z = torch.tensor([float("inf"), -float("inf"), float("nan")], device=DEV).to(BF)[:, None]
    for dtype in (torch.float32, BF):
        up, down, none = value(llm, z, act, dtype)[:, 0].tolist()
        assert up == float("inf") and down == 0 and none != none
    for s in slopes(llm, z, act):
        up, down, none = s[:, 0].tolist()
        assert up == 1 and down == 0 and none != none


# Roundings of fp32, 2^-24 of the value, one after the other.  The fast exponential is right to four of them, the reciprocal to two.
# GELU: the exponential's square 8 + 1, what its argument leaves out 1; the polynomial and its argument 10.4 (evaluated in fp32 beside 64 bits), the reciprocal
# in it 1.3 more; two products 2.
GELU = 24 * R.U32
# SiLU: the exponential 4 + 1, 1 + it 1, the reciprocal 2, two products 2.
SILU = 10 * R.U32


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_precision_of_32_bit_results(llm, act):
    """Relative to the value, in the lower tail too; a slope relative to its terms, which have opposite signs below zero."""
    z = every_number()
    z = z[(z.abs() <= 13) & (z.abs() > 2.0 ** -40)][:, None]
    d = R.d(z)
    y, want = R.d(value(llm, z, act)), R.act(act, d)
    bad = (y - want).abs() / want.abs()
    assert float(bad.max()) <= (GELU if act == "gelu" else SILU), float(d[bad.argmax()])
    s, want = R.d(slopes(llm, z, act)[0]), R.slope(act, d)
    size = R.phi(d) + d.abs() * torch.exp(-0.5 * d * d) * 0.4 if act == "gelu" else torch.sigmoid(d) * (1 + d.abs() * torch.sigmoid(-d))
    bad = (s - want).abs() / size
    assert float(bad.max()) <= (GELU + 2 * R.U32 if act == "gelu" else 2 * SILU), float(d[bad.argmax()])
