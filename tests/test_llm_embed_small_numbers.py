"""The embedding's gradient added to what is there, down to the smallest numbers."""

import pytest
import torch

from tests import llm_layers_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
LEAST = 2.0 ** -126


@pytest.mark.parametrize("T", [6, 300, 5000])
def test_numbers_below_the_normal_range_count_as_zero(T):
    """Each of the three numbers of an addition is off by less than 2^-126 where it is below that; rows that move four numbers at a time and one at a time
    agree bit by bit, rows of no token keep theirs."""
    from paper_2308_15164_b200 import llm

    V, W = 9, 8
    g = torch.Generator(device=DEV).manual_seed(T)
    size = lambda *s: torch.randn(*s, generator=g, device=DEV) * 2.0 ** torch.randint(-140, -120, s, generator=g, device=DEV).float()  # noqa: E731
    ids = torch.full((T,), -1, dtype=torch.int32, device=DEV)
    ids[:6] = torch.tensor([0, 1, 2, 3, 4, 5], dtype=torch.int32, device=DEV)         # one token a row: no sums of their own
    dy, base = size(T, W), size(V, W)
    out = base.clone()
    llm.embed_backward(dy, ids, V, out=out, accumulate=True)
    want = R.d(base)
    want[:6] += R.d(dy[:6])
    assert ((R.d(out) - want).abs() <= 3 * LEAST + R.U32 * want.abs()).all() and torch.equal(out[6:], base[6:])
    buf = torch.zeros(V * W + 1, device=DEV)
    other = buf[1:].view(V, W)                                                        # not aligned to 16 bytes
    other.copy_(base)
    llm.embed_backward(dy, ids, V, out=other, accumulate=True)
    assert torch.equal(other, out)
    # without adding, they are kept
    llm.embed_backward(dy, ids, V, out=out)
    assert torch.equal(out[:6], dy[:6]) and (out[6:] == 0).all()
