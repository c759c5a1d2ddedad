"""How exactly a linear layer's sums are held when the result is bf16: the residual takes away what the rounding would hide."""

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def positive(*s, seed):
    return (0.5 + torch.rand(*s, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)).to(BF)


def limit(K, size):
    """16 products at a time, 64 times at most until a sum is taken over, each dropping less than 2^-23 of what is there; the sums taken over and the
    parts of a cut tile are added with half of that, one after the other; a few roundings behind."""
    return (64 + (K // 1024 + 2) / 2 + 4) * 2.0 ** -23 * size


# one sum, two, many; more tiles than pairs of SMs (whole ones and cut ones), few tiles (all cut), rows that are moved one element at a time
@pytest.mark.parametrize("T,K,N", [(2560, 16384, 2048), (2600, 20000, 2040), (700, 1024, 512), (700, 1032, 512), (300, 3000, 515), (64, 60000, 256)])
@pytest.mark.parametrize("way", ["forward", "dgrad"])
def test_sums_of_bf16_results_do_not_lose_digits_with_their_length(llm, way, T, K, N):
    x, w = positive(T, K, seed=1), positive(K, N, seed=2)
    z = x.double() @ w.double()                       # all terms are positive: the sum is its terms' size
    res = (-z).to(BF)
    if way == "forward":
        y = llm.linear(x, w, residual=res).y
    else:
        y = llm.linear_dgrad(x, w.t().contiguous(), residual=res)
    llm.check()
    want = z + res.double()
    err = (y.double() - want).abs()
    assert bool((err <= limit(K, z) + 2.0 ** -8 * (want.abs() + limit(K, z))).all()), float((err / limit(K, z)).max())
