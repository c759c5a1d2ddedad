"""Precision of the language-model operators where a formula's obvious form loses it: against the definitions in 64 bits, with
bounds relative to the result itself."""

import pytest
import torch

from tests import llm_reference as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda"


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def logits(T, V, dtype, seed, shift=0.0):
    return (2 * torch.randn(T, V, generator=gen(seed), device=DEV) + shift).to(DT[dtype])


def labels(T, V, seed):
    return torch.randint(0, V, (T,), generator=gen(seed), device=DEV, dtype=torch.int32)


def at_another_alignment(z):
    """A place for the gradient whose rows start elsewhere between 16-byte boundaries than those of z."""
    return torch.empty(z.shape[0], z.shape[1] + 9, dtype=z.dtype, device=DEV)[:, 1:1 + z.shape[1]]


# (rows, vocabulary): a warp per row, a cluster per row, a CTA per row with 64, 128 and 256 threads
ROWS = [(200, 1000), (40, 8192), (100, 5000), (100, 12288), (90, 40000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0.0, 30.0, 200.0, -200.0, 5000.0])
@pytest.mark.parametrize("T,V", ROWS)
def test_log_probabilities_do_not_depend_on_a_common_offset(llm, T, V, shift, dtype):
    """A row's logits carry a common offset; logp is of the values as they are stored.  Bounds, without the offset: differences
    of logits are exact or rounded once; an exponential is off by 1e-6 (2^-22 and the rounding of its argument, each weighted
    by its share of the sum), a sum by at most 40 roundings one after the other, the logarithm's result by two of logp's size.
    The errors of a row's thousands of terms are not of one sign: over the rows, 1e-6 rms and a rounding of logp's size."""
    z, y = logits(T, V, dtype, V, shift), labels(T, V, V + 1)
    want, p, _ = R.rows_logp(z, y)
    one, adv = torch.ones(T, device=DEV), torch.full((T,), 1.0, device=DEV)
    old = want.float().to(DEV) - 0.1                              # ratio 1.1: within the clip
    off = torch.tensor([0, T // 2, T], dtype=torch.int32, device=DEV)

    def check(got):
        err = (R.d(got) - want).abs()
        assert (err <= 1e-6 + 40 * R.U32 + 4 * R.U32 * want.abs()).all(), float(err.max())
        assert float(err.square().mean().sqrt()) <= 1e-6 + R.U32 * float(want.abs().max()), float(err.square().mean().sqrt())

    for kw in (dict(), dict(dlogits=at_another_alignment(z)), dict(need_grad=False)):
        r = llm.policy_loss(z, y, old, adv, one, **kw)
        check(r.logp)
    r = llm.preference_loss(z, y, off, torch.zeros(2, device=DEV))
    s = torch.stack([want[: T // 2].sum(), want[T // 2:].sum()])
    # a sum in 64 bits of T / 2 such numbers, rounded once
    assert ((R.d(r.seq_logp) - s).abs() <= T * (1e-6 + R.U32 * float(want.abs().max())) + R.U32 * s.abs()).all()
