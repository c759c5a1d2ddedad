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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", ROWS)
def test_maxima_on_either_side_of_1e30(llm, T, V, dtype):
    """Logits of 1e30 and more: of two different ones the smaller has probability 0, wherever in the row they stand."""
    z, y = logits(T, V, dtype, V), labels(T, V, 3)
    at, c = torch.arange(T, device=DEV), torch.tensor
    small, large = (c(v).to(DT[dtype]).to(DEV) for v in (0.99e30, 1.1e30))
    first = torch.randint(0, V - 1, (T,), generator=gen(5), device=DEV)
    second = first + 1 + (torch.rand(T, generator=gen(6), device=DEV) * (V - 1 - first)).long()
    z[at, first], z[at, second] = small, large                    # the larger one comes later
    half = T // 2
    z[half:] = small                                              # all of one value but one that is below it
    z[half:] *= -1
    z[at[half:], first[half:]] = -large
    y[:half] = second[:half].int()
    want = torch.zeros(T, dtype=R.D)                              # logp of the only largest one
    y[half:] = second[half:].int()
    want[half:] = -torch.log(torch.tensor(float(V - 1), dtype=R.D))
    one = torch.ones(T, device=DEV)
    for kw in (dict(), dict(dlogits=at_another_alignment(z))):
        r = llm.policy_loss(z, y, want.float().to(DEV), one, one, **kw)
        R.close(r.logp, want, 1e-5, "logp")
        R.close(r.loss[None], torch.tensor([-float(T)], dtype=R.D), T * 1e-5, "loss")
        p = torch.zeros(T, V, dtype=R.D)
        p[half:] = 1.0 / (V - 1)
        p[torch.arange(T)[half:], first[half:].cpu()] = 0
        p[torch.arange(half), second[:half].cpu()] = 1
        grad = p.clone()
        grad[torch.arange(T), y.cpu().long()] -= 1
        R.close(r.dlogits, grad, 1e-5 * torch.ones(T, V, dtype=R.D) * p + 1e-5 * (grad != 0), "dlogits")
    r = llm.preference_loss(z, y, torch.tensor([0, half, T], dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV))
    R.close(r.seq_logp, torch.stack([want[:half].sum(), want[half:].sum()]), 1e-5 * T, "seq_logp")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [2.0 ** 24, 1e8, 2.0 ** 30, 1e9, 1.5e9, 1e10, 1e15, 1e25])
@pytest.mark.parametrize("T,V", ROWS)
def test_rows_of_large_numbers(llm, T, V, size, dtype):
    """All logits around +-size, a few units in the last place apart (masks of -1e9 or -1e10 over a whole row, for one)."""
    unit = float(torch.finfo(DT[dtype]).eps) / 2 * 2.0 ** torch.tensor(size).log2().ceil().item()
    z = size + unit * torch.randint(-2, 3, (T, V), generator=gen(3), device=DEV).double()
    z[::2] *= -1
    z[1::4, : V // 2] /= 4
    z = z.to(DT[dtype])
    y = labels(T, V, 3)
    want, p, _ = R.rows_logp(z, y)
    w = torch.where(want > -60, 1.0 / T, 0.0).float().to(DEV)      # beyond that a ratio or a probability is nothing
    live = (w != 0).cpu()
    want = torch.where(live, want, torch.zeros((), dtype=R.D))
    one = torch.ones(T, device=DEV)
    grad = p * live[:, None]
    grad[torch.arange(T), y.cpu().long()] -= live.to(R.D)
    # an exponential's exponent has up to 64 units of the common factor in it: off by 2^-18, 2.7e-6 of it; the sum's logarithm likewise
    tol = 2e-5
    for kw in (dict(), dict(dlogits=at_another_alignment(z))):
        r = llm.policy_loss(z, y, want.float().to(DEV), one, w, **kw)
        R.close(r.logp, want, tol + 4 * R.U32 * want.abs(), "logp")
        R.close(r.loss[None], -live.to(R.D).mean()[None], 3 * tol, "loss")
        R.close(r.dlogits, grad / T, (3 * tol * (p + (grad < 0)) + 1e-18) / T, "dlogits")
    yy = torch.where(w != 0, y, torch.full_like(y, -1))
    r = llm.preference_loss(z, yy, torch.tensor([0, T // 2, T], dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV))
    R.close(r.seq_logp, torch.stack([want[: T // 2].sum(), want[T // 2:].sum()]), T * tol + 4 * R.U32 * want.abs().sum(), "seq_logp")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("smoothing", [0.0, 0.1, 1.0])
def test_preference_gradient_at_large_margins(llm, smoothing, dtype):
    """A well separated pair's gradient is small, not lost: relative to itself it is as exact as any other."""
    V, margins = 500, [0.0, 1.0, -1.0, 4.0, 8.0, -8.0, 12.0, -12.0, 16.0, -16.0, 17.0, 20.0, -20.0, 40.0, -40.0, 80.0, -80.0]
    n = len(margins)
    z, y = logits(4 * n, V, dtype, 1), labels(4 * n, V, 2)
    off = torch.arange(0, 4 * n + 1, 2, dtype=torch.int32, device=DEV)
    s = R.preference(z, y, off, torch.zeros(2 * n))["seq_logp"]
    ref = s.float()
    ref[0::2] -= torch.tensor(margins)
    r = llm.preference_loss(z, y, off, ref.to(DEV), beta=1.0, smoothing=smoothing, scale=1.0)
    want = R.preference(z, y, off, ref, 1.0, smoothing, 1.0)
    sm = float(torch.tensor(smoothing))
    h = want["h"]
    # without a difference of nearly equal numbers; h is off by the four rows' logp, 1.5e-5 together
    g = sm * torch.sigmoid(h) - (1 - sm) * torch.sigmoid(-h)
    assert torch.allclose(g, want["g"][::4], rtol=1e-6, atol=1e-15)
    eh = 1.5e-5
    eg = eh * (sm * torch.sigmoid(h) * torch.sigmoid(-h) + (1 - sm) * torch.sigmoid(-h) * torch.sigmoid(h)) + 4e-7 * (sm * torch.sigmoid(h) + (1 - sm) * torch.sigmoid(-h))
    row = g.repeat_interleave(4) * torch.tensor([1.0, 1.0, -1.0, -1.0], dtype=R.D).repeat(n)
    _, p, _ = R.rows_logp(z, y)
    grad = -row[:, None] * p
    grad[torch.arange(4 * n), y.cpu().long()] += row
    R.close(r.dlogits, grad, (eg.repeat_interleave(4) + 1e-5 * row.abs())[:, None], "dlogits")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", ROWS)
def test_a_reference_without_a_coefficient_changes_nothing(llm, T, V, dtype):
    """logp_ref given for its statistic alone: however far it is, a term with coefficient 0 adds nothing to loss and gradient."""
    z, y = logits(T, V, dtype, 9), labels(T, V, 10)
    old = R.rows_logp(z, y)[0].float().to(DEV)
    z[1, y[1].long()] = float("-inf")                             # the label has probability 0: its kl_t has no bound
    adv, w = torch.randn(T, generator=gen(4), device=DEV), torch.full((T,), 1.0 / T, device=DEV)
    ref = old.clone()
    ref[2], ref[3] = 200.0, float("inf")
    for place in (lambda: None, lambda: at_another_alignment(z)):
        a = llm.policy_loss(z, y, old, adv, w, dlogits=place())
        b = llm.policy_loss(z, y, old, adv, w, logp_ref=ref, kl_coef=0.0, dlogits=place())
        assert torch.isfinite(a.loss) and torch.isfinite(a.dlogits).all()
        assert torch.equal(a.loss, b.loss) and torch.equal(a.logp, b.logp) and torch.equal(a.clipped, b.clipped)
        assert torch.equal(a.dlogits, b.dlogits)
