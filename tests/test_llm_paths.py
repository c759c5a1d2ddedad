"""Forms of the losses' kernels that other sizes and alignments take: a CTA per row with 128 threads, and the preference loss with
logits and gradient that are not aligned alike."""

import pytest
import torch

from tests import llm_reference as R
from tests.test_llm_losses import check_policy, check_pref, policy_case, pref_case

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


# rows of 24 to 48 KB
@pytest.mark.parametrize("T,V,dtype", [(100, 9000, "f32"), (150, 6200, "f32"), (90, 12288, "f32"), (100, 16001, "bf16"), (400, 24570, "bf16")])
def test_rows_of_a_few_tens_of_kilobytes(llm, T, V, dtype):
    z, y, old, adv, w, ref = policy_case(T, V, dtype, T + V)
    w[::7] = 0.0
    y[5::13] = V
    want = R.policy(z, y, old, adv, w, ref, kl_coef=0.1)
    a = llm.policy_loss(z, y, old, adv, w, logp_ref=ref, kl_coef=0.1)
    check_policy(a, want, z, 0.1)
    only = llm.policy_loss(z, y, old, adv, w, logp_ref=ref, kl_coef=0.1, need_grad=False)
    assert torch.equal(only.loss, a.loss) and torch.equal(only.logp, a.logp)
    off = torch.tensor([0, T // 5, T // 2, T - 3, T], dtype=torch.int32, device=DEV)
    sums = R.preference(z, y, off, torch.zeros(4))["seq_logp"].float().to(DEV)
    sref = sums + torch.tensor([2.0, -1.0, 0.5, 0.0], device=DEV)
    p = llm.preference_loss(z, y, off, sref, beta=0.2, smoothing=0.1)
    check_pref(p, R.preference(z, y, off, sref, 0.2, 0.1), z, 0.2, 0.5)
    spare = z.clone()
    b = llm.preference_loss(spare, y, off, sref, beta=0.2, smoothing=0.1, dlogits=spare)
    assert torch.equal(b.dlogits, p.dlogits)
    b = llm.policy_loss(z, y, old, adv, w, logp_ref=ref, kl_coef=0.1, dlogits=z)
    for u, v in zip(a, b):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,V", [((5, 6, 0, 7), 40), ((9, 3), 1000), ((30, 41, 8, 2), 1025), ((3, 2), 20001), ((60, 60), 9001)])
def test_preference_gradient_at_another_alignment(llm, lens, V, dtype):
    z, y, off, ref = pref_case(lens, V, dtype, V, 1)
    T = z.shape[0]
    z[0] = float("-inf")
    for left, oleft, gap in ((0, 1, 9), (1, 0, 9), (3, 2, 10), (0, 0, 1), (2, 0, 3)):
        big = torch.full((T, V + 8), float("nan"), dtype=z.dtype, device=DEV)
        big[:, left:left + V] = z
        obig = torch.full((T, V + oleft + gap), 7.0, dtype=z.dtype, device=DEV)
        out = obig[:, oleft:oleft + V]
        r = llm.preference_loss(big[:, left:left + V], y, off, ref, beta=0.2, smoothing=0.05, dlogits=out)
        clean = torch.where(torch.isinf(z), torch.zeros_like(z), z)
        yy = y.clone()
        yy[0] = -1                                            # a row of -inf is not counted
        check_pref(r, R.preference(clean, yy, off, ref, 0.2, 0.05), clean, 0.2, 2.0 / len(lens))
        assert r.dlogits.data_ptr() == out.data_ptr()
        assert (obig[:, :oleft] == 7).all() and (obig[:, oleft + V:] == 7).all()
