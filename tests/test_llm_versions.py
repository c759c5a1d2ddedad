"""Outputs that are given to the language-model operators count as modified: autograd refuses to use what it had saved."""

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def f32(*s):
    return torch.ones(*s, device=DEV)


def b16(*s):
    return torch.ones(*s, device=DEV, dtype=torch.bfloat16)


def calls(llm):
    i32 = torch.zeros(4, dtype=torch.int32, device=DEV)
    off = torch.tensor([0, 1, 4], dtype=torch.int32, device=DEV)
    c = llm.ckpt8_quantize(b16(4, 40))
    back = dict(w_post=f32(8), gate=b16(4, 8))
    return [
        (lambda **o: llm.policy_loss(f32(4, 5), i32, f32(4), f32(4), f32(4), **o), dict(dlogits=lambda: f32(4, 5))),
        (lambda **o: llm.preference_loss(f32(4, 5), i32, off, f32(2), **o), dict(dlogits=lambda: f32(4, 5))),
        (lambda **o: llm.residual_norm(b16(4, 8), b16(4, 8), f32(8), **o), dict(y=lambda: b16(4, 8), n=lambda: b16(4, 8))),
        (lambda **o: llm.residual_norm_backward(b16(4, 8), None, b16(4, 8), b16(4, 8), f32(8), **back, **o),
         dict(dx=lambda: b16(4, 8), dh=lambda: b16(4, 8), dgate=lambda: b16(4, 8), dw_pre=lambda: f32(8), dw_post=lambda: f32(8))),
        (lambda **o: llm.ckpt8_dequantize(c, **o), dict(out=lambda: b16(4, 40))),
        (lambda **o: llm.ckpt8_wgrad(c, b16(4, 6), **o), dict(out=lambda: f32(40, 6))),
    ]


def test_given_outputs_count_as_modified(llm):
    for call, makers in calls(llm):
        outs = {k: m() for k, m in makers.items()}
        whole = {k: torch.stack((v, v)) for k, v in outs.items()}
        views = {k: v[1] for k, v in whole.items()}              # a view and its base have one counter
        before = {k: v._version for k, v in outs.items()}, {k: v._version for k, v in whole.items()}
        call(**outs)
        call(**views)
        for k in outs:
            assert outs[k]._version == before[0][k] + 1, k
            assert whole[k]._version == before[1][k] + 1, k
        with torch.inference_mode():                             # there is nothing to count
            call(**{k: m() for k, m in makers.items()})


def test_a_refused_call_has_modified_nothing(llm):
    out = f32(4, 5)
    with pytest.raises(Exception):
        llm.policy_loss(f32(4, 5), torch.zeros(4, dtype=torch.int32, device=DEV), f32(4), f32(4), f32(4), clip_low=-1.0, dlogits=out)
    assert out._version == 0


def test_inputs_do_not_count_as_modified(llm):
    z, x = f32(4, 5), b16(4, 8)
    versions = z._version, x._version
    llm.policy_loss(z, torch.zeros(4, dtype=torch.int32, device=DEV), f32(4), f32(4), f32(4))
    llm.residual_norm(x, x.clone(), f32(8))
    assert (z._version, x._version) == versions


def test_autograd_notices_logits_that_were_overwritten(llm):
    x = torch.randn(4, 5, device=DEV, requires_grad=True)
    z = torch.tanh(x)                                            # saved for its own backward pass
    r = llm.policy_loss(z, torch.zeros(4, dtype=torch.int32, device=DEV), f32(4), f32(4), f32(4), dlogits=z.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward(r.dlogits)
    z = torch.tanh(x)
    r = llm.policy_loss(z, torch.zeros(4, dtype=torch.int32, device=DEV), f32(4), f32(4), f32(4))
    z.backward(r.dlogits)
    assert torch.isfinite(x.grad).all()
