"""The operators together, as a training step uses them: the flat gradient of a micro-batch against autograd in 64 bits, and
a few iterations of the delayed synchronous step with it."""

import pytest
import torch

pytestmark = pytest.mark.gpu


def reference_gradient(flat, b, s, objective):
    """The same micro-batch by autograd in 64 bits, from the values that the operators were given."""
    from paper_2308_15164_b200 import llm_example as E

    full = flat.double().requires_grad_()
    p = E.views(full, s)
    w_in, w_head = p["w_in"], p["w_head"]
    x = b.x.double()
    rms = lambda v: (v.square().mean(1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
    h = x @ w_in
    y = s.scale * x + p["gate"] * (h / rms(h) * p["w_post"])
    logits = (y / rms(y) * p["w_pre"]) @ w_head
    logp = torch.log_softmax(logits, 1).gather(1, b.labels.long()[:, None])[:, 0]
    if objective == "policy":
        r = (logp - b.logp_ref.double()).exp()
        A, x_ = b.advantage.double(), b.logp_ref.double() - logp
        loss = (-torch.minimum(r * A, r.clamp(0.8, 1.2) * A) + 0.02 * (x_.exp() - x_ - 1)).mean()
    else:
        at = b.offsets.tolist()
        sums = torch.stack([logp[a:c].sum() for a, c in zip(at[:-1], at[1:])]) - b.logp_ref.double()
        loss = -torch.nn.functional.logsigmoid(0.1 * (sums[0::2] - sums[1::2])).mean()
    loss.backward()
    return float(loss.detach()), full.grad


@pytest.mark.parametrize("objective", ["policy", "preference"])
@pytest.mark.parametrize("width,vocab,tokens", [(256, 1000, 160), (200, 777, 99), (512, 4096, 768)])
def test_gradient_of_a_micro_batch(objective, width, vocab, tokens):
    from paper_2308_15164_b200 import llm_example as E

    s = E.Sizes(width, vocab, tokens)
    flat = E.init_params(s, 1, torch.device("cuda"))
    b = E.make_batch(E.views(flat, s), s, objective, 5)
    moved = flat + 0.02 * torch.randn(flat.shape, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda") * flat.abs()
    grad = torch.full_like(flat, float("nan"))
    loss = E.micro_batch(moved, grad, b, s, objective)
    want_loss, want = reference_gradient(moved, b, s, objective)
    # bf16 products and activations: each of the handful of roundings on the way (2^-9 rms of a value) and 8 bits for the inputs of the weight
    # gradients (0.7 % rms) leave a few per cent of a gradient's norm at most
    assert abs(float(loss) - want_loss) <= 0.02 * max(1.0, abs(want_loss))
    for name, g in E.views(grad, s).items():
        w = E.views(want, s)[name]
        assert torch.isfinite(g).all(), name
        assert float((g.double() - w).norm() / w.norm()) <= 0.05, name


@pytest.mark.parametrize("objective", ["policy", "preference"])
def test_training_lowers_the_loss(objective):
    from paper_2308_15164_b200 import llm, llm_example as E

    losses = E.train(objective, iterations=6, sizes=E.Sizes(256, 1024, 256), lr=0.5)
    # the first two iterations see x_0 and x_1 = x_0 (the step is delayed)
    assert losses[0] == losses[1] and losses[-1] < losses[0]
    llm.check()
