"""The operators from tokens to logits and back together, as a recurrent language model's training step and its generation use them: the flat
gradient of a micro-batch against autograd in 64 bits, steps against the packed pass, a captured step, and the training command."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    from paper_2308_15164_b200 import llm_recurrent

    return llm_recurrent


def reference_logits(p, ids, offsets, s):
    F = torch.nn.functional
    x = p["table"][ids.long()] * s.width ** 0.5
    cuts = offsets.tolist()
    for i in range(s.layers):
        q = lambda k: p[f"{i}.{k}"]  # noqa: E731,B023
        n = F.layer_norm(x, (s.width,), q("norm_1.w"), q("norm_1.b"), 1e-5)
        u, a = n @ q("in.w") + q("in.b"), torch.sigmoid(n @ q("gate.w") + q("gate.b"))
        rows = []
        for b, e in zip(cuts[:-1], cuts[1:]):
            h = torch.zeros(s.width, dtype=x.dtype, device=x.device)
            for t in range(b, e):
                h = a[t] * h + (1 - a[t]) * u[t]
                rows.append(h)
        x = torch.stack(rows) @ q("out.w") + q("out.b") + x
        m = F.layer_norm(x, (s.width,), q("norm_2.w"), q("norm_2.b"), 1e-5)
        x = F.gelu(m @ q("up.w") + q("up.b")) @ q("down.w") + q("down.b") + x
    return F.layer_norm(x, (s.width,), p["norm.w"], p["norm.b"], 1e-5) @ p["head"]


def reference_gradient(M, flat, b, s, objective):
    full = flat.double().requires_grad_()
    logits = reference_logits(M.views(full, s), b.ids, b.offsets, s)
    on = b.labels >= 0
    logp = torch.log_softmax(logits, 1).gather(1, b.labels.clamp(min=0).long()[:, None])[:, 0] * on
    if objective == "policy":
        r = (logp - b.logp_ref.double()).exp()
        A, x = b.advantage.double(), b.logp_ref.double() - logp
        loss = ((-torch.minimum(r * A, r.clamp(0.8, 1.2) * A) + 0.02 * (x.exp() - x - 1)) * on).sum() / on.numel()
    else:
        at = b.offsets.tolist()
        sums = torch.stack([logp[i:j].sum() for i, j in zip(at[:-1], at[1:])]) - b.logp_ref.double()
        loss = -torch.nn.functional.logsigmoid(0.1 * (sums[0::2] - sums[1::2])).mean()
    loss.backward()
    return float(loss.detach()), full.grad


@pytest.mark.parametrize("objective", ["policy", "preference"])
@pytest.mark.parametrize("width,vocab,tokens,hidden,layers", [(64, 300, 160, 96, 1), (72, 333, 200, 130, 2)])
def test_gradient_of_a_micro_batch(M, objective, width, vocab, tokens, hidden, layers):
    s = M.Sizes(width, vocab, tokens, hidden, layers, sequences=4, prompt=3)
    flat = M.init_params(s, 1, torch.device("cuda"))
    b = M.make_batch(M.views(flat, s), s, objective, 5)
    assert b.ids.numel() == int(b.offsets[-1]) == b.labels.numel()
    noise = torch.randn(flat.shape, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    moved = flat + 0.02 * noise * flat.abs()
    grad = torch.full_like(flat, float("nan"))
    loss = M.micro_batch(moved, grad, b, s, objective)
    want_loss, want = reference_gradient(M, moved, b, s, objective)
    # bf16 weights and activations: some ten roundings of 2^-9 rms a layer, and for the policy an advantage of either sign, so that a gradient is a
    # difference of sums several times its size
    assert abs(float(loss) - want_loss) <= 0.02 * max(1.0, abs(want_loss))
    for name, g in M.views(grad, s).items():
        w = M.views(want, s)[name]
        assert torch.isfinite(g).all(), name
        assert float((g.double() - w).norm()) <= 0.08 * float(w.norm()) + 1e-7 * math.sqrt(w.numel()), name


def test_steps_give_the_logits_of_the_packed_pass(M):
    s = M.Sizes(64, 200, 60, 96, 2, sequences=3, prompt=2)
    flat = M.init_params(s, 3, torch.device("cuda"))
    p = M.views(flat, s)
    ids = torch.randint(0, s.vocab, (3, 20), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.int32)
    offsets = torch.tensor([0, 20, 40, 60], dtype=torch.int32, device="cuda")
    packed = M.forward(p, ids.reshape(-1), offsets, s)[0].view(3, 20, -1)
    states = M.start(s, 3, ids.device)
    for t in range(20):
        logits = M.step(p, ids[:, t].contiguous(), states, s)
        # the same operators on other numbers of rows: bf16 roundings of a handful of layers may fall differently
        assert float((logits.float() - packed[:, t].float()).norm() / packed[:, t].float().norm()) <= 0.01
    out = M.generate(p, ids[:, :4].contiguous(), 5, s, torch.Generator(device="cuda").manual_seed(2))
    assert out.shape == (3, 9) and torch.equal(out[:, :4], ids[:, :4]) and int(out.min()) >= 0 and int(out.max()) < s.vocab


def test_a_micro_batch_captured_and_replayed(M):
    """Forward and backward pass as a CUDA graph: replays give the bits of the eager call, also with other parameters."""
    s = M.Sizes(64, 300, 160, 96, 2, sequences=4, prompt=3)
    params = M.init_params(s, 1, torch.device("cuda"))
    b = M.make_batch(M.views(params, s), s, "preference", 7)
    grad, want = torch.empty_like(params), torch.empty_like(params)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        M.micro_batch(params, grad, b, s, "preference")
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = M.micro_batch(params, grad, b, s, "preference")
    for k in range(3):
        params.mul_(1.0 + 0.01 * k)
        eager = M.micro_batch(params, want, b, s, "preference")
        grad.fill_(float("nan"))
        graph.replay()
        assert torch.equal(grad, want) and torch.equal(loss, eager)


@pytest.mark.parametrize("objective", ["policy", "preference"])
def test_training_runs(M, objective):
    from paper_2308_15164_b200 import llm, llm_example as E

    losses = E.train(objective, iterations=4, sizes=M.Sizes(64, 256, 128, 96, 1, sequences=4, prompt=3), lr=0.1, block="recurrent")
    # the first two iterations see x_0 and x_1 = x_0 (the step is delayed)
    assert len(losses) == 4 and losses[0] == losses[1] and all(math.isfinite(v) for v in losses)
    llm.check()
