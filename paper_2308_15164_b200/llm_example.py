"""A small model trained by W workers with the delayed synchronous step: how the operators of ``llm`` are used together, and how
their gradients reach the accumulators.

    python -m paper_2308_15164_b200.llm_example [--block gated|recurrent] [--objective policy|preference] [--iterations N]

--block gated: a gated residual block with a vocabulary head, on given hidden states.  --block recurrent: a recurrent language model from its
tokens on (``llm_recurrent``).  One micro-batch of one worker, at the published parameters x_t, with the gated block:

    h = x W_in                                       (a plain product)
    y, n = residual_norm(x, h, w_pre, w_post, gate)  norm behind the block, learned gate, residual, norm in front of the head
    logits = n W_head                                (a plain product)
    loss, dlogits = policy_loss | preference_loss
    dW_head = n^T dlogits   from n kept in 8 bits    dn = dlogits W_head^T
    dh, dw_pre, dw_post, dgate = residual_norm_backward(dn)
    dW_in = x^T dh          from x kept in 8 bits

All parameters are slices of the flat vector; every gradient is written straight into its slice of a flat gradient, which
``AbsSgd.accumulate`` adds to the worker's row.  Everything runs on the context's ``stream_acc``."""

from __future__ import annotations

import argparse
import sys
from typing import List, NamedTuple

import torch


class Sizes(NamedTuple):
    width: int = 512
    vocab: int = 4096
    tokens: int = 768          # of a micro-batch
    scale: float = 0.5         # of the residual branch


def layout(s: Sizes):
    """(name, shape) of the parameters, in the order of the flat vector."""
    D, V = s.width, s.vocab
    return [("w_in", (D, D)), ("w_post", (D,)), ("gate", (D,)), ("w_pre", (D,)), ("w_head", (D, V))]


def views(flat: torch.Tensor, s: Sizes):
    out, at = {}, 0
    for name, shape in layout(s):
        n = 1
        for k in shape:
            n *= k
        out[name] = flat[at:at + n].view(shape)
        at += n
    return out


def init_params(s: Sizes, seed: int, device) -> torch.Tensor:
    g = torch.Generator(device=device).manual_seed(seed)
    flat = torch.empty(sum(torch.Size(shape).numel() for _, shape in layout(s)), device=device)
    p = views(flat, s)
    p["w_in"].normal_(0.0, s.width ** -0.5, generator=g)
    p["w_post"].fill_(1.0)
    p["gate"].fill_(0.5)
    p["w_pre"].fill_(1.0)
    p["w_head"].normal_(0.0, s.width ** -0.5, generator=g)
    return flat


def forward(p, x, s: Sizes):
    """(logits, what the backward pass keeps: y and h, and the inputs of the two products in 8 bits)."""
    from . import llm

    h = x @ p["w_in"].bfloat16()
    y, n = llm.residual_norm(x, h, p["w_pre"], w_post=p["w_post"], gate=p["gate"], scale=s.scale)
    kept = (llm.ckpt8_quantize(x), y, h, llm.ckpt8_quantize(n))
    return n @ p["w_head"].bfloat16(), kept


def backward(p, grad, kept, dlogits, s: Sizes):
    """Writes the gradient of every parameter into its slice of `grad`."""
    from . import llm

    x8, y, h, n8 = kept
    g = views(grad, s)
    llm.ckpt8_wgrad(n8, dlogits, out=g["w_head"])
    dn = dlogits @ p["w_head"].bfloat16().t()
    r = llm.residual_norm_backward(dn, None, y, h, p["w_pre"], w_post=p["w_post"], gate=p["gate"], scale=s.scale, dw_pre=g["w_pre"],
                                   dw_post=g["w_post"], dgate=g["gate"])
    llm.ckpt8_wgrad(x8, r.dh, out=g["w_in"])


class Batch(NamedTuple):
    x: torch.Tensor            # [tokens, width] bf16: the hidden states that the block sees
    labels: torch.Tensor       # [tokens] int32: the tokens that were taken
    logp_ref: torch.Tensor     # policy: [tokens]; preference: [answers]
    advantage: torch.Tensor    # policy: [tokens]
    offsets: torch.Tensor      # preference: first rows of the answers, preferred and other in turn


def make_batch(p_ref, s: Sizes, objective: str, seed: int) -> Batch:
    """Tokens from the reference model on random states.  Tokens of the lower half of the vocabulary are the good ones: their
    advantage is positive, answers made of them are the preferred ones."""
    from . import llm

    dev = p_ref["w_in"].device
    g = torch.Generator(device=dev).manual_seed(seed)
    T, V = s.tokens, s.vocab
    x = torch.randn(T, s.width, generator=g, device=dev).bfloat16()
    logits, _ = forward(p_ref, x, s)
    offsets = torch.arange(0, T + 1, max(1, T // 8), device=dev, dtype=torch.int32)
    offsets = torch.cat((offsets[: (offsets.numel() - 1) // 2 * 2], offsets[-1:]))
    if objective == "policy":
        labels = torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=g)[:, 0]
        advantage = torch.where(labels < V // 2, 1.0, -1.0)
    else:
        answer = torch.bucketize(torch.arange(T, device=dev, dtype=torch.int32), offsets[1:], right=True)
        labels = torch.randint(0, V // 2, (T,), generator=g, device=dev) + (V // 2) * (answer % 2)
        advantage = torch.zeros(T, device=dev)
    labels = labels.to(torch.int32)
    one = torch.ones(T, device=dev)
    if objective == "policy":
        ref = llm.policy_loss(logits, labels, one, one, one, need_grad=False).logp
    else:
        ref = llm.preference_loss(logits, labels, offsets, torch.zeros(offsets.numel() - 1, device=dev), need_grad=False).seq_logp
    return Batch(x, labels, ref, advantage, offsets)


def micro_batch(params, grad, b: Batch, s: Sizes, objective: str) -> torch.Tensor:
    """Loss of one micro-batch (a device scalar); its gradient goes to `grad`."""
    from . import llm

    p = views(params, s)
    logits, kept = forward(p, b.x, s)
    if objective == "policy":
        weight = torch.full_like(b.advantage, 1.0 / s.tokens)
        # sampled by the reference model, which is a few updates old
        r = llm.policy_loss(logits, b.labels, b.logp_ref, b.advantage, weight, logp_ref=b.logp_ref, kl_coef=0.02, dlogits=logits)
    else:
        r = llm.preference_loss(logits, b.labels, b.offsets, b.logp_ref, beta=0.1, dlogits=logits)
    backward(p, grad, kept, r.dlogits, s)
    return r.loss


def train(objective: str = "policy", iterations: int = 8, W: int = 4, micro_batches=(1, 1, 2, 3), lr: float = 0.2, sizes=None,
          seed: int = 0, block: str = "gated") -> List[float]:
    """Mean loss of each iteration.  micro_batches[i]: what worker i manages in an iteration; sizes: the block's, its own defaults if not given."""
    from . import binding, llm_recurrent

    model = {"gated": sys.modules[__name__], "recurrent": llm_recurrent}[block]
    sizes = model.Sizes() if sizes is None else sizes
    device = torch.device("cuda", torch.cuda.current_device())
    flat = model.init_params(sizes, seed, device)
    eng = binding.AbsSgd(flat, W, lr, momentum=0.9, pipelined=True)
    losses = []
    with torch.cuda.stream(eng.stream_acc):
        reference = model.views(flat.clone(), sizes)
        batches = [[model.make_batch(reference, sizes, objective, 1000 * i + k) for k in range(micro_batches[i])] for i in range(W)]
        grad = torch.empty_like(flat)
        for _ in range(iterations):
            x_t, step = eng.params(), []
            for i in range(W):
                for b in batches[i]:
                    step.append(model.micro_batch(x_t, grad, b, sizes, objective))
                    eng.accumulate(i, grad)
            losses.append(torch.stack(step).mean())
            eng.sync_step()
        losses = [float(v) for v in torch.stack(losses).cpu()]
    eng.check()
    eng.destroy()
    return losses


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--block", choices=("gated", "recurrent"), default="gated")
    ap.add_argument("--objective", choices=("policy", "preference"), default="policy")
    ap.add_argument("--iterations", type=int, default=8)
    a = ap.parse_args()
    for t, v in enumerate(train(a.objective, a.iterations, block=a.block)):
        print(f"iteration {t}: loss {v:.5f}")


if __name__ == "__main__":
    main()
