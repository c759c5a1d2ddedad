"""A small recurrent language model made of the operators of ``llm``, from tokens to the gradient of every parameter: the
``--block recurrent`` of ``llm_example``.

A layer, on the packed tokens of ragged sequences (x is the residual stream):

    n  = layer_norm(x)                  u = linear(n)   g = linear(n)
    h  = gated_recurrence(u, g)         x = linear(h) + x
    m  = layer_norm(x)                  x = linear(gelu(linear(m))) + x

in front of it ``embed``, behind it a last ``layer_norm`` and the head.  The way back calls the same operators' gradients in reverse and writes
every one of them into its slice of a flat gradient.  ``generate`` takes one token of each sequence at a time
(``gated_recurrence_step``)."""

from __future__ import annotations

import math
from typing import List, NamedTuple

import torch


class Sizes(NamedTuple):
    width: int = 256
    vocab: int = 2048
    tokens: int = 768          # of a micro-batch
    hidden: int = 512
    layers: int = 2
    sequences: int = 8         # of a micro-batch
    prompt: int = 6            # tokens of a sequence that do not count


_LAYER = ("norm_1.w", "norm_1.b", "in.w", "in.b", "gate.w", "gate.b", "out.w", "out.b", "norm_2.w", "norm_2.b", "up.w", "up.b", "down.w", "down.b")


def layout(s: Sizes):
    """(name, shape) of the parameters, in the order of the flat vector."""
    D, H = s.width, s.hidden
    shape = {"norm_1.w": (D,), "norm_1.b": (D,), "in.w": (D, D), "in.b": (D,), "gate.w": (D, D), "gate.b": (D,), "out.w": (D, D), "out.b": (D,),
             "norm_2.w": (D,), "norm_2.b": (D,), "up.w": (D, H), "up.b": (H,), "down.w": (H, D), "down.b": (D,)}
    each = [(f"{i}.{k}", shape[k]) for i in range(s.layers) for k in _LAYER]
    return [("table", (s.vocab, D))] + each + [("norm.w", (D,)), ("norm.b", (D,)), ("head", (D, s.vocab))]


def views(flat: torch.Tensor, s: Sizes):
    out, at = {}, 0
    for name, shape in layout(s):
        n = math.prod(shape)
        out[name] = flat[at:at + n].view(shape)
        at += n
    return out


def init_params(s: Sizes, seed: int, device) -> torch.Tensor:
    g = torch.Generator(device=device).manual_seed(seed)
    flat = torch.zeros(sum(math.prod(shape) for _, shape in layout(s)), device=device)
    for name, p in views(flat, s).items():
        if name == "table":
            p.normal_(0.0, s.width ** -0.5, generator=g)
        elif p.dim() == 2:
            p.normal_(0.0, p.shape[0] ** -0.5, generator=g)
        elif name.endswith("norm.w") or ".norm_" in name and name.endswith(".w"):
            p.fill_(1.0)
        elif name.endswith("gate.b"):
            p.fill_(2.0)               # gates that mostly keep
    return flat


def _scale(s: Sizes) -> float:
    return s.width ** 0.5


class Layer(NamedTuple):
    """What the way back of one layer needs."""
    x: torch.Tensor
    n: torch.Tensor
    u: torch.Tensor
    g: torch.Tensor
    h: torch.Tensor
    x1: torch.Tensor
    m: torch.Tensor
    z: torch.Tensor
    a: torch.Tensor


def forward(p, ids, offsets, s: Sizes):
    """(logits, what the way back keeps)."""
    from . import llm

    kept: List[Layer] = []
    x = llm.embed(ids, p["table"], scale=_scale(s))
    for i in range(s.layers):
        w = lambda k: p[f"{i}.{k}.w"].bfloat16()  # noqa: E731
        b = lambda k: p[f"{i}.{k}.b"]  # noqa: E731
        n = llm.layer_norm(x, p[f"{i}.norm_1.w"], b("norm_1"))
        u, g = llm.linear(n, w("in"), b("in")).y, llm.linear(n, w("gate"), b("gate")).y
        h = llm.gated_recurrence(u, g, offsets).y
        x1 = llm.linear(h, w("out"), b("out"), residual=x).y
        m = llm.layer_norm(x1, p[f"{i}.norm_2.w"], b("norm_2"))
        a = llm.linear(m, w("up"), b("up"), act="gelu", keep=True)
        kept.append(Layer(x, n, u, g, h, x1, m, a.z, a.y))
        x = llm.linear(a.y, w("down"), b("down"), residual=x1).y
    n = llm.layer_norm(x, p["norm.w"], p["norm.b"])
    return llm.linear(n, p["head"].bfloat16()).y, (kept, x, n)


def backward(p, grad, kept, dlogits, ids, offsets, s: Sizes):
    """Writes the gradient of every parameter into its slice of `grad`."""
    from . import llm

    layers, x, n = kept
    d = views(grad, s)

    def norm_back(dn, at, name, skip):
        return llm.layer_norm_backward(dn, at, p[name + ".w"], dskip=skip, dw=d[name + ".w"], db=d[name + ".b"]).dx

    def wgrad(name, at, dy):
        llm.linear_wgrad(at, dy, bias=True, dw=d[name + ".w"], db=d[name + ".b"])

    llm.linear_wgrad(n, dlogits, dw=d["head"])
    dx = norm_back(llm.linear_dgrad(dlogits, p["head"].bfloat16()), x, "norm", None)
    for i in reversed(range(s.layers)):
        k = layers[i]
        w = lambda name: p[f"{i}.{name}.w"].bfloat16()  # noqa: E731
        wgrad(f"{i}.down", k.a, dx)
        dz = llm.linear_dgrad(dx, w("down"), act="gelu", z=k.z)
        wgrad(f"{i}.up", k.m, dz)
        dx = norm_back(llm.linear_dgrad(dz, w("up")), k.x1, f"{i}.norm_2", dx)
        wgrad(f"{i}.out", k.h, dx)
        r = llm.gated_recurrence_backward(llm.linear_dgrad(dx, w("out")), k.u, k.g, k.h, offsets)
        wgrad(f"{i}.in", k.n, r.dx)
        wgrad(f"{i}.gate", k.n, r.dg)
        dn = llm.linear_dgrad(r.dx, w("in"))
        dn = llm.linear_dgrad(r.dg, w("gate"), residual=dn, dx=dn)
        dx = norm_back(dn, k.x, f"{i}.norm_1", dx)
    llm.embed_backward(dx, ids, s.vocab, scale=_scale(s), out=d["table"])


def start(s: Sizes, sequences: int, device):
    """The states of sequences that have not begun: one [sequences, width] for each layer."""
    return [torch.zeros(sequences, s.width, device=device) for _ in range(s.layers)]


def step(p, ids, states, s: Sizes):
    """Logits behind one more token of each sequence; the states move on."""
    from . import llm

    x = llm.embed(ids, p["table"], scale=_scale(s))
    for i in range(s.layers):
        w = lambda k: p[f"{i}.{k}.w"].bfloat16()  # noqa: E731
        b = lambda k: p[f"{i}.{k}.b"]  # noqa: E731
        n = llm.layer_norm(x, p[f"{i}.norm_1.w"], b("norm_1"))
        u, g = llm.linear(n, w("in"), b("in")).y, llm.linear(n, w("gate"), b("gate")).y
        h = llm.gated_recurrence_step(u, g, states[i], out=states[i]).y
        x = llm.linear(h, w("out"), b("out"), residual=x).y
        m = llm.layer_norm(x, p[f"{i}.norm_2.w"], b("norm_2"))
        x = llm.linear(llm.linear(m, w("up"), b("up"), act="gelu").y, w("down"), b("down"), residual=x).y
    return llm.linear(llm.layer_norm(x, p["norm.w"], p["norm.b"]), p["head"].bfloat16()).y


def generate(p, prompts, length: int, s: Sizes, generator=None):
    """int32 [sequences, prompt + length]: the prompts continued by tokens drawn from the model."""
    states = start(s, prompts.shape[0], prompts.device)
    out = [prompts[:, i].contiguous() for i in range(prompts.shape[1])]
    for i in range(prompts.shape[1] + length - 1):
        logits = step(p, out[i], states, s)
        if i + 1 >= prompts.shape[1]:
            out.append(torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=generator)[:, 0].to(torch.int32))
    return torch.stack(out, 1)


class Batch(NamedTuple):
    ids: torch.Tensor          # [tokens] int32, the sequences one after the other
    offsets: torch.Tensor      # [sequences + 1] int32
    labels: torch.Tensor       # [tokens] int32: the next token where it counts, otherwise -100
    logp_ref: torch.Tensor     # policy: [tokens]; preference: [sequences]
    advantage: torch.Tensor    # policy: [tokens]


def make_batch(p_ref, s: Sizes, objective: str, seed: int) -> Batch:
    """Ragged sequences.  Policy: prompts continued by the reference model, tokens of the lower half of the vocabulary have a positive advantage.
    Preference: answers made of tokens of the lower half are the preferred ones."""
    from . import llm

    dev, V, Q = p_ref["table"].device, s.vocab, s.sequences
    g = torch.Generator(device=dev).manual_seed(seed)
    most = s.tokens // Q
    lens = [max(s.prompt + 2, most - (q * 7919) % (most // 2)) for q in range(Q)]
    if objective == "policy":
        whole = generate(p_ref, torch.randint(0, V, (Q, s.prompt), generator=g, device=dev, dtype=torch.int32), most - s.prompt, s, g)
    else:
        whole = torch.randint(0, V // 2, (Q, most), generator=g, device=dev, dtype=torch.int32)
        whole[1::2, s.prompt:] += V // 2
        whole[1::2, :s.prompt] = whole[0::2, :s.prompt]
    ids = torch.cat([whole[q, :n] for q, n in enumerate(lens)])
    offsets = torch.tensor([0] + lens, device=dev).cumsum(0).to(torch.int32)
    labels = torch.cat([torch.cat((torch.full((s.prompt - 1,), -100, dtype=torch.int32, device=dev), whole[q, s.prompt:n],
                                   torch.full((1,), -100, dtype=torch.int32, device=dev))) for q, n in enumerate(lens)])
    logits, _ = forward(p_ref, ids, offsets, s)
    if objective == "policy":
        one = torch.ones(ids.numel(), device=dev)
        ref = llm.policy_loss(logits, labels, one, one, one, need_grad=False).logp
        advantage = torch.where(labels < V // 2, 1.0, -1.0)
    else:
        ref = llm.preference_loss(logits, labels, offsets, torch.zeros(Q, device=dev), need_grad=False).seq_logp
        advantage = torch.zeros(ids.numel(), device=dev)
    return Batch(ids, offsets, labels, ref, advantage)


def micro_batch(params, grad, b: Batch, s: Sizes, objective: str) -> torch.Tensor:
    """Loss of one micro-batch (a device scalar); its gradient goes to `grad`."""
    from . import llm

    p = views(params, s)
    logits, kept = forward(p, b.ids, b.offsets, s)
    if objective == "policy":
        weight = torch.where(b.labels >= 0, 1.0 / b.labels.numel(), 0.0)
        r = llm.policy_loss(logits, b.labels, b.logp_ref, b.advantage, weight, logp_ref=b.logp_ref, kl_coef=0.02, dlogits=logits)
    else:
        r = llm.preference_loss(logits, b.labels, b.offsets, b.logp_ref, beta=0.1, dlogits=logits)
    backward(p, grad, kept, r.dlogits, b.ids, b.offsets, s)
    return r.loss
