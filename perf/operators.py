"""Cases for measuring the language-model training operators (paper_2308_15164_b200.llm).

One case is one call, or one pair of calls, of a micro-batch's training pass:

* ``policy``             clipped policy loss with a KL term: loss, per-token log-probabilities, gradient of the logits
* ``preference``         paired preference loss: loss, per-pair loss, sequence log-probabilities, gradient of the logits
* ``residual_forward``   norm behind a block, gate, scaled residual, norm in front of the next block
* ``residual_backward``  its gradients (activations, gate, norm weights)
* ``ckpt8``              an activation into 8 bits and back
* ``wgrad``              the gradient of a linear layer's weight from an activation held in 8 bits

With ``own`` false ``run`` computes the plain form: elementary torch operations in 32 bits, rounded once at the end.
"""

import torch

_llm = None  # the package, imported where the framework's own calls are made

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-6


def _calls():
    global _llm
    if _llm is None:
        from paper_2308_15164_b200 import llm

        _llm = llm
    return _llm


def listed():
    return [
        # a handful of sampled tokens scored by a small-vocabulary model: the time of the call itself
        {"name": "policy_few_tokens", "op": "policy", "tokens": 7, "vocab": 8192, "dtype": "f32", "kl": True, "banned": False},
        # an ordinary policy micro-batch: four packed rollouts of about a thousand tokens, KL to a reference model
        {"name": "policy_bf16", "op": "policy", "tokens": 4096, "vocab": 32768, "dtype": "bf16", "kl": True, "banned": False},
        # fp32 logits over an odd vocabulary (rows start at every alignment), tokens the sampler had excluded at -inf
        {"name": "policy_f32_odd_vocab", "op": "policy", "tokens": 1531, "vocab": 50257, "dtype": "f32", "kl": False, "banned": True},
        # one short pair, as at the end of an epoch
        {"name": "preference_one_pair", "op": "preference", "pairs": 1, "length": 33, "vocab": 32000, "dtype": "bf16", "smoothing": 0.0},
        # an ordinary preference micro-batch: eight pairs of ragged answers, label smoothing on
        {"name": "preference_bf16", "op": "preference", "pairs": 8, "length": 512, "vocab": 32000, "dtype": "bf16", "smoothing": 0.1},
        # a residual join of very few tokens
        {"name": "residual_forward_few", "op": "residual_forward", "tokens": 5, "width": 1024, "dtype": "bf16", "gate": "channel", "post": True},
        # a long micro-batch of a wide model, a learned gate for each channel
        {"name": "residual_forward_bf16", "op": "residual_forward", "tokens": 16384, "width": 4096, "dtype": "bf16", "gate": "channel", "post": True},
        # the way back through it, with a gate computed from the token
        {"name": "residual_backward_bf16", "op": "residual_backward", "tokens": 8192, "width": 4096, "dtype": "bf16", "gate": "element", "post": True},
        # fp32 activations, odd sizes, a plain pre-norm block with a learned gate
        {"name": "residual_backward_f32_odd", "op": "residual_backward", "tokens": 1003, "width": 1537, "dtype": "f32", "gate": "channel", "post": False},
        # the activations of a long micro-batch packed and unpacked
        {"name": "ckpt8_bf16", "op": "ckpt8", "tokens": 16384, "width": 4096, "dtype": "bf16"},
        # weight gradient of a square layer over a long micro-batch
        {"name": "wgrad_square", "op": "wgrad", "tokens": 8192, "width": 4096, "out": 4096},
        # odd sizes on every side: a ragged micro-batch and a classifier head
        {"name": "wgrad_odd", "op": "wgrad", "tokens": 515, "width": 1000, "out": 1111},
    ]


def _log_int(rng, lo, hi):
    import math

    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["policy", "policy", "preference", "residual_forward", "residual_backward", "ckpt8", "wgrad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "policy":
        vocab = _log_int(rng, 200, 152064)
        return {"op": op, "tokens": _log_int(rng, 1, min(32768, (1 << 27) // vocab)), "vocab": vocab, "dtype": dtype,
                "kl": rng.random() < 0.5, "banned": rng.random() < 0.3}
    if op == "preference":
        vocab = _log_int(rng, 200, 152064)
        pairs = _log_int(rng, 1, 16)
        return {"op": op, "pairs": pairs, "length": _log_int(rng, 2, max(2, min(2048, (1 << 27) // (2 * pairs * vocab)))), "vocab": vocab,
                "dtype": dtype, "smoothing": rng.choice([0.0, 0.1])}
    if op in ("residual_forward", "residual_backward"):
        width = _log_int(rng, 64, 8192)
        return {"op": op, "tokens": _log_int(rng, 1, min(65536, (1 << 26) // width)), "width": width, "dtype": dtype,
                "gate": rng.choice(["none", "channel", "element"]), "post": rng.random() < 0.6}
    if op == "ckpt8":
        width = _log_int(rng, 64, 16384)
        return {"op": op, "tokens": _log_int(rng, 1, min(65536, (1 << 26) // width)), "width": width, "dtype": dtype}
    width, out = _log_int(rng, 64, 4096), _log_int(rng, 16, 4096)
    return {"op": op, "tokens": _log_int(rng, 1, 8192), "width": width, "out": out}


# ---------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """Tokens of each of the 2 * pairs answers: ragged, by a fixed pattern."""
    n = case["length"]
    return [max(1, n - (q * 7919) % (n // 2 + 1)) for q in range(2 * case["pairs"])]


def _kept(case):
    """Tokens of a policy micro-batch that count: every eighth is prompt or padding."""
    return case["tokens"] - case["tokens"] // 8


def _logits(g, tokens, vocab, dtype, labels):
    """Logits of a model that gives its own tokens most of the weight."""
    z = torch.randn(tokens, vocab, generator=g, device=DEV) * 2.0
    z[torch.arange(tokens, device=DEV), labels.long()] += 9.0
    return z.to(DTYPES[dtype])


def _pick(z, labels):
    z = z.float()
    return z.gather(1, labels.long()[:, None])[:, 0] - torch.logsumexp(z, 1)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2654435761 % (1 << 31) + 17)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    op, s = case["op"], {"case": dict(case)}
    if op == "policy":
        T, V = case["tokens"], case["vocab"]
        labels = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
        z = _logits(g, T, V, case["dtype"], labels)
        if case["banned"]:  # tokens that top-k / grammar sampling had taken out; never the sampled one
            ban = torch.rand(T, V, generator=g, device=DEV) < 0.3
            ban[torch.arange(T, device=DEV), labels.long()] = False
            z.masked_fill_(ban, float("-inf"))
            del ban
        lp = _pick(z, labels)
        ratio = 0.15 * normal(T)
        # the gradient jumps where the ratio meets a bound of the clip, and either side is right there: none sits within 1e-3
        for b in (0.8, 1.2):
            at = float(torch.tensor(b).log())
            ratio = torch.where((ratio - at).abs() < 1e-3, ratio + 4e-3, ratio)
        s |= {"logits": z, "labels": labels, "logp_old": lp - ratio, "advantage": normal(T) + 0.25,
              "logp_ref": lp + 0.2 * normal(T) if case["kl"] else None}
        keep = (torch.arange(T, device=DEV) % 8) != 7
        s["weight"] = keep.float() / max(1, _kept(case))
    elif op == "preference":
        lens, V = _lengths(case), case["vocab"]
        T = sum(lens)
        labels = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
        z = _logits(g, T, V, case["dtype"], labels)
        offsets = torch.tensor([0] + lens, device=DEV).cumsum(0).to(torch.int32)
        seq = torch.repeat_interleave(torch.arange(len(lens), device=DEV), torch.tensor(lens, device=DEV))
        lead = torch.arange(T, device=DEV) - offsets[:-1].long()[seq]
        counted = lead >= torch.tensor([n // 4 for n in lens], device=DEV)[seq]  # the prompt's tokens do not count
        lp = torch.where(counted, _pick(z, labels), torch.zeros((), device=DEV))
        total = torch.zeros(len(lens), device=DEV, dtype=torch.float64).index_add_(0, seq, lp.double()).float()
        labels = torch.where(counted, labels, torch.full_like(labels, -100))
        s |= {"logits": z, "labels": labels, "offsets": offsets, "logp_ref": total + 4.0 * normal(len(lens))}
    elif op == "residual_forward":
        T, D, dt = case["tokens"], case["width"], DTYPES[case["dtype"]]
        x = normal(T, D) * 3.0
        x[:, :: max(1, D // 8)] *= 12.0  # a residual stream has a few channels far above the others
        s |= {"x": x.to(dt), "h": normal(T, D).to(dt)}
    elif op == "residual_backward":
        T, D, dt = case["tokens"], case["width"], DTYPES[case["dtype"]]
        y = normal(T, D) * 3.0
        y[:, :: max(1, D // 8)] *= 12.0
        s |= {"y": y.to(dt), "h": normal(T, D).to(dt), "dn": (0.1 * normal(T, D)).to(dt), "dy": (0.02 * normal(T, D)).to(dt)}
    elif op == "ckpt8":
        T, D, dt = case["tokens"], case["width"], DTYPES[case["dtype"]]
        x = normal(T, D)
        x[:, :: max(1, D // 8)] *= 20.0
        s["x"] = x.to(dt)
    else:
        T, D, N = case["tokens"], case["width"], case["out"]
        s["q"], s["e"] = _pack(normal(T, D))
        s["dy"] = (0.05 * normal(T, N)).to(torch.bfloat16)
    if op.startswith("residual"):
        s["w_pre"] = 1.0 + 0.1 * normal(D)
        s["w_post"] = 1.0 + 0.1 * normal(D) if case["post"] else None
        s["gate"] = {"none": None, "channel": 0.5 + 0.2 * normal(D), "element": normal(T, D).to(dt)}[case["gate"]]
        s["scale"] = 0.75
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _policy(s):
    z, w = s["logits"].float(), s["weight"]
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    at = s["labels"].long()[:, None]
    kept = w != 0
    logp = torch.where(kept, (z.gather(1, at) - top - torch.log(total))[:, 0], torch.zeros_like(w))
    ratio = torch.exp(logp - s["logp_old"])
    A = s["advantage"]
    clipped = torch.where(A > 0, ratio > 1.2, ratio < 0.8) & (A != 0)
    loss = -torch.minimum(ratio * A, ratio.clamp(0.8, 1.2) * A)
    slope = torch.where(clipped, torch.zeros_like(A), -ratio * A)
    kl = torch.zeros_like(A)
    if s["logp_ref"] is not None:
        d = s["logp_ref"] - logp
        kl = torch.exp(d) - d - 1.0
        loss = loss + 0.05 * kl
        slope = slope + 0.05 * (1.0 - torch.exp(d))
    zero = torch.zeros_like(A)
    slope = torch.where(kept, w * slope, zero)
    grad = e / total * -slope[:, None]
    grad.scatter_add_(1, at, slope[:, None])
    return {"loss": (torch.where(kept, loss, zero) * w).sum(), "kl": (torch.where(kept, kl, zero) * w).sum(),
            "clipped": (torch.where(kept & clipped, w, zero)).sum(), "logp": logp,
            "dlogits": torch.where(kept[:, None], grad, zero[:, None]).to(s["logits"].dtype)}


def _preference(s, smoothing, beta=0.1):
    z = s["logits"].float()
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    counted = s["labels"] >= 0
    at = s["labels"].clamp(min=0).long()[:, None]
    logp = torch.where(counted, (z.gather(1, at) - top - torch.log(total))[:, 0], torch.zeros((), device=z.device))
    row = torch.arange(z.shape[0], device=z.device)
    member = (row >= s["offsets"][:-1, None]) & (row < s["offsets"][1:, None])  # [answers, tokens]
    answer = torch.where(member, logp, torch.zeros_like(logp)).sum(1)
    margin = answer - s["logp_ref"]
    h = beta * (margin[0::2] - margin[1::2])
    soft = torch.log1p(torch.exp(-h.abs()))  # -log sigmoid(h) = soft + max(-h, 0)
    pair = (1.0 - smoothing) * (soft + (-h).clamp(min=0)) + smoothing * (soft + h.clamp(min=0))
    scale = 1.0 / h.numel()
    c = scale * beta * (1.0 / (1.0 + torch.exp(-h)) - (1.0 - smoothing))
    signed = torch.stack([c, -c], 1).reshape(-1)
    slope = torch.where(member, signed[:, None], torch.zeros_like(signed[:, None])).sum(0) * counted
    grad = e / total * -slope[:, None]
    grad.scatter_add_(1, at, slope[:, None])
    return {"loss": pair.sum() * scale, "pair_loss": pair, "seq_logp": answer, "dlogits": grad.to(s["logits"].dtype)}


def _gate(s):
    g = s["gate"]
    if g is None:
        return None
    return g if g.dim() == 1 else 1.0 / (1.0 + torch.exp(-g.float()))


def _residual_forward(s):
    x, h, g = s["x"].float(), s["h"].float(), _gate(s)
    u = h
    if s["w_post"] is not None:
        u = h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * s["w_post"]
    y = s["scale"] * x + (u if g is None else g * u)
    n = y / torch.sqrt((y * y).mean(1, keepdim=True) + EPS) * s["w_pre"]
    return {"y": y.to(s["x"].dtype), "n": n.to(s["x"].dtype)}


def _residual_backward(s):
    y, h, dn, dt = s["y"].float(), s["h"].float(), s["dn"].float(), s["y"].dtype
    g = _gate(s)
    ry = 1.0 / torch.sqrt((y * y).mean(1, keepdim=True) + EPS)
    a = dn * s["w_pre"]
    yn = y * ry
    dyt = s["dy"].float() + ry * (a - yn * (a * yn).mean(1, keepdim=True))
    out = {"dx": (s["scale"] * dyt).to(dt), "dw_pre": (dn * yn).sum(0)}
    rh = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    hn = h * rh
    u = h if s["w_post"] is None else hn * s["w_post"]
    if g is not None and s["gate"].dim() == 1:
        out["dgate"] = (dyt * u).sum(0)
    elif g is not None:
        out["dgate"] = (dyt * u * g * (1.0 - g)).to(dt)
    du = dyt if g is None else dyt * g
    if s["w_post"] is None:
        out["dh"] = du.to(dt)
    else:
        out["dw_post"] = (du * hn).sum(0)
        b = du * s["w_post"]
        out["dh"] = (rh * (b - hn * (b * hn).mean(1, keepdim=True))).to(dt)
    return out


def _pack(x):
    """int8 values [T, W] and biased exponents uint8 [T, W / 32] of x [T, D], W = D rounded up to 32."""
    T, D = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -D % 32)).reshape(T, -1, 32)
    m, e = torch.frexp(x.abs().amax(2))  # amax = m 2^e, 0.5 <= m < 1: the smallest power with amax <= 127 2^k
    k = e - 7 + (m > 127.0 / 128.0).int()
    k = torch.where(m == 0, torch.full_like(k, -127), k.clamp(min=-127))
    q = torch.round(torch.ldexp(torch.ldexp(x, -(k // 2)[:, :, None]), -(k - k // 2)[:, :, None]))
    return q.to(torch.int8).reshape(T, -1), (k + 127).to(torch.uint8)


def _unpack(q, e, D):
    T = q.shape[0]
    x = torch.ldexp(q.float().reshape(T, -1, 32), e.int()[:, :, None] - 127)
    return x.reshape(T, -1)[:, :D]


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "policy":
            return _policy(s)
        if op == "preference":
            return _preference(s, case["smoothing"])
        if op == "residual_forward":
            return _residual_forward(s)
        if op == "residual_backward":
            return _residual_backward(s)
        if op == "ckpt8":
            q, e = _pack(s["x"])
            return {"values": _unpack(q, e, case["width"]).to(s["x"].dtype)}
        return {"dw": _unpack(s["q"], s["e"], case["width"]).t() @ s["dy"].float()}
    llm = _llm or _calls()
    if op == "policy":
        r = llm.policy_loss(s["logits"], s["labels"], s["logp_old"], s["advantage"], s["weight"], logp_ref=s["logp_ref"],
                            clip_low=0.2, clip_high=0.2, kl_coef=0.05 if case["kl"] else 0.0)
        return {"loss": r.loss, "kl": r.kl, "clipped": r.clipped, "logp": r.logp, "dlogits": r.dlogits}
    if op == "preference":
        r = llm.preference_loss(s["logits"], s["labels"], s["offsets"], s["logp_ref"], beta=0.1, smoothing=case["smoothing"])
        return {"loss": r.loss, "pair_loss": r.pair_loss, "seq_logp": r.seq_logp, "dlogits": r.dlogits}
    if op == "residual_forward":
        y, n = llm.residual_norm(s["x"], s["h"], s["w_pre"], w_post=s["w_post"], gate=s["gate"], scale=s["scale"], eps=EPS)
        return {"y": y, "n": n}
    if op == "residual_backward":
        r = llm.residual_norm_backward(s["dn"], s["dy"], s["y"], s["h"], s["w_pre"], w_post=s["w_post"], gate=s["gate"],
                                       scale=s["scale"], eps=EPS)
        return {k: v for k, v in r._asdict().items() if v is not None}
    if op == "ckpt8":
        return {"values": llm.ckpt8_dequantize(llm.ckpt8_quantize(s["x"]), s["x"].dtype)}
    return {"dw": llm.ckpt8_wgrad(llm.Ckpt8(s["q"], s["e"], case["width"]), s["dy"])}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    op = case["op"]
    if op in ("policy", "preference"):
        V, es = case["vocab"], SIZE[case["dtype"]]
        if op == "policy":
            T, read, small = case["tokens"], _kept(case), 24 * case["tokens"]
        else:
            lens = _lengths(case)
            T, read, small = sum(lens), sum(n - n // 4 for n in lens), 4 * sum(lens)
        return {"bytes": (read + T) * V * es + small, "flops": 8 * read * V}
    T, D = case["tokens"], case["width"]
    if op == "wgrad":
        N, W = case["out"], -(-D // 32) * 32
        return {"bytes": T * (W + W // 32) + 2 * T * N + 4 * D * N, "flops": 2 * T * D * N}
    es = SIZE[case["dtype"]]
    if op == "ckpt8":
        W = -(-D // 32) * 32
        return {"bytes": 2 * T * (D * es + W + W // 32), "flops": 4 * T * D}
    gate = case["gate"] == "element"
    if op == "residual_forward":
        return {"bytes": T * D * es * (4 + gate) + 8 * D, "flops": 12 * T * D}
    return {"bytes": T * D * es * (6 + 2 * gate) + 20 * D, "flops": 30 * T * D}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    d = lambda t: None if t is None else t.double()  # noqa: E731
    if op == "policy":
        lp, soft = torch.zeros(case["tokens"], device=DEV, dtype=torch.float64), torch.log_softmax(s["logits"].double(), 1)
        y, w, A = s["labels"].long(), d(s["weight"]), d(s["advantage"])
        on = w > 0
        lp = soft[torch.arange(len(y), device=DEV), y] * on
        r = (lp - d(s["logp_old"])).exp()
        up, down = (A >= 0) & (r > 1.2), (A < 0) & (r < 0.8)
        gone = (up & (A > 0)) | down
        each = torch.where(up, -1.2 * A, torch.where(down, -0.8 * A, -r * A))
        by = torch.where(gone, 0.0, -r * A)
        kl = torch.zeros_like(A)
        if case["kl"]:
            x = (d(s["logp_ref"]) - lp).exp()
            kl = x - 1 - x.log()
            each, by = each + 0.05 * kl, by + 0.05 * (1 - x)
        by = by * w
        grad = soft.exp_().mul_(-by[:, None])
        grad[torch.arange(len(y), device=DEV), y] += by
        return {"loss": (w * each).sum(), "kl": (w * kl).sum(), "clipped": (w * gone).sum(), "logp": lp, "dlogits": grad}
    if op == "preference":
        soft, lens, beta, eps = torch.log_softmax(s["logits"].double(), 1), _lengths(case), 0.1, case["smoothing"]
        y = s["labels"].long()
        on = y >= 0
        lp = soft.gather(1, y.clamp(min=0)[:, None])[:, 0] * on
        total = torch.stack([p.sum() for p in lp.split(lens)])
        over = total - d(s["logp_ref"])
        h = beta * (over[::2] - over[1::2])
        ls = torch.nn.functional.logsigmoid
        pair = -(1 - eps) * ls(h) - eps * ls(-h)
        c = beta * (torch.sigmoid(h) - 1 + eps) / len(h)
        by = torch.repeat_interleave(torch.stack((c, -c), 1).flatten(), torch.tensor(lens, device=DEV)) * on
        grad = soft.exp_().mul_(-by[:, None])
        grad[torch.arange(len(y), device=DEV), y.clamp(min=0)] += by
        return {"loss": pair.mean(), "pair_loss": pair, "seq_logp": total, "dlogits": grad}
    if op == "ckpt8":
        x = d(s["x"])
        T, D = x.shape
        W = -(-D // 32) * 32
        blocks = torch.zeros(T, W, device=DEV, dtype=torch.float64)
        blocks[:, :D] = x
        blocks = blocks.view(T, W // 32, 32)
        top = blocks.abs().amax(-1, keepdim=True)
        step = torch.exp2(torch.ceil(torch.log2((top / 127).clamp(min=2.0 ** -127))))
        step = torch.where(step * 127 < top, step * 2, step)
        step = torch.where((step * 63.5 >= top) & (step > 2.0 ** -127), step / 2, step)
        return {"values": ((blocks / step).round() * step).reshape(T, W)[:, :D]}
    if op == "wgrad":
        x = s["q"].double() * torch.exp2(s["e"].double() - 127).repeat_interleave(32, 1)
        return {"dw": torch.einsum("ti,to->io", x[:, : case["width"]], d(s["dy"]))}
    rms = lambda v: (v.square().mean(1, keepdim=True) + EPS).sqrt()  # noqa: E731
    h, w1, w2, g = d(s["h"]), d(s["w_post"]), d(s["w_pre"]), d(s["gate"])
    u = h if w1 is None else h / rms(h) * w1
    G = torch.ones((), device=DEV, dtype=torch.float64) if g is None else g if g.dim() == 1 else torch.sigmoid(g)
    if op == "residual_forward":
        y = s["scale"] * d(s["x"]) + G * u
        return {"y": y, "n": y / rms(y) * w2}
    y, dn = d(s["y"]), d(s["dn"])
    q = rms(y)
    inner = (dn * w2 * y).mean(1, keepdim=True)
    top = d(s["dy"]) + dn * w2 / q - y * inner / q ** 3
    out = {"dx": s["scale"] * top, "dw_pre": (dn * y / q).sum(0)}
    if g is not None:
        out["dgate"] = (top * u).sum(0) if g.dim() == 1 else top * u * G * (1 - G)
    back = top * G
    if w1 is None:
        out["dh"] = back
    else:
        p = rms(h)
        out["dw_post"] = (back * h / p).sum(0)
        out["dh"] = back * w1 / p - h * (back * w1 * h).mean(1, keepdim=True) / p ** 3
    return out
