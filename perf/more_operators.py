"""Cases for measuring the operators between a language model's tokens and its logits (paper_2308_15164_b200.llm).

One case is one call, or the calls of one layer, of a micro-batch's forward or backward pass:

* ``embed``                scaled embedding lookup
* ``embed_backward``       its gradient, the whole table
* ``layer_norm``           layer norm
* ``layer_norm_backward``  its gradients, with the gradient that comes around the norm
* ``linear``               product with bias, activation and residual
* ``linear_backward``      the way back through a layer: gradient of the input (times the derivative of the activation that made it), of
                           weight and bias
* ``recurrence``           gated linear recurrence over packed sequences
* ``recurrence_backward``  its gradients
* ``recurrence_step``      one token of each sequence

With ``own`` false ``run`` computes the plain form: elementary torch operations in 32 bits, rounded once at the end.
"""

import math

import numpy as np
import torch

_llm = None  # the package, imported where the framework's own calls are made

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-5


def _calls():
    global _llm
    if _llm is None:
        from paper_2308_15164_b200 import llm

        _llm = llm
    return _llm


def listed():
    return [
        # a long micro-batch into the residual stream, a few positions of padding
        {"name": "embed_bf16", "op": "embed", "tokens": 16384, "vocab": 32000, "width": 4096, "dtype": "bf16", "pad": True},
        # a handful of tokens of a small vocabulary, fp32 activations of odd width: the time of the call itself
        {"name": "embed_backward_few", "op": "embed_backward", "tokens": 77, "vocab": 777, "width": 333, "dtype": "f32", "pad": False},
        # an ordinary micro-batch: most rows of the table get no token and are zero
        {"name": "embed_backward_bf16", "op": "embed_backward", "tokens": 8192, "vocab": 32000, "width": 2048, "dtype": "bf16", "pad": True},
        # a norm of very few tokens
        {"name": "layer_norm_few", "op": "layer_norm", "tokens": 5, "width": 1024, "dtype": "bf16", "bias": True},
        # the way back through a pre-norm of a long micro-batch of a wide model, the residual stream's gradient added
        {"name": "layer_norm_backward_bf16", "op": "layer_norm_backward", "tokens": 16384, "width": 4096, "dtype": "bf16", "bias": True, "skip": True},
        # fp32 activations, odd sizes
        {"name": "layer_norm_backward_f32_odd", "op": "layer_norm_backward", "tokens": 1003, "width": 1537, "dtype": "f32", "bias": True, "skip": False},
        # the first layer of an MLP: bias and activation, pre-activation kept for the way back
        {"name": "linear_gelu", "op": "linear", "tokens": 8192, "in": 2048, "out": 8192, "act": "gelu", "keep": True, "residual": False},
        # odd sizes on every side, as of a ragged micro-batch and a small head, with the residual stream added
        {"name": "linear_residual_odd", "op": "linear", "tokens": 515, "in": 1000, "out": 1111, "act": "none", "keep": False, "residual": True},
        # the way back through the second layer of an MLP, down to the first one's pre-activation
        {"name": "linear_backward", "op": "linear_backward", "tokens": 4096, "in": 8192, "out": 2048, "act": "gelu", "bias": True},
        # one token for each of sixteen rollouts
        {"name": "recurrence_step", "op": "recurrence_step", "seqs": 16, "width": 2048, "dtype": "bf16", "kind": "blend"},
        # one very long document through a narrow layer: the time axis is all there is to work on at once
        {"name": "recurrence_long", "op": "recurrence", "tokens": 65536, "seqs": 1, "width": 1024, "dtype": "bf16", "kind": "blend", "state": False},
        # the way back through a wide layer over packed answers of ragged lengths that continue a prompt's state
        {"name": "recurrence_backward", "op": "recurrence_backward", "tokens": 16384, "seqs": 24, "width": 4096, "dtype": "bf16", "kind": "blend", "state": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["embed", "embed_backward", "embed_backward", "layer_norm", "layer_norm_backward", "linear", "linear", "linear_backward",
                     "recurrence", "recurrence_backward", "recurrence_step"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("embed", "embed_backward"):
        width = _log_int(rng, 32, 8192)
        vocab = _log_int(rng, 100, min(152064, (1 << 27) // width))
        return {"op": op, "tokens": _log_int(rng, 1, min(65536, (1 << 26) // width)), "vocab": vocab, "width": width, "dtype": dtype,
                "pad": rng.random() < 0.5}
    if op in ("layer_norm", "layer_norm_backward"):
        width = _log_int(rng, 32, 8192)
        case = {"op": op, "tokens": _log_int(rng, 1, min(65536, (1 << 26) // width)), "width": width, "dtype": dtype, "bias": rng.random() < 0.7}
        if op == "layer_norm_backward":
            case["skip"] = rng.random() < 0.5
        return case
    if op in ("linear", "linear_backward"):
        inner, out = _log_int(rng, 16, 8192), _log_int(rng, 16, 8192)
        tokens = _log_int(rng, 1, min(8192, (1 << 36) // (inner * out)))
        case = {"op": op, "tokens": tokens, "in": inner, "out": out, "act": rng.choice(["none", "relu", "gelu", "silu"])}
        if op == "linear":
            return case | {"keep": case["act"] != "none" and rng.random() < 0.5, "residual": rng.random() < 0.5}
        return case | {"bias": rng.random() < 0.5}
    width, kind = _log_int(rng, 16, 8192), rng.choice(["blend", "add"])
    if op == "recurrence_step":
        return {"op": op, "seqs": _log_int(rng, 1, 512), "width": width, "dtype": dtype, "kind": kind}
    tokens = _log_int(rng, 1, min(65536, (1 << 26) // width))
    return {"op": op, "tokens": tokens, "seqs": _log_int(rng, 1, min(64, tokens)), "width": width, "dtype": dtype, "kind": kind, "state": rng.random() < 0.5}


# ---------------------------------------------------------------------------------------------- inputs
def _shares(vocab):
    """How often the tokens of a vocabulary occur, most frequent first: the usual power law."""
    p = 1.0 / (np.arange(vocab) + 2.7)
    return p / p.sum()


def _distinct(case):
    """Expected number of different tokens."""
    n = case["tokens"] - (case["tokens"] // 16 if case["pad"] else 0)
    return int(round(float((1.0 - (1.0 - _shares(case["vocab"])) ** n).sum())))


def _lengths(case):
    """Tokens of each sequence: ragged, by a fixed pattern; all of them together are the case's tokens."""
    n, parts = case["tokens"], case["seqs"]
    share = [1.0 + (q * 7919 % 13) / 4.0 for q in range(parts)]
    ends = [int(n * sum(share[: q + 1]) / sum(share)) for q in range(parts)]
    ends[-1] = n
    return [b - a for a, b in zip([0] + ends[:-1], ends)]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2654435761 % (1 << 31) + 29)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    op, s = case["op"], {"case": dict(case)}
    if op.startswith("embed"):
        T, V, D, dt = case["tokens"], case["vocab"], case["width"], DTYPES[case["dtype"]]
        order = torch.randperm(V, generator=g, device=DEV)  # frequent tokens have any number
        share = torch.from_numpy(_shares(V)).to(DEV)
        ids = order[torch.multinomial(share, T, replacement=True, generator=g)].to(torch.int32)
        if case["pad"]:
            ids[T - T // 16:] = -1
        s |= {"ids": ids, "scale": math.sqrt(D)}
        if op == "embed":
            s["table"] = 0.02 * normal(V, D)
        else:
            s["dy"] = (0.05 * normal(T, D)).to(dt)
        return s
    if op.startswith("layer_norm"):
        T, D, dt = case["tokens"], case["width"], DTYPES[case["dtype"]]
        x = normal(T, D) * 3.0 + 0.5
        x[:, :: max(1, D // 8)] *= 12.0  # a residual stream has a few channels far above the others
        s |= {"x": x.to(dt), "w": 1.0 + 0.1 * normal(D), "b": 0.1 * normal(D) if case["bias"] else None}
        if op == "layer_norm_backward":
            s["dn"] = (0.1 * normal(T, D)).to(dt)
            s["skip"] = (0.1 * normal(T, D)).to(dt) if case["skip"] else None
        return s
    if op.startswith("linear"):
        T, K, N, bf = case["tokens"], case["in"], case["out"], torch.bfloat16
        s["w"] = (normal(K, N) / math.sqrt(K)).to(bf)
        if op == "linear":
            s |= {"x": normal(T, K).to(bf), "b": 0.1 * normal(N), "residual": normal(T, N).to(bf) if case["residual"] else None}
            return s
        z = normal(T, K).to(bf)
        s |= {"x": _act(case["act"], z.float()).to(bf), "z": None if case["act"] == "none" else z, "dy": (0.05 * normal(T, N)).to(bf)}
        return s
    D, dt = case["width"], DTYPES[case["dtype"]]
    T = case["seqs"] if op == "recurrence_step" else case["tokens"]
    s |= {"x": normal(T, D).to(dt), "g": (2.0 + 1.5 * normal(T, D)).to(dt)}  # gates that mostly keep
    if op == "recurrence_step":
        s["h"] = normal(T, D)
        return s
    lens = _lengths(case)
    s["offsets"] = torch.tensor([0] + lens, device=DEV).cumsum(0).to(torch.int32)
    s["h0"] = normal(len(lens), D) if case["state"] else None
    if op == "recurrence_backward":
        s["y"] = _recurrence(s)["y"]
        s["dy"] = (0.05 * normal(T, D)).to(dt)
        s["dlast"] = 0.05 * normal(len(lens), D) if case["state"] else None
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _act(act, z):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(act, z):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    a = 1.0 / (1.0 + torch.exp(-z))
    return a * (1.0 + z * (1.0 - a))


def _embed(s):
    ids = s["ids"].long()
    known = ((ids >= 0) & (ids < s["table"].shape[0]))[:, None]
    rows = s["table"][ids.clamp(0, s["table"].shape[0] - 1)] * s["scale"]
    return {"y": torch.where(known, rows, torch.zeros_like(rows)).to(DTYPES[s["case"]["dtype"]])}


def _embed_backward(s):
    V, D = s["case"]["vocab"], s["case"]["width"]
    ids = s["ids"].long()
    known = (ids >= 0) & (ids < V)
    rows = torch.where(known[:, None], s["dy"].float(), torch.zeros((), device=DEV))
    out = torch.zeros(V, D, device=DEV)
    out.index_add_(0, torch.where(known, ids, torch.zeros_like(ids)), rows)
    return {"dtable": out * s["scale"]}


def _norm_of(x):
    c = x - x.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    return c * r, r


def _layer_norm(s):
    n = _norm_of(s["x"].float())[0] * s["w"]
    if s["b"] is not None:
        n = n + s["b"]
    return {"n": n.to(s["x"].dtype)}


def _layer_norm_backward(s):
    xh, r = _norm_of(s["x"].float())
    dn = s["dn"].float()
    a = dn * s["w"]
    dx = r * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    if s["skip"] is not None:
        dx = dx + s["skip"].float()
    out = {"dx": dx.to(s["x"].dtype), "dw": (dn * xh).sum(0)}
    if s["b"] is not None:
        out["db"] = dn.sum(0)
    return out


def _linear(s):
    case = s["case"]
    z = s["x"].float() @ s["w"].float() + s["b"]
    y = _act(case["act"], z)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(torch.bfloat16)}
    if case["keep"]:
        out["z"] = z.to(torch.bfloat16)
    return out


def _linear_backward(s):
    case, dy = s["case"], s["dy"].float()
    dx = dy @ s["w"].float().t()
    if s["z"] is not None:
        dx = dx * _act_slope(case["act"], s["z"].float())
    out = {"dx": dx.to(torch.bfloat16), "dw": s["x"].float().t() @ dy}
    if case["bias"]:
        out["db"] = dy.sum(0)
    return out


def _starts(s):
    """[T] first rows of sequences, and the sequence of each row."""
    T = s["x"].shape[0]
    row = torch.arange(T, device=DEV)
    seq = torch.bucketize(row, s["offsets"][1:].long(), right=True)
    return row == s["offsets"].long()[seq], seq


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the rows by doubling."""
    a, b, step = a.clone(), b.clone(), 1
    while step < a.shape[0]:
        b = torch.cat((b[:step], b[step:] + a[step:] * b[:-step]))
        a = torch.cat((a[:step], a[step:] * a[:-step]))
        step *= 2
    return b


def _recurrence(s):
    kind, x, g = s["case"]["kind"], s["x"].float(), s["g"].float()
    a = 1.0 / (1.0 + torch.exp(-g))
    b = x / (1.0 + torch.exp(g)) if kind == "blend" else x
    first, seq = _starts(s)
    if s["h0"] is not None:
        b = torch.where(first[:, None], b + a * s["h0"][seq], b)
    h = _scan(torch.where(first[:, None], torch.zeros_like(a), a), b)
    end = s["offsets"].long()
    last = h[(end[1:] - 1).clamp(min=0)]
    before = torch.zeros_like(last) if s["h0"] is None else s["h0"]
    last = torch.where((end[1:] > end[:-1])[:, None], last, before)
    return {"y": h.to(s["x"].dtype), "last": last}


def _recurrence_backward(s):
    kind, x, g, y, dt = s["case"]["kind"], s["x"].float(), s["g"].float(), s["y"].float(), s["x"].dtype
    a, rest = 1.0 / (1.0 + torch.exp(-g)), 1.0 / (1.0 + torch.exp(g))
    first, seq = _starts(s)
    zero = torch.zeros((), device=DEV)
    d = s["dy"].float()
    final = torch.cat((first[1:], first.new_ones(1)))
    if s["dlast"] is not None:
        d = torch.where(final[:, None], d + s["dlast"][seq], d)
    follow = torch.cat((a[1:], torch.zeros_like(a[:1])))
    d = _scan(torch.where(final[:, None], zero, follow).flip(0), d.flip(0)).flip(0)
    before = torch.cat((torch.zeros_like(y[:1]), y[:-1]))
    begin = zero if s["h0"] is None else s["h0"][seq]
    before = torch.where(first[:, None], begin, before)
    out = {"dx": (d * rest if kind == "blend" else d).to(dt), "dg": (d * (before - x if kind == "blend" else before) * a * rest).to(dt)}
    if s["h0"] is not None:
        at = s["offsets"].long()
        there = (at[1:] > at[:-1])[:, None]
        row = at[:-1].clamp(max=x.shape[0] - 1)
        out["dh0"] = torch.where(there, (a * d)[row], s["dlast"] if s["dlast"] is not None else zero)
    return out


def _recurrence_step(s):
    x, g = s["x"].float(), s["g"].float()
    h = s["h"] / (1.0 + torch.exp(-g)) + (x / (1.0 + torch.exp(g)) if s["case"]["kind"] == "blend" else x)
    return {"y": h.to(s["x"].dtype), "h": h}


_PLAIN = {"embed": _embed, "embed_backward": _embed_backward, "layer_norm": _layer_norm, "layer_norm_backward": _layer_norm_backward, "linear": _linear,
          "linear_backward": _linear_backward, "recurrence": _recurrence, "recurrence_backward": _recurrence_backward, "recurrence_step": _recurrence_step}


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return _PLAIN[op](s)
    llm = _llm or _calls()
    if op == "embed":
        return {"y": llm.embed(s["ids"], s["table"], scale=s["scale"], dtype=DTYPES[case["dtype"]])}
    if op == "embed_backward":
        return {"dtable": llm.embed_backward(s["dy"], s["ids"], case["vocab"], scale=s["scale"])}
    if op == "layer_norm":
        return {"n": llm.layer_norm(s["x"], s["w"], s["b"], eps=EPS)}
    if op == "layer_norm_backward":
        r = llm.layer_norm_backward(s["dn"], s["x"], s["w"], dskip=s["skip"], bias=case["bias"], eps=EPS)
        return {k: v for k, v in r._asdict().items() if v is not None}
    if op == "linear":
        r = llm.linear(s["x"], s["w"], s["b"], act=case["act"], residual=s["residual"], keep=case["keep"])
        return {"y": r.y, "z": r.z} if case["keep"] else {"y": r.y}
    if op == "linear_backward":
        dx = llm.linear_dgrad(s["dy"], s["w"], act=case["act"], z=s["z"])
        r = llm.linear_wgrad(s["x"], s["dy"], bias=case["bias"])
        return {"dx": dx, "dw": r.dw, "db": r.db} if case["bias"] else {"dx": dx, "dw": r.dw}
    if op == "recurrence":
        r = llm.gated_recurrence(s["x"], s["g"], s["offsets"], h0=s["h0"], kind=case["kind"])
        return {"y": r.y, "last": r.last}
    if op == "recurrence_backward":
        r = llm.gated_recurrence_backward(s["dy"], s["x"], s["g"], s["y"], s["offsets"], h0=s["h0"], dlast=s["dlast"], kind=case["kind"])
        return {k: v for k, v in r._asdict().items() if v is not None}
    r = llm.gated_recurrence_step(s["x"], s["g"], s["h"], kind=case["kind"])
    return {"y": r.y, "h": r.last}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    op = case["op"]
    if op.startswith("linear"):
        T, K, N = case["tokens"], case["in"], case["out"]
        if op == "linear":
            return {"bytes": 2 * (T * K + K * N) + 4 * N + 2 * T * N * (1 + case["keep"] + case["residual"]), "flops": 2 * T * K * N}
        return {"bytes": 2 * (2 * T * K + K * N + T * N) + 4 * K * N + (2 * T * K if case["act"] != "none" else 0) + (4 * N if case["bias"] else 0),
                "flops": 4 * T * K * N}
    D, es = case["width"], SIZE[case["dtype"]]
    if op == "recurrence_step":
        return {"bytes": case["seqs"] * D * (3 * es + 8), "flops": 10 * case["seqs"] * D}
    T = case["tokens"]
    if op == "embed":
        return {"bytes": T * D * es + 4 * D * _distinct(case) + 4 * T, "flops": T * D}
    if op == "embed_backward":
        kept = T - (T // 16 if case["pad"] else 0)
        return {"bytes": kept * D * es + 4 * D * case["vocab"] + 4 * T, "flops": 2 * kept * D}
    if op == "layer_norm":
        return {"bytes": 2 * T * D * es + 4 * D * (1 + case["bias"]), "flops": 8 * T * D}
    if op == "layer_norm_backward":
        return {"bytes": T * D * es * (3 + case["skip"]) + 4 * D * (2 + case["bias"]), "flops": 16 * T * D}
    states = 4 * D * case["seqs"]
    if op == "recurrence":
        return {"bytes": 3 * T * D * es + states * (1 + case["state"]), "flops": 10 * T * D}
    return {"bytes": 6 * T * D * es + states * (3 if case["state"] else 0), "flops": 16 * T * D}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    d = lambda t: None if t is None else t.double()  # noqa: E731
    F = torch.nn.functional
    if op == "embed":
        table = torch.cat((d(s["table"]) * s["scale"], torch.zeros(1, case["width"], device=DEV, dtype=torch.float64)))
        return {"y": table[torch.where(s["ids"] < 0, case["vocab"], s["ids"]).long()]}
    if op == "embed_backward":
        out = torch.zeros(case["vocab"] + 1, case["width"], device=DEV, dtype=torch.float64)
        at = torch.where(s["ids"] < 0, case["vocab"], s["ids"]).long()
        out.scatter_add_(0, at[:, None].expand(-1, case["width"]), d(s["dy"]))
        return {"dtable": out[:-1] * s["scale"]}
    if op == "layer_norm":
        x = d(s["x"])
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        return {"n": (x - mean) / (var + EPS).sqrt() * d(s["w"]) + (0.0 if s["b"] is None else d(s["b"]))}
    if op == "layer_norm_backward":
        x, w, dn = d(s["x"]), d(s["w"]), d(s["dn"])
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        sd = (var + EPS).sqrt()
        up, c = dn * w, x - mean
        dx = (up - up.mean(1, keepdim=True)) / sd - c * (up * c).mean(1, keepdim=True) / sd ** 3
        out = {"dx": dx if s["skip"] is None else dx + d(s["skip"]), "dw": torch.einsum("td,td->d", dn, c / sd)}
        if case["bias"]:
            out["db"] = torch.einsum("td->d", dn)
        return out
    if op == "linear":
        z = torch.addmm(d(s["b"]), d(s["x"]), d(s["w"]))
        y = {"none": lambda v: v, "relu": torch.relu, "gelu": F.gelu, "silu": F.silu}[case["act"]](z)
        out = {"y": y if s["residual"] is None else y + d(s["residual"])}
        if case["keep"]:
            out["z"] = z
        return out
    if op == "linear_backward":
        dy = d(s["dy"])
        dx = torch.einsum("to,io->ti", dy, d(s["w"]))
        if s["z"] is not None:
            z = d(s["z"])
            p = torch.special.ndtr(z)
            a = torch.sigmoid(z)
            dx = dx * {"relu": lambda: (z > 0).double(), "gelu": lambda: p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),
                       "silu": lambda: a + z * a * torch.sigmoid(-z)}[case["act"]]()
        out = {"dx": dx, "dw": torch.einsum("ti,to->io", d(s["x"]), dy)}
        if case["bias"]:
            out["db"] = torch.einsum("to->o", dy)
        return out
    x, keep, new = d(s["x"]), torch.sigmoid(d(s["g"])), torch.sigmoid(-d(s["g"]))
    feed = x * new if case["kind"] == "blend" else x
    if op == "recurrence_step":
        h = keep * s["h"].double() + feed
        return {"y": h, "h": h}
    # one row after the other, all sequences side by side from their ends (they are ragged: those that have ended wait)
    lens = _lengths(case)
    ends = np.cumsum(lens).tolist()
    begins = [e - n for e, n in zip(ends, lens)]
    state = torch.zeros(len(lens), case["width"], device=DEV, dtype=torch.float64) if s["h0"] is None else d(s["h0"]).clone()
    rows = [[begins[q] + i for q in range(len(lens)) if i < lens[q]] for i in range(max(lens))]
    live = [[q for q in range(len(lens)) if i < lens[q]] for i in range(max(lens))]
    flat_rows = torch.tensor([r for part in rows for r in part], device=DEV)
    flat_live = torch.tensor([r for part in live for r in part], device=DEV)
    at = np.cumsum([0] + [len(part) for part in rows]).tolist()
    if op == "recurrence":
        y = torch.empty_like(x)
        for i in range(len(rows)):
            r, q = flat_rows[at[i]:at[i + 1]], flat_live[at[i]:at[i + 1]]
            v = keep[r] * state[q] + feed[r]
            state[q] = v
            y[r] = v
        return {"y": y, "last": state}
    y, back = d(s["y"]), torch.zeros_like(state) if s["dlast"] is None else d(s["dlast"]).clone()
    up = d(s["dy"]).clone()
    for i in reversed(range(len(rows))):
        r, q = flat_rows[at[i]:at[i + 1]], flat_live[at[i]:at[i + 1]]
        v = up[r] + back[q]
        up[r] = v
        back[q] = v * keep[r]
    before = torch.roll(y, 1, 0)
    for q in range(len(lens)):
        if lens[q]:
            before[begins[q]] = state[q]
    out = {"dx": up * new if case["kind"] == "blend" else up, "dg": up * keep * new * (before - x if case["kind"] == "blend" else before)}
    if s["h0"] is not None:
        out["dh0"] = back
    return out
