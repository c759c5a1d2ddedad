"""Embedding, layer norm, linear layer and recurrence refuse bad arguments before they touch a GPU (every call here returns from its
checks), and the 64-bit definitions that the GPU tests compare with hold against autograd."""

import pytest
import torch

from tests import llm_layers_reference as R
from tests.test_llm_refusals import B, NAN, INF, P, WS  # noqa: F401  (B: the fixture)


def embed(B, **kw):  # noqa: F811
    a = dict(ids=P, T=4, table=2 * P, ld_table=16, V=8, D=16, scale=1.0, dtype=1, y=3 * P, ld_y=16) | kw
    return B.lib.abs_embed(*a.values(), None)


def embed_back(B, **kw):  # noqa: F811
    a = dict(dy=P, ld_dy=16, dtype=1, ids=P, T=4, V=8, D=16, scale=1.0, out=2 * P, ld_out=16, acc=0, ws=P, n=WS) | kw
    return B.lib.abs_embed_backward(*a.values(), None)


def norm(B, **kw):  # noqa: F811
    a = dict(x=P, ld_x=16, w=P, b=P, eps=1e-5, dtype=1, T=4, D=16, n=2 * P, ld_n=16) | kw
    return B.lib.abs_layer_norm(*a.values(), None)


def norm_back(B, **kw):  # noqa: F811
    a = dict(dn=P, ld_dn=16, x=P, ld_x=16, skip=P, ld_skip=16, w=P, eps=1e-5, dtype=1, T=4, D=16, dx=2 * P, ld_dx=16, dw=3 * P, db=4 * P, acc=0, ws=P, n=WS) | kw
    return B.lib.abs_layer_norm_backward(*a.values(), None)


def linear(B, **kw):  # noqa: F811
    a = dict(x=P, ld_x=16, w=2 * P, ld_w=24, b=P, act=2, res=3 * P, ld_res=24, dtype=1, T=4, K=16, N=24, y=4 * P, ld_y=24, z=5 * P, ld_z=24, ws=P, n=WS) | kw
    return B.lib.abs_linear(*a.values(), None)


def dgrad(B, **kw):  # noqa: F811
    a = dict(dy=P, ld_dy=24, w=2 * P, ld_w=24, act=2, z=3 * P, ld_z=16, res=4 * P, ld_res=16, dtype=1, T=4, K=16, N=24, dx=5 * P, ld_dx=16, ws=P, n=WS) | kw
    return B.lib.abs_linear_dgrad(*a.values(), None)


def wgrad(B, **kw):  # noqa: F811
    a = dict(x=P, ld_x=16, dy=2 * P, ld_dy=24, T=4, K=16, N=24, dw=3 * P, ld_dw=24, db=4 * P, acc=0, ws=P, n=WS) | kw
    return B.lib.abs_linear_wgrad(*a.values(), None)


def through(B, **kw):  # noqa: F811
    a = dict(dy=P, ld_dy=16, dtype=0, z=2 * P, ld_z=16, act=1, T=4, D=16, dz=3 * P, ld_dz=16) | kw
    return B.lib.abs_activation_backward(*a.values(), None)


def scan(B, **kw):  # noqa: F811
    a = dict(x=P, ld_x=16, g=2 * P, ld_g=16, off=P, seqs=2, h0=P, kind=0, dtype=1, T=400, D=16, y=3 * P, ld_y=16, last=4 * P, ws=P, n=WS) | kw
    return B.lib.abs_recurrence(*a.values(), None)


def scan_back(B, **kw):  # noqa: F811
    a = dict(dy=P, ld_dy=16, x=2 * P, ld_x=16, g=3 * P, ld_g=16, y=4 * P, ld_y=16, off=P, seqs=2, h0=P, dlast=9 * P, kind=0, dtype=1, T=400, D=16, dx=5 * P, ld_dx=16,
             dg=6 * P, ld_dg=16, dh0=7 * P, ws=P, n=WS) | kw
    return B.lib.abs_recurrence_backward(*a.values(), None)


def step(B, **kw):  # noqa: F811
    a = dict(x=P, ld_x=16, g=2 * P, ld_g=16, h=P, kind=0, dtype=1, S=4, D=16, y=3 * P, ld_y=16, out=4 * P) | kw
    return B.lib.abs_recurrence_step(*a.values(), None)


CASES = [
    (embed, dict(dtype=2)), (embed, dict(D=0)), (embed, dict(V=0)), (embed, dict(scale=NAN)), (embed, dict(ld_table=15)), (embed, dict(ld_y=8)), (embed, dict(table=P + 2)),
    (embed, dict(y=P + 1)), (embed, dict(ids=P + 2)), (embed, dict(ids=None)), (embed, dict(table=None)), (embed, dict(y=None)), (embed, dict(y=2 * P)),
    (embed_back, dict(dtype=7)), (embed_back, dict(V=0)), (embed_back, dict(scale=INF)), (embed_back, dict(ld_out=15)), (embed_back, dict(ld_dy=1)), (embed_back, dict(out=None)),
    (embed_back, dict(out=2 * P + 2)), (embed_back, dict(dy=None)), (embed_back, dict(ids=None)), (embed_back, dict(ids=P + 1)), (embed_back, dict(ws=None)),
    (embed_back, dict(ws=P + 64)), (embed_back, dict(out=P)),
    (norm, dict(dtype=4)), (norm, dict(D=0)), (norm, dict(w=None)), (norm, dict(w=P + 2)), (norm, dict(b=P + 1)), (norm, dict(eps=0.0)), (norm, dict(eps=NAN)),
    (norm, dict(ld_x=15)), (norm, dict(ld_n=15)), (norm, dict(x=None)), (norm, dict(n=None)), (norm, dict(x=P + 1)), (norm, dict(n=P, ld_n=24)),
    (norm_back, dict(w=None)), (norm_back, dict(eps=-1.0)), (norm_back, dict(dw=None)), (norm_back, dict(db=3 * P)), (norm_back, dict(db=P + 2)), (norm_back, dict(ws=None)),
    (norm_back, dict(ws=P + 4)), (norm_back, dict(dn=None)), (norm_back, dict(x=None)), (norm_back, dict(dx=None)), (norm_back, dict(ld_skip=3)),
    (norm_back, dict(dx=P, ld_dx=32)),
    (linear, dict(dtype=3)), (linear, dict(act=4)), (linear, dict(K=0)), (linear, dict(N=0)), (linear, dict(ld_x=15)), (linear, dict(ld_w=23)), (linear, dict(ld_res=8)),
    (linear, dict(ld_y=23)), (linear, dict(ld_z=23)), (linear, dict(x=None)), (linear, dict(w=None)), (linear, dict(y=None)), (linear, dict(x=P + 1)), (linear, dict(b=P + 2)),
    (linear, dict(y=P)), (linear, dict(y=2 * P)), (linear, dict(z=P)), (linear, dict(z=4 * P)), (linear, dict(y=3 * P, ld_y=32)), (linear, dict(z=3 * P)),
    (linear, dict(x=P + 2, ws=None)), (linear, dict(ld_w=25, ws=P + 8)),
    (dgrad, dict(dtype=3)), (dgrad, dict(act=9)), (dgrad, dict(act=0)), (dgrad, dict(z=None)), (dgrad, dict(dy=None)), (dgrad, dict(w=None)), (dgrad, dict(dx=None)),
    (dgrad, dict(dx=P)), (dgrad, dict(dx=2 * P)), (dgrad, dict(ld_z=15)), (dgrad, dict(dx=3 * P, ld_dx=24)), (dgrad, dict(dx=3 * P, dtype=0)), (dgrad, dict(ld_dy=25, ws=None)),
    (wgrad, dict(K=0)), (wgrad, dict(N=0)), (wgrad, dict(dw=None)), (wgrad, dict(dw=P + 2)), (wgrad, dict(db=3 * P)), (wgrad, dict(db=P + 2)), (wgrad, dict(x=None)),
    (wgrad, dict(dy=None)), (wgrad, dict(dw=P)), (wgrad, dict(db=2 * P)), (wgrad, dict(ld_dw=23)), (wgrad, dict(ws=None)),
    (through, dict(dtype=2)), (through, dict(act=5)), (through, dict(D=0)), (through, dict(dy=None)), (through, dict(z=None)), (through, dict(dz=None)), (through, dict(ld_dz=1)),
    (through, dict(dz=P)), (through, dict(dz=2 * P, ld_dz=20)),
    (scan, dict(dtype=2)), (scan, dict(kind=2)), (scan, dict(D=0)), (scan, dict(off=None)), (scan, dict(off=P + 2)), (scan, dict(h0=P + 1)), (scan, dict(last=P + 2)), (scan, dict(last=P)),
    (scan, dict(x=None)), (scan, dict(g=None)), (scan, dict(y=None)), (scan, dict(ld_x=15)), (scan, dict(ld_y=15)), (scan, dict(y=P, ld_y=20)), (scan, dict(ws=None)),
    (scan, dict(ws=P + 8)),
    (scan_back, dict(dtype=2)), (scan_back, dict(kind=5)), (scan_back, dict(off=None)), (scan_back, dict(dy=None)), (scan_back, dict(x=None)), (scan_back, dict(g=None)),
    (scan_back, dict(y=None)), (scan_back, dict(dx=None)), (scan_back, dict(dg=None)), (scan_back, dict(dx=6 * P)), (scan_back, dict(dx=4 * P)), (scan_back, dict(dg=4 * P)),
    (scan_back, dict(dx=P, ld_dx=24)), (scan_back, dict(dh0=P)), (scan_back, dict(dh0=9 * P)), (scan_back, dict(dh0=P + 2)), (scan_back, dict(dlast=P + 2)), (scan_back, dict(ws=None)),
    (step, dict(dtype=2)), (step, dict(kind=2)), (step, dict(D=0)), (step, dict(x=None)), (step, dict(h=None)), (step, dict(out=None)), (step, dict(y=None)), (step, dict(h=P + 2)),
    (step, dict(y=P, ld_y=24)), (step, dict(ld_g=1)),
]


@pytest.mark.parametrize("call,kw", CASES, ids=lambda v: v.__name__ if callable(v) else "-".join(v))
def test_bad_arguments(B, call, kw):  # noqa: F811
    assert call(B, **kw) == B.EINVAL
    assert B.lib.abs_last_error(None) != b""


def test_sizes_beyond_the_limits_and_short_workspaces(B):  # noqa: F811
    big = 1 << 31
    assert embed(B, T=big) == B.ELIMIT and embed(B, V=big) == B.ELIMIT and embed(B, D=1 << 24, ld_table=big, ld_y=big) == B.ELIMIT
    assert embed_back(B, T=big) == B.ELIMIT and embed_back(B, V=big) == B.ELIMIT and embed_back(B, D=1 << 24, ld_dy=big, ld_out=big) == B.ELIMIT
    assert norm(B, D=32769, ld_x=big, ld_n=big) == B.ELIMIT
    assert norm_back(B, D=32769, ld_dn=big, ld_x=big, ld_skip=big, ld_dx=big) == B.ELIMIT
    assert linear(B, T=big) == B.ELIMIT and dgrad(B, T=big) == B.ELIMIT and wgrad(B, T=big) == B.ELIMIT and linear(B, K=big, ld_x=big) == B.ELIMIT
    assert scan(B, T=big) == B.ELIMIT and scan_back(B, seqs=big) == B.ELIMIT and step(B, S=big) == B.ELIMIT
    assert scan(B, T=(1 << 31) - 1024, D=1 << 14, ld_x=big, ld_g=big, ld_y=big) == B.ELIMIT          # tiles
    assert embed_back(B, n=B.lib.abs_embed_backward_workspace(4, 8, 16) - 1) == B.ENOMEM
    assert norm_back(B, n=B.lib.abs_layer_norm_workspace(4, 16) - 1) == B.ENOMEM
    assert scan(B, n=B.lib.abs_recurrence_workspace(400, 16) - 1) == B.ENOMEM and scan_back(B, n=0) == B.ENOMEM
    need = B.lib.abs_linear_workspace(4, 16, 24, P + 2, 16, 2 * P, 24)
    assert need > 0 and linear(B, x=P + 2, n=need - 1) == B.ENOMEM
    need = B.lib.abs_linear_wgrad_workspace(4, 16, 24, P, 16, 2 * P, 24)
    assert wgrad(B, n=need - 1) == B.ENOMEM
    need = B.lib.abs_linear_dgrad_workspace(4, 16, 24, P, 25, 2 * P, 24)
    assert need > 0 and dgrad(B, ld_dy=25, n=need - 1) == B.ENOMEM
    for call in (embed, norm, linear, dgrad, through):
        assert call(B, T=0) == B.OK
    assert scan(B, T=0, last=None) == B.OK and scan_back(B, T=0, dh0=None) == B.OK and step(B, S=0) == B.OK


def test_tensor_functions_refuse_what_is_no_cuda_tensor_and_unknown_names(B):  # noqa: F811
    from paper_2308_15164_b200 import llm

    z, i, f = torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32), torch.zeros(4)
    h = z.bfloat16()
    for call in (lambda: llm.embed(i, z), lambda: llm.embed_backward(z, i, 5), lambda: llm.layer_norm(z, f), lambda: llm.layer_norm_backward(z, z, f), lambda: llm.linear(h, h.t()),
                 lambda: llm.linear_dgrad(h, h), lambda: llm.linear_wgrad(h, h), lambda: llm.activation_backward(z, h, "relu"), lambda: llm.gated_recurrence(z, z),
                 lambda: llm.gated_recurrence_backward(z, z, z, z), lambda: llm.gated_recurrence_step(z, z, z), lambda: llm.embed(i, z, dtype=torch.float16),
                 lambda: llm.linear(h, h, dtype=torch.float64)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: llm.linear(h, h, act="tanh"), lambda: llm.linear_dgrad(h, h, act=None), lambda: llm.activation_backward(z, h, ["relu"]),
                 lambda: llm.gated_recurrence(z, z, kind="mix"), lambda: llm.gated_recurrence_step(z, z, z, kind=0)):
        with pytest.raises(ValueError):
            call()


# ---- the definitions themselves -------------------------------------------------------------------------------------
def leaf(*s, seed):
    return torch.randn(*s, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).requires_grad_()


def test_definition_of_the_embedding_against_autograd():
    table, ids, dy = leaf(6, 3, seed=1), torch.tensor([5, 0, -1, 5, 6, 2], dtype=torch.int32), leaf(6, 3, seed=2).detach()
    y = torch.stack([table[i] * 1.5 if 0 <= i < 6 else torch.zeros(3, dtype=torch.float64) for i in ids.tolist()])
    assert torch.equal(R.embed(ids, table, 1.5), y.detach())
    (y * dy).sum().backward()
    assert torch.allclose(R.embed_backward(dy, ids, 6, 1.5)[0], table.grad, rtol=1e-13)


@pytest.mark.parametrize("skip", [True, False])
def test_definition_of_the_layer_norm_against_autograd(skip):
    x, w, b = leaf(4, 9, seed=1), leaf(9, seed=2), leaf(9, seed=3)
    dn, sk = leaf(4, 9, seed=4).detach(), leaf(4, 9, seed=5).detach()
    n = torch.nn.functional.layer_norm(x, (9,), w, b, 1e-5)
    assert torch.allclose(R.layer_norm(x, w, b, 1e-5)[0], n.detach(), rtol=1e-12)
    ((n * dn).sum() + ((x * sk).sum() if skip else 0.0)).backward()
    out, _ = R.layer_norm_backward(dn, x, w, sk if skip else None, 1e-5)
    for k, t in (("dx", x), ("dw", w), ("db", b)):
        assert torch.allclose(out[k], t.grad, rtol=1e-9, atol=1e-12), k


@pytest.mark.parametrize("name", ["none", "relu", "gelu", "silu"])
def test_definitions_of_the_activations_against_autograd(name):
    z = leaf(200, seed=1)
    F = torch.nn.functional
    y = {"none": lambda v: v, "relu": F.relu, "gelu": F.gelu, "silu": F.silu}[name](z)
    assert torch.allclose(R.act(name, z.detach()), y.detach(), rtol=1e-11, atol=1e-15)
    (g,) = torch.autograd.grad(y.sum(), z)
    assert torch.allclose(R.slope(name, z.detach()), g, rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("kind", ["blend", "add"])
@pytest.mark.parametrize("cuts", [(0, 7), (1, 3, 3, 6), (0, 1, 7, 7)])
def test_definition_of_the_recurrence_against_autograd(kind, cuts):
    T, W, S = 7, 3, len(cuts) - 1
    x, g, h0 = leaf(T, W, seed=1), leaf(T, W, seed=2), leaf(S, W, seed=3)
    dy, dl = leaf(T, W, seed=4).detach(), leaf(S, W, seed=5).detach()
    rows, last = [torch.zeros(W, dtype=torch.float64)] * T, []
    for q in range(S):
        h = h0[q]
        for t in range(cuts[q], cuts[q + 1]):
            a = torch.sigmoid(g[t])
            h = a * h + ((1 - a) * x[t] if kind == "blend" else x[t])
            rows[t] = h
        last.append(h)
    y, last, off = torch.stack(rows), torch.stack(last), torch.tensor(cuts, dtype=torch.int32)
    wy, _, wl, _ = R.recurrence(x, g, off, h0, kind)
    assert torch.allclose(wy, y.detach(), rtol=1e-12) and torch.allclose(wl, last.detach(), rtol=1e-12)
    ((y * dy).sum() + (last * dl).sum()).backward()
    out, _ = R.recurrence_backward(dy, x, g, y, off, h0, dl, kind)
    for k, t in (("dx", x), ("dg", g), ("dh0", h0)):
        assert torch.allclose(out[k], t.grad, rtol=1e-9, atol=1e-12), k
