"""The language-model operators refuse bad arguments before they touch a GPU (these run without one: every call here must
return from its checks), and the 64-bit definitions that the GPU tests compare with hold against differences and autograd."""

import ctypes

import pytest
import torch

from tests import llm_reference as R


@pytest.fixture(scope="module")
def B():
    from paper_2308_15164_b200 import build

    build.build()
    from paper_2308_15164_b200 import binding

    return binding


P = 1 << 20          # an address that is never dereferenced
WS = 1 << 30


def policy(B, **kw):
    a = dict(logits=P, dtype=0, T=4, V=8, ld=8, labels=P, old=P, ref=P, adv=P, weight=P, lo=0.2, hi=0.2, kl=0.1, stats=P, logp=P, d=2 * P, ld_d=8, ws=P, n=WS) | kw
    return B.lib.abs_policy_loss(*a.values(), None)


def preference(B, **kw):
    a = dict(logits=P, dtype=0, T=4, V=8, ld=8, labels=P, off=P, pairs=1, ref=P, beta=0.1, smoothing=0.0, scale=1.0, stats=P, pair=P, seq=P, d=2 * P, ld_d=8,
             ws=P, n=WS) | kw
    return B.lib.abs_preference_loss(*a.values(), None)


def forward(B, **kw):
    a = dict(x=P, ld_x=16, h=P, ld_h=16, gate=P, ld_gate=16, kind=2, w_post=P, w_pre=P, scale=1.0, eps=1e-6, dtype=1, T=4, D=16, y=P, ld_y=16, n=P, ld_n=16) | kw
    return B.lib.abs_residual_norm(*a.values(), None)


def backward(B, **kw):
    a = dict(dn=P, ld_dn=16, dy=P, ld_dy=16, y=P, ld_y=16, h=P, ld_h=16, gate=P, ld_gate=16, kind=2, w_post=P, w_pre=P, scale=1.0, eps=1e-6, dtype=1, T=4, D=16,
             dx=P, ld_dx=16, dh=P, ld_dh=16, dgate=P, ld_dgate=16, dw_pre=P, dw_post=P, acc=0, ws=P, n=WS) | kw
    return B.lib.abs_residual_norm_backward(*a.values(), None)


def wgrad(B, **kw):
    a = dict(q=P, e=P, dy=P, ld=64, T=4, D=32, N=64, dw=P, ld_dw=64, acc=0, ws=P, n=WS) | kw
    return B.lib.abs_ckpt8_wgrad(*a.values(), None)


NAN, INF = float("nan"), float("inf")
CASES = [
    (policy, dict(dtype=2)), (policy, dict(V=0)), (policy, dict(ld=7)), (policy, dict(ld_d=7)), (policy, dict(logits=None)), (policy, dict(labels=None)),
    (policy, dict(logits=P + 2)), (policy, dict(dtype=1, logits=P + 1)), (policy, dict(labels=P + 2)), (policy, dict(old=None)), (policy, dict(adv=None)),
    (policy, dict(weight=None)), (policy, dict(logp=None)), (policy, dict(stats=None)), (policy, dict(stats=P + 1)), (policy, dict(lo=-0.1)), (policy, dict(hi=NAN)),
    (policy, dict(kl=INF)), (policy, dict(ref=None)), (policy, dict(ws=None)), (policy, dict(ws=P + 8)), (policy, dict(d=P, ld=9)),
    (preference, dict(dtype=9)), (preference, dict(ld=3)), (preference, dict(off=None)), (preference, dict(ref=None)), (preference, dict(pair=None)),
    (preference, dict(seq=None)), (preference, dict(stats=None)), (preference, dict(beta=NAN)), (preference, dict(scale=INF)), (preference, dict(smoothing=1.5)),
    (preference, dict(smoothing=NAN)), (preference, dict(ws=None)), (preference, dict(off=P + 2)),
    (forward, dict(dtype=3)), (forward, dict(D=0)), (forward, dict(kind=3)), (forward, dict(gate=None)), (forward, dict(kind=0)), (forward, dict(w_pre=None)),
    (forward, dict(eps=0.0)), (forward, dict(eps=NAN)), (forward, dict(scale=INF)), (forward, dict(ld_x=15)), (forward, dict(ld_gate=15)), (forward, dict(ld_n=1)),
    (forward, dict(x=None)), (forward, dict(y=None)), (forward, dict(h=P + 1)), (forward, dict(w_post=P + 2)), (forward, dict(kind=1, gate=P + 2)),
    (forward, dict(y=P, ld_y=24)), (forward, dict(n=P, ld_n=32)), (backward, dict(dx=P, ld_dx=24)), (backward, dict(dgate=P, ld_dgate=24)),
    (backward, dict(dn=None)), (backward, dict(dw_post=None)), (backward, dict(w_post=None)), (backward, dict(dgate=None)), (backward, dict(gate=None)),
    (backward, dict(dw_pre=None)), (backward, dict(dw_pre=P + 2)), (backward, dict(ws=None)), (backward, dict(ws=P + 16)), (backward, dict(ld_dh=8)),
    (backward, dict(kind=1, dgate=P + 2)), (backward, dict(dx=P + 1)),
    (wgrad, dict(D=0)), (wgrad, dict(N=0)), (wgrad, dict(ld=63)), (wgrad, dict(ld_dw=63)), (wgrad, dict(dw=None)), (wgrad, dict(dw=P + 2)), (wgrad, dict(q=None)),
    (wgrad, dict(q=P + 8)), (wgrad, dict(e=None)), (wgrad, dict(dy=P + 1)), (wgrad, dict(T=1 << 14, ws=None)), (wgrad, dict(T=1 << 14, ws=P + 8)),
]


@pytest.mark.parametrize("call,kw", CASES, ids=lambda v: v.__name__ if callable(v) else "-".join(v))
def test_bad_arguments(B, call, kw):
    assert call(B, **kw) == B.EINVAL
    assert B.lib.abs_last_error(None) != b""


def test_sizes_beyond_the_limits_and_short_workspaces(B):
    assert policy(B, V=1 << 31, ld=1 << 31, ld_d=1 << 31) == B.ELIMIT
    assert preference(B, T=1 << 31) == B.ELIMIT
    wide = {k: 1 << 20 for k in ("ld_x", "ld_h", "ld_gate", "ld_y", "ld_n")}
    assert forward(B, D=32769, **wide) == B.ELIMIT
    wide = {k: 1 << 20 for k in ("ld_dn", "ld_dy", "ld_y", "ld_h", "ld_gate", "ld_dx", "ld_dh", "ld_dgate")}
    assert backward(B, D=32769, **wide) == B.ELIMIT
    assert wgrad(B, T=1 << 31) == B.ELIMIT
    assert policy(B, n=B.lib.abs_policy_loss_workspace() - 1) == B.ENOMEM
    assert preference(B, n=B.lib.abs_preference_loss_workspace(4) - 1) == B.ENOMEM
    assert backward(B, n=B.lib.abs_residual_norm_workspace(4, 16) - 1) == B.ENOMEM
    need = B.lib.abs_ckpt8_wgrad_workspace(1 << 14, 32, 64, P, 64)
    assert need > 0 and wgrad(B, T=1 << 14, n=need - 1) == B.ENOMEM
    for fn in (B.lib.abs_ckpt8_quantize,):
        assert fn(P, 32, 2, 4, 32, P, P, None) == B.EINVAL and fn(P, 31, 0, 4, 32, P, P, None) == B.EINVAL and fn(P, 32, 0, 4, 0, P, P, None) == B.EINVAL
        assert fn(P, 32, 0, 4, 32, P + 8, P, None) == B.EINVAL and fn(None, 32, 0, 4, 32, P, P, None) == B.EINVAL
        assert fn(P, 32, 0, 0, 32, P, P, None) == B.OK
    assert B.lib.abs_ckpt8_dequantize(P, P, 4, 32, P, 31, 0, None) == B.EINVAL
    assert B.lib.abs_ckpt8_dequantize(P, None, 4, 32, P, 32, 0, None) == B.EINVAL
    assert forward(B, T=0) == B.OK


def test_tensor_functions_refuse_what_is_no_cuda_tensor(B):
    from paper_2308_15164_b200 import llm

    z, y, f = torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    with pytest.raises(TypeError):
        llm.policy_loss(z, y, f, f, f)
    with pytest.raises(TypeError):
        llm.preference_loss(z, y, y, f)
    with pytest.raises(TypeError):
        llm.residual_norm(z, z, f)
    with pytest.raises(TypeError):
        llm.ckpt8_quantize(z)
    with pytest.raises(TypeError):
        llm.ckpt8_wgrad(llm.Ckpt8(torch.zeros(3, 32, dtype=torch.int8), torch.zeros(3, 1, dtype=torch.uint8), 4), z)


# ---- the definitions themselves -------------------------------------------------------------------------------------
def gen(*s, seed=0):
    return torch.randn(*s, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def test_definition_of_the_policy_loss_against_autograd():
    T, V = 9, 13
    z, y = gen(T, V).requires_grad_(), torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    lp = R.rows_logp(z, y)[0]
    old, ref, adv, w = (lp.detach() + 0.4 * gen(T, seed=2)), lp.detach() + gen(T, seed=3), gen(T, seed=4), torch.rand(T, dtype=torch.float64)
    out = R.policy(z, y, old, adv, w, ref, kl_coef=0.3)
    logp = torch.log_softmax(z, 1)[torch.arange(T), y.long()]
    r = (logp - old).exp()
    lo, hi = 1 - float(torch.tensor(0.2)), 1 + float(torch.tensor(0.2))
    x = ref - logp
    loss = (w * (-torch.minimum(r * adv, r.clamp(lo, hi) * adv) + 0.3 * (x.exp() - x - 1))).sum()
    loss.backward()
    assert torch.allclose(out["loss"], loss.detach(), rtol=1e-12) and torch.allclose(out["dlogits"], z.grad, rtol=1e-10, atol=1e-14)


def test_definition_of_the_preference_loss_against_autograd():
    V, lens = 11, (3, 2, 0, 4)
    T = sum(lens)
    z, y = gen(T, V).requires_grad_(), torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    y[1] = -100
    off = torch.tensor([0, 3, 5, 5, 9], dtype=torch.int32)
    ref = gen(4, seed=5)
    out = R.preference(z, y, off, ref, beta=0.25, smoothing=0.125, scale=0.5)
    logp = torch.log_softmax(z, 1)[torch.arange(T), y.long().clamp(min=0)] * (y >= 0)
    s = torch.stack([p.sum() for p in logp.split(lens)]) - ref
    h = 0.25 * (s[0::2] - s[1::2])
    loss = 0.5 * (-(1 - 0.125) * torch.nn.functional.logsigmoid(h) - 0.125 * torch.nn.functional.logsigmoid(-h)).sum()
    loss.backward()
    assert torch.allclose(out["loss"], loss.detach(), rtol=1e-12) and torch.allclose(out["dlogits"], z.grad, rtol=1e-10, atol=1e-14)


@pytest.mark.parametrize("gate", ["none", "channel", "element"])
@pytest.mark.parametrize("post", [False, True])
def test_definition_of_the_residual_gradients_against_autograd(gate, post):
    T, D = 4, 10
    leaf = lambda *s, seed: gen(*s, seed=seed).requires_grad_()  # noqa: E731
    x, h, w_pre = leaf(T, D, seed=1), leaf(T, D, seed=2), leaf(D, seed=3)
    w_post = leaf(D, seed=4) if post else None
    g = {"none": None, "channel": leaf(D, seed=5), "element": leaf(T, D, seed=6)}[gate]
    dn, dy = gen(T, D, seed=7), gen(T, D, seed=8)
    rms = lambda v: (v.square().mean(1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
    u = h / rms(h) * w_post if post else h
    y = 0.6 * x + (u if g is None else (g if gate == "channel" else torch.sigmoid(g)) * u)
    n = y / rms(y) * w_pre
    wy, wn, *_ = R.residual(x, h, w_pre, w_post, g, scale=0.6)
    assert torch.allclose(wy, y.detach(), rtol=1e-12) and torch.allclose(wn, n.detach(), rtol=1e-12)
    ((n * dn).sum() + (y * dy).sum()).backward()
    out, _ = R.residual_backward(dn, dy, y, h, w_pre, w_post, g, scale=0.6)
    for k, t in (("dx", x), ("dh", h), ("dw_pre", w_pre), ("dw_post", w_post), ("dgate", g)):
        assert (t is None) == (k not in out)
        if t is not None:
            assert torch.allclose(out[k], t.grad, rtol=1e-9, atol=1e-12), k


def test_definition_of_the_8_bit_format():
    x = torch.tensor([[127.0, 0.5, -2.5, 1.5] + [0.0] * 28 + [127.5] + [0.0] * 3], dtype=torch.float64)
    q, e = R.pack(x)
    assert e.tolist() == [[127, 128]] and q[0, :4].tolist() == [127, 0, -2, 2] and q[0, 32] == 64 and q.shape == (1, 64)
    v = gen(50, 70) * torch.exp2(torch.randint(-60, 60, (50, 1), generator=torch.Generator().manual_seed(1)).double())
    q, e = R.pack(v)
    step = torch.exp2(e.double() - 127).repeat_interleave(32, 1)[:, :70]
    assert q.abs().max() <= 127 and ((R.unpack(q, e, 70) - v).abs() <= step / 2).all()
    top = torch.nn.functional.pad(v, (0, 26)).view(50, 3, 32).abs().amax(2)
    assert (top > 127 * torch.exp2(e.double() - 128)).all()           # no smaller power would do
