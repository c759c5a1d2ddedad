"""What the functions on tensors check, return and keep: refusals by type, shape, stride and device, outputs that are given, the
library's status as an exception, no reference and no memory left behind."""

import gc
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2308_15164_b200 import build

    build.build()
    from paper_2308_15164_b200 import llm

    return llm


def f32(*s):
    return torch.zeros(*s, device="cuda")


def b16(*s):
    return torch.zeros(*s, device="cuda", dtype=torch.bfloat16)


def i32(*s):
    return torch.zeros(*s, device="cuda", dtype=torch.int32)


def policy(L, **kw):
    return L.policy_loss(**(dict(logits=f32(3, 5), labels=i32(3), logp_old=f32(3), advantage=f32(3), weight=f32(3)) | kw))


def preference(L, **kw):
    return L.preference_loss(**(dict(logits=f32(4, 5), labels=i32(4), offsets=torch.tensor([0, 1, 4], dtype=torch.int32, device="cuda"), logp_ref=f32(2)) | kw))


def forward(L, **kw):
    return L.residual_norm(**(dict(x=b16(3, 8), h=b16(3, 8), w_pre=f32(8)) | kw))


def backward(L, **kw):
    return L.residual_norm_backward(**(dict(dn=b16(3, 8), dy=b16(3, 8), y=b16(3, 8), h=b16(3, 8), w_pre=f32(8)) | kw))


def pack(L, **kw):
    return L.ckpt8_quantize(**(dict(x=b16(3, 40)) | kw))


def unpack(L, **kw):
    c = L.Ckpt8(torch.zeros(3, 64, dtype=torch.int8, device="cuda"), torch.zeros(3, 2, dtype=torch.uint8, device="cuda"), 40)
    return L.ckpt8_dequantize(c._replace(**{k: v for k, v in kw.items() if k in "qe" or k == "width"}), **{k: v for k, v in kw.items() if k in ("dtype", "out")})


def wgrad(L, **kw):
    c = L.Ckpt8(torch.zeros(3, 64, dtype=torch.int8, device="cuda"), torch.zeros(3, 2, dtype=torch.uint8, device="cuda"), 40)
    return L.ckpt8_wgrad(c._replace(**{k: v for k, v in kw.items() if k in "qe" or k == "width"}),
                         **(dict(dy=b16(3, 6)) | {k: v for k, v in kw.items() if k in ("dy", "out", "accumulate")}))


REFUSED = [
    (policy, TypeError, dict(logits=None)), (policy, TypeError, dict(logits=lambda: f32(3))), (policy, TypeError, dict(logits=lambda: f32(3, 5).half())),
    (policy, TypeError, dict(logits=lambda: torch.zeros(3, 5))), (policy, TypeError, dict(labels=lambda: i32(3).long())), (policy, ValueError, dict(labels=lambda: i32(4))),
    (policy, ValueError, dict(weight=lambda: f32(6)[::2])), (policy, TypeError, dict(weight=lambda: b16(3))), (policy, TypeError, dict(advantage=1.0)),
    (policy, TypeError, dict(logp_old=None)), (policy, ValueError, dict(logp_ref=lambda: f32(3, 1))), (policy, TypeError, dict(clip_low="a")),
    (policy, ValueError, dict(logits=lambda: f32(5, 3).t())), (policy, ValueError, dict(logits=lambda: f32(5).expand(3, 5))),
    (policy, ValueError, dict(dlogits=lambda: f32(3, 5), need_grad=False)), (policy, ValueError, dict(dlogits=lambda: f32(3, 6))),
    (policy, TypeError, dict(dlogits=lambda: b16(3, 5))), (policy, ValueError, dict(dlogits=lambda: f32(5, 3).t())),
    (policy, TypeError, dict(weight=lambda: torch._neg_view(f32(3)))), (policy, TypeError, dict(logits=lambda: f32(3, 5).to_sparse())),
    (preference, ValueError, dict(offsets=lambda: i32(4))), (preference, ValueError, dict(offsets=None)), (preference, TypeError, dict(offsets=lambda: i32(3).long())),
    (preference, ValueError, dict(logp_ref=lambda: f32(3))), (preference, TypeError, dict(scale="x")), (preference, ValueError, dict(labels=lambda: i32(5))),
    (forward, ValueError, dict(h=lambda: b16(3, 7))), (forward, TypeError, dict(h=lambda: f32(3, 8))), (forward, ValueError, dict(w_pre=lambda: f32(7))),
    (forward, TypeError, dict(w_post=lambda: b16(8))), (forward, ValueError, dict(gate=lambda: f32(7))), (forward, TypeError, dict(gate=lambda: f32(3, 8))),
    (forward, TypeError, dict(gate=2.0)), (forward, ValueError, dict(n=lambda: b16(2, 8))), (forward, TypeError, dict(y=1)),
    (backward, ValueError, dict(dw_post=lambda: f32(8))), (backward, ValueError, dict(dgate=lambda: f32(8))), (backward, TypeError, dict(dn=None)),
    (backward, ValueError, dict(dw_pre=lambda: f32(9))), (backward, ValueError, dict(gate=lambda: f32(8), dgate=lambda: f32(16)[::2])),
    (backward, ValueError, dict(gate=lambda: b16(3, 8), dgate=lambda: b16(8, 3).t())), (backward, TypeError, dict(dh=lambda: f32(3, 8))),
    (pack, TypeError, dict(x=lambda: f32(3, 40).double())), (pack, ValueError, dict(x=lambda: b16(40, 3).t())), (pack, TypeError, dict(x=lambda: b16(3))),
    (unpack, TypeError, dict(q=lambda: torch.zeros(3, 64, dtype=torch.uint8, device="cuda"))), (unpack, ValueError, dict(width=30)), (unpack, ValueError, dict(width=65)),
    (unpack, ValueError, dict(width=-1)), (unpack, ValueError, dict(e=lambda: torch.zeros(3, 3, dtype=torch.uint8, device="cuda"))), (unpack, TypeError, dict(width="a")),
    (unpack, TypeError, dict(dtype=torch.float16)), (unpack, ValueError, dict(out=lambda: b16(3, 41))), (unpack, TypeError, dict(out=lambda: f32(3, 40))),
    (unpack, TypeError, dict(q=lambda: torch.zeros(3, 64, dtype=torch.int8))),
    (wgrad, TypeError, dict(dy=lambda: f32(3, 6))), (wgrad, ValueError, dict(dy=lambda: b16(4, 6))), (wgrad, ValueError, dict(accumulate=True)),
    (wgrad, ValueError, dict(out=lambda: f32(41, 6))), (wgrad, TypeError, dict(out=lambda: b16(40, 6))), (wgrad, TypeError, dict(dy=lambda: b16(3))),
]


@pytest.mark.parametrize("call,kind,kw", REFUSED, ids=lambda v: v.__name__ if callable(v) else "-".join(v) if isinstance(v, dict) else "")
def test_refused(L, call, kind, kw):
    made = {k: v() if callable(v) else v for k, v in kw.items()}
    with pytest.raises(kind):
        call(L, **made)
    call(L)                       # and the next call is served


def test_a_status_is_an_exception(L):
    from paper_2308_15164_b200 import binding

    for call, kw in ((policy, dict(clip_low=-1.0)), (preference, dict(smoothing=2.0)), (forward, dict(eps=0.0)), (backward, dict(scale=float("inf")))):
        with pytest.raises(binding.AbsError) as e:
            call(L, **kw)
        assert e.value.code == binding.EINVAL and "status -1" in str(e.value)
    with pytest.raises(TypeError):
        L._t.policy_loss(1, 2)


def test_given_outputs_are_the_ones_returned(L):
    z = f32(3, 5)
    r = policy(L, logits=z, dlogits=z)
    assert r.dlogits is z and r.loss.shape == r.kl.shape == r.clipped.shape == () and r.logp.shape == (3,)
    assert policy(L, need_grad=False).dlogits is None and preference(L, need_grad=False).dlogits is None
    wide = f32(3, 9)
    assert policy(L, logits=wide[:, :5]).dlogits.shape == (3, 5) and policy(L, logits=wide[:, :5]).dlogits.is_contiguous()
    x, h = b16(3, 8), b16(3, 8)
    y, n = forward(L, x=x, h=h, y=x, n=h)
    assert y is x and n is h
    w, g = f32(8), f32(8)
    r = backward(L, gate=g, dw_pre=w)
    assert r.dw_pre is w and r.dw_post is None and r.dgate.shape == (8,) and backward(L).dgate is None
    out = f32(40, 6)
    assert wgrad(L, out=out) is out
    p = torch.nn.Parameter(f32(8))
    forward(L, w_pre=p)
    assert isinstance(policy(L, clip_low=1, kl_coef=torch.tensor(0.0)), L.PolicyLoss)


def test_scalars_outlive_what_they_came_with(L):
    torch.manual_seed(0)
    z = torch.randn(7, 100, device="cuda")
    a = dict(logits=z, labels=i32(7), advantage=f32(7) + 1, weight=f32(7) + 0.5, logp_old=f32(7) - 5)
    want = [float(v) for v in policy(L, **a)[:3]]
    kept = [policy(L, **a)[i] for i in range(3)]
    for _ in range(20):
        torch.full((3,), 7.0, device="cuda")
    assert [float(v) for v in kept] == want and want[0] != 0
    total = kept[0] + kept[1] * 2            # they take part in arithmetic as any tensor does
    assert float(total) == pytest.approx(want[0] + 2 * want[1])


def test_nothing_is_left_behind(L):
    z, y, v = f32(3, 5), i32(3), f32(3)
    bad = b16(3)
    calls = [lambda: policy(L, logits=z, labels=y, weight=v), lambda: preference(L), lambda: forward(L), lambda: backward(L, accumulate=True),
             lambda: unpack(L), lambda: wgrad(L), lambda: pack(L)]
    for c in calls:
        c()
    gc.collect()
    torch.cuda.synchronize()
    held, refs, none = torch.cuda.memory_allocated(), [sys.getrefcount(t) for t in (z, y, v, bad)], sys.getrefcount(None)
    for _ in range(200):
        for c in calls:
            c()
        for kw in (dict(weight=bad), dict(clip_low=-1.0), dict(kl_coef="x")):
            with pytest.raises(Exception):
                policy(L, logits=z, labels=y, **kw)
    gc.collect()
    assert torch.cuda.memory_allocated() == held
    assert [sys.getrefcount(t) for t in (z, y, v, bad)] == refs
    assert abs(sys.getrefcount(None) - none) < 150


def test_a_call_uses_the_current_stream(L):
    torch.manual_seed(1)
    z = torch.randn(64, 5000, device="cuda")
    a = dict(labels=i32(64), advantage=f32(64) + 1, weight=f32(64) + 0.5, logp_old=f32(64))
    want = policy(L, logits=z, **a).dlogits
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        later = torch.zeros_like(z)
        torch.cuda._sleep(2_000_000)         # the copy below has not run when the call is made
        later.copy_(z)
        got = policy(L, logits=later, **a).dlogits
    s.synchronize()
    assert torch.equal(got, want)
