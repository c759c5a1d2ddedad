"""What the functions of embedding, layer norm, linear layer and recurrence check, return and keep: refusals by type, shape, stride and
device, outputs that are given, the library's status as an exception, another stream than the default one."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2308_15164_b200 import llm

    return llm


def f32(*s):
    return torch.ones(*s, device="cuda")


def b16(*s):
    return torch.ones(*s, device="cuda", dtype=torch.bfloat16)


def i32(*s):
    return torch.zeros(*s, device="cuda", dtype=torch.int32)


def offs(*v):
    return torch.tensor(v, device="cuda", dtype=torch.int32)


def embed(L, **kw):
    return L.embed(**(dict(ids=i32(3), table=f32(5, 8)) | kw))


def embed_back(L, **kw):
    return L.embed_backward(**(dict(dy=b16(3, 8), ids=i32(3), vocab=5) | kw))


def norm(L, **kw):
    return L.layer_norm(**(dict(x=b16(3, 8), w=f32(8)) | kw))


def norm_back(L, **kw):
    return L.layer_norm_backward(**(dict(dn=b16(3, 8), x=b16(3, 8), w=f32(8)) | kw))


def linear(L, **kw):
    return L.linear(**(dict(x=b16(3, 8), w=b16(8, 6)) | kw))


def dgrad(L, **kw):
    return L.linear_dgrad(**(dict(dy=b16(3, 6), w=b16(8, 6)) | kw))


def wgrad(L, **kw):
    return L.linear_wgrad(**(dict(x=b16(3, 8), dy=b16(3, 6)) | kw))


def through(L, **kw):
    return L.activation_backward(**(dict(dy=f32(3, 8), z=b16(3, 8), act="silu") | kw))


def scan(L, **kw):
    return L.gated_recurrence(**(dict(x=b16(4, 8), g=b16(4, 8), offsets=offs(0, 1, 4)) | kw))


def scan_back(L, **kw):
    return L.gated_recurrence_backward(**(dict(dy=b16(4, 8), x=b16(4, 8), g=b16(4, 8), y=b16(4, 8), offsets=offs(0, 1, 4)) | kw))


def step(L, **kw):
    return L.gated_recurrence_step(**(dict(x=b16(4, 8), g=b16(4, 8), h=f32(4, 8)) | kw))


REFUSED = [
    (embed, TypeError, dict(ids=lambda: i32(3).long())), (embed, TypeError, dict(ids=lambda: i32(3, 1))), (embed, ValueError, dict(ids=lambda: i32(6)[::2])),
    (embed, TypeError, dict(table=lambda: b16(5, 8))), (embed, TypeError, dict(table=lambda: f32(8))), (embed, ValueError, dict(table=lambda: f32(8, 5).t())),
    (embed, TypeError, dict(scale="a")), (embed, ValueError, dict(y=lambda: b16(3, 7))), (embed, TypeError, dict(y=lambda: f32(3, 8))),
    (embed, TypeError, dict(ids=lambda: torch.zeros(3, dtype=torch.int32))),
    (embed_back, TypeError, dict(dy=lambda: b16(3, 8).half())), (embed_back, ValueError, dict(ids=lambda: i32(4))), (embed_back, ValueError, dict(vocab=0)),
    (embed_back, TypeError, dict(vocab="a")), (embed_back, ValueError, dict(out=lambda: f32(4, 8))), (embed_back, TypeError, dict(out=lambda: b16(5, 8))),
    (embed_back, ValueError, dict(accumulate=True)),
    (norm, TypeError, dict(x=lambda: f32(3, 8).double())), (norm, ValueError, dict(w=lambda: f32(7))), (norm, TypeError, dict(w=lambda: b16(8))),
    (norm, ValueError, dict(b=lambda: f32(9))), (norm, ValueError, dict(n=lambda: b16(2, 8))), (norm, ValueError, dict(x=lambda: b16(8, 3).t())),
    (norm_back, ValueError, dict(dn=lambda: b16(3, 7))), (norm_back, TypeError, dict(dskip=lambda: f32(3, 8))), (norm_back, ValueError, dict(db=lambda: f32(8), bias=False)),
    (norm_back, ValueError, dict(dw=lambda: f32(16)[::2])), (norm_back, TypeError, dict(dx=lambda: f32(3, 8))),
    (linear, TypeError, dict(x=lambda: f32(3, 8))), (linear, TypeError, dict(w=lambda: f32(8, 6))), (linear, ValueError, dict(w=lambda: b16(7, 6))),
    (linear, ValueError, dict(b=lambda: f32(5))), (linear, ValueError, dict(act="tanh")), (linear, ValueError, dict(residual=lambda: b16(3, 5))),
    (linear, TypeError, dict(residual=lambda: f32(3, 6))), (linear, ValueError, dict(z=lambda: b16(3, 6))), (linear, TypeError, dict(dtype=torch.float16)),
    (linear, ValueError, dict(w=lambda: b16(6, 8).t())),
    (dgrad, ValueError, dict(w=lambda: b16(8, 5))), (dgrad, ValueError, dict(act="gelu")), (dgrad, ValueError, dict(z=lambda: b16(3, 8))),
    (dgrad, ValueError, dict(act="relu", z=lambda: b16(3, 7))), (dgrad, TypeError, dict(act="relu", z=lambda: f32(3, 8))), (dgrad, TypeError, dict(dx=lambda: f32(3, 8))),
    (wgrad, ValueError, dict(dy=lambda: b16(4, 6))), (wgrad, TypeError, dict(dy=lambda: f32(3, 6))), (wgrad, ValueError, dict(accumulate=True)),
    (wgrad, ValueError, dict(accumulate=True, bias=True, dw=lambda: f32(8, 6))), (wgrad, ValueError, dict(db=lambda: f32(6))), (wgrad, ValueError, dict(dw=lambda: f32(8, 7))),
    (through, TypeError, dict(z=lambda: f32(3, 8))), (through, ValueError, dict(act="")), (through, ValueError, dict(dz=lambda: b16(3, 9))),
    (scan, ValueError, dict(g=lambda: b16(4, 7))), (scan, TypeError, dict(g=lambda: f32(4, 8))), (scan, TypeError, dict(offsets=lambda: offs(0, 4).long())),
    (scan, ValueError, dict(offsets=lambda: i32(0))), (scan, ValueError, dict(h0=lambda: f32(3, 8))), (scan, TypeError, dict(h0=lambda: b16(2, 8))),
    (scan, ValueError, dict(kind="sum")), (scan, ValueError, dict(last=lambda: f32(2, 16)[:, ::2])), (scan, ValueError, dict(h0=lambda: f32(8, 2).t())),
    (scan_back, ValueError, dict(y=lambda: b16(3, 8))), (scan_back, ValueError, dict(dlast=lambda: f32(1, 8))), (scan_back, TypeError, dict(dx=lambda: f32(4, 8))),
    (step, ValueError, dict(h=lambda: f32(3, 8))), (step, TypeError, dict(h=lambda: b16(4, 8))), (step, ValueError, dict(out=lambda: f32(4, 7))),
]


@pytest.mark.parametrize("call,kind,kw", REFUSED, ids=lambda v: v.__name__ if callable(v) else "-".join(v) if isinstance(v, dict) else "")
def test_refused(L, call, kind, kw):
    made = {k: v() if callable(v) else v for k, v in kw.items()}
    with pytest.raises(kind):
        call(L, **made)
    call(L)                       # and the next call is served


def test_a_status_is_an_exception(L):
    from paper_2308_15164_b200 import binding

    h0, w = f32(2, 8), b16(8, 8)
    for call, kw in ((embed, dict(scale=float("inf"))), (embed_back, dict(scale=float("nan"))), (norm, dict(eps=0.0)), (norm_back, dict(eps=-1.0)), (linear, dict(w=w, y=w[:3])),
                     (scan, dict(h0=h0, last=h0)), (scan_back, dict(dlast=h0, dh0=h0))):
        with pytest.raises(binding.AbsError) as e:
            call(L, **kw)
        assert e.value.code == binding.EINVAL


def calls():
    back = dict(h0=f32(2, 8))
    return [
        (embed, dict(y=lambda: b16(3, 8))), (embed_back, dict(out=lambda: f32(5, 8))), (norm, dict(n=lambda: b16(3, 8))),
        (norm_back, dict(dx=lambda: b16(3, 8), dw=lambda: f32(8), db=lambda: f32(8))),
        (lambda L, **o: linear(L, keep=True, **o), dict(y=lambda: b16(3, 6), z=lambda: b16(3, 6))), (dgrad, dict(dx=lambda: b16(3, 8))),
        (lambda L, **o: wgrad(L, bias=True, **o), dict(dw=lambda: f32(8, 6), db=lambda: f32(6))), (through, dict(dz=lambda: b16(3, 8))),
        (scan, dict(y=lambda: b16(4, 8), last=lambda: f32(2, 8))),
        (lambda L, **o: scan_back(L, **back, **o), dict(dx=lambda: b16(4, 8), dg=lambda: b16(4, 8), dh0=lambda: f32(2, 8))), (step, dict(y=lambda: b16(4, 8), out=lambda: f32(4, 8))),
    ]


def test_given_outputs_are_used_and_count_as_modified(L):
    for call, makers in calls():
        outs = {k: m() for k, m in makers.items()}
        whole = {k: torch.stack((v, v)) for k, v in outs.items()}
        views = {k: v[1] for k, v in whole.items()}              # a view and its base have one counter
        before = {k: v._version for k, v in outs.items()}, {k: v._version for k, v in whole.items()}
        kept = {k: v[0].clone() for k, v in whole.items()}
        fresh = call(L)
        call(L, **outs)
        call(L, **views)
        fresh = fresh if isinstance(fresh, tuple) else (fresh,)
        for k, want in zip(outs, [t for t in fresh if t is not None]):
            assert outs[k]._version == before[0][k] + 1 and whole[k]._version == before[1][k] + 1
            assert torch.equal(outs[k], want) and torch.equal(views[k], want) and torch.equal(whole[k][0], kept[k])


def test_another_stream(L):
    """The calls go to the current stream: work that is enqueued there before them is seen."""
    side = torch.cuda.Stream()
    T, W = 4000, 512
    x = torch.zeros(T, W, device="cuda", dtype=torch.bfloat16)
    src = torch.randn(T, W, device="cuda").bfloat16()
    w, b = torch.randn(W, W, device="cuda").bfloat16(), torch.randn(W, device="cuda")
    ids = torch.randint(0, 300, (T,), device="cuda", dtype=torch.int32)
    torch.cuda.synchronize()

    def all_of(t):
        n = L.layer_norm(t, b, b)
        y = L.linear(n, w, b, act="gelu").y
        h = L.gated_recurrence(y, n)
        r = L.gated_recurrence_backward(t, y, n, h.y)
        return [n, y, h.y, h.last, r.dx, r.dg, *L.linear_wgrad(t, r.dx, bias=True), L.linear_dgrad(r.dg, w), L.embed_backward(r.dx, ids, 300), *L.layer_norm_backward(t, n, b)]

    want = all_of(src)
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        x.copy_(src)
        got = all_of(x)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    L.check()
