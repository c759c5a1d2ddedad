"""The layer operators captured into CUDA graphs and replayed on other inputs, and two calls at once on two streams: every path that sizes and
alignment choose."""

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def fill(t, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    if t.dtype == torch.int32:
        t.copy_(torch.randint(-2, 400, t.shape, generator=g, device=DEV, dtype=torch.int32))
    else:
        t.copy_(torch.randn(t.shape, generator=g, device=DEV))
    return t


def m(T, W, dtype=BF, shift=0):
    return torch.empty(T * W + shift, device=DEV, dtype=dtype)[shift:].view(T, W)


def v(n):
    return torch.empty(n, device=DEV)


def ids(T):
    return torch.empty(T, device=DEV, dtype=torch.int32)


def both_ways(L, x, g, d, h, offsets):
    r = L.gated_recurrence(x, g, offsets, h0=h)
    return [*r, *L.gated_recurrence_backward(d, x, g, r.y, offsets, h0=h, dlast=h)]


OFF = {T: tuple(sorted({0, T // 3, T // 3 + 1, T // 2, T})) for T in (300, 9000)}
CASES = {
    "embed": (lambda L, i, t: [L.embed(i, t)], lambda: [ids(3000), m(300, 64, torch.float32)]),
    **{f"embed_backward_{T}": (lambda L, d, i: [L.embed_backward(d, i, 300, scale=0.5)], lambda T=T: [m(T, 72), ids(T)]) for T in (60, 1500, 9000, 20000)},
    "embed_backward_odd": (lambda L, d, i: [L.embed_backward(d, i, 300)], lambda: [m(3000, 33, torch.float32), ids(3000)]),
    **{f"norm_{W}_{s}": (lambda L, x, w, b, d, k: [L.layer_norm(x, w, b), *L.layer_norm_backward(d, x, w, dskip=k)],
                         lambda W=W, s=s: [m(100, W), v(W), v(W), m(100, W), m(100, W, shift=s)]) for W, s in ((100, 0), (1000, 0), (4096, 0), (1000, 1), (9000, 0))},
    **{f"linear_{T}_{K}_{N}": (lambda L, x, w, b, r, z, d: [*L.linear(x, w, b, act="gelu", residual=r, keep=True), L.linear_dgrad(d, w, act="silu", z=z, residual=x), *L.linear_wgrad(x, d, bias=True)],
                               lambda T=T, K=K, N=N: [m(T, K), m(K, N), v(N), m(T, N), m(T, K), m(T, N)]) for T, K, N in ((70, 64, 128), (515, 333, 411), (40, 1600, 1000), (3000, 520, 264))},
    **{f"recurrence_{T}_{W}": (lambda L, x, g, d, h, T=T: both_ways(L, x, g, d, h, OFFSETS[T]),
        lambda T=T, W=W: [m(T, W), m(T, W), m(T, W), torch.empty(len(OFF[T]) - 1, W, device=DEV)]) for T, W in ((300, 64), (300, 33), (9000, 64), (9000, 130))},
    "step": (lambda L, x, g, h: [*L.gated_recurrence_step(x, g, h)], lambda: [m(16, 200), m(16, 200), torch.empty(16, 200, device=DEV)]),
    "activation": (lambda L, d, z: [L.activation_backward(d, z, "gelu")], lambda: [m(100, 200, torch.float32), m(100, 200)]),
}
OFFSETS = {}


@pytest.fixture(autouse=True)
def _offsets():
    for T, cuts in OFF.items():
        OFFSETS.setdefault(T, torch.tensor(cuts, dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("name", CASES)
def test_captured_and_replayed(llm, name):
    call, make = CASES[name]
    inputs = make()
    for k, t in enumerate(inputs):
        fill(t, k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(llm, *inputs)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(llm, *inputs)
    for seed in (10, 20):
        for k, t in enumerate(inputs):
            fill(t, seed + k)
        for o in got:
            if o is not None:
                o.fill_(3.0)
        graph.replay()
        graph.replay()
        want = call(llm, *inputs)
        for a, b in zip(got, want):
            assert (a is None and b is None) or torch.equal(a, b)
    llm.check()


@pytest.mark.parametrize("name", ["embed_backward_9000", "norm_4096_0", "linear_515_333_411", "linear_3000_520_264", "recurrence_9000_130"])
def test_two_calls_at_once(llm, name):
    call, make = CASES[name]
    sets = [[fill(t, 100 * i + k) for k, t in enumerate(make())] for i in range(2)]
    want = [call(llm, *s) for s in sets]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(call(llm, *sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for one in got[i]:
            for a, b in zip(one, want[i]):
                assert (a is None and b is None) or torch.equal(a, b)
    llm.check()
