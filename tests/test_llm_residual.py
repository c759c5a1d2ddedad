"""The residual join of a transformer block, forward and backward, against its definition in 64 bits and against differences."""

import pytest
import torch

from tests import llm_reference as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda"


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def make(T, D, dtype, gate, post, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    dt = DT[dtype]
    a = {"x": (3 * n(T, D)).to(dt), "h": n(T, D).to(dt), "y": (3 * n(T, D)).to(dt), "dn": (0.1 * n(T, D)).to(dt), "dy": (0.05 * n(T, D)).to(dt)}
    p = {"w_pre": 1 + 0.2 * n(D), "w_post": 1 + 0.2 * n(D) if post else None,
         "gate": {"none": None, "channel": n(D), "element": (2 * n(T, D)).to(dt)}[gate]}
    return a, p


def check_forward(llm, a, p, scale, **kw):
    y, n = llm.residual_norm(a["x"], a["h"], **p, scale=scale, **kw)
    wy, wn, ty, tn = R.residual(a["x"], a["h"], **p, scale=scale)
    R.close(y, wy, ty, "y")
    R.close(n, wn, tn, "n")
    return y, n


def check_backward(llm, a, p, scale, dy=True, **kw):
    up = a["dy"] if dy else None
    r = llm.residual_norm_backward(a["dn"], up, a["y"], a["h"], **p, scale=scale, **kw)
    want, tol = R.residual_backward(a["dn"], up, a["y"], a["h"], **p, scale=scale)
    for k, v in r._asdict().items():
        assert (v is None) == (k not in want), k
        if v is not None:
            R.close(v, want[k], tol[k], k)
    return r


SHAPES = [(1, 1), (2, 3), (3, 31), (5, 32), (1, 64), (4, 100), (7, 257), (300, 64), (2, 1000), (3, 1024), (650, 1024), (9, 1537), (2, 4096), (3, 5120), (2, 8192),
          (1, 16384), (2, 20001), (1, 32768)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["none", "channel", "element"])
@pytest.mark.parametrize("post", [False, True], ids=["plain", "post"])
def test_forward_and_backward(llm, dtype, gate, post):
    for i, (T, D) in enumerate(SHAPES):
        a, p = make(T, D, dtype, gate, post, 100 + i)
        check_forward(llm, a, p, 0.7)
        check_backward(llm, a, p, 0.7, dy=i % 3 != 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["none", "channel", "element"])
def test_strides_alignments_and_outputs_in_place(llm, dtype, gate):
    T, D = 21, 136
    a, p = make(T, D, dtype, gate, True, 7)

    def shifted(t, left, right, fill=float("nan")):
        big = torch.full((T, D + left + right), fill, dtype=t.dtype, device=DEV)
        big[:, left:left + D] = t
        return big[:, left:left + D]

    flat = torch.randn(4 * D + 3, device=DEV)                     # parameters and their gradients as slices of a flat vector
    flat_g = torch.zeros(4 * D + 3, device=DEV)
    q = dict(p)
    q["w_pre"] = flat[1:1 + D].copy_(p["w_pre"])
    q["w_post"] = flat[1 + D:1 + 2 * D].copy_(p["w_post"])
    if gate == "channel":
        q["gate"] = flat[2 + 2 * D:2 + 3 * D].copy_(p["gate"])
    for left, right in ((0, 0), (1, 2), (8, 0), (0, 8), (3, 1)):
        b = {k: shifted(v, left, right) for k, v in a.items()}
        if gate == "element":
            q["gate"] = shifted(p["gate"], right, left)
        out = shifted(a["x"], 2, 3, 5.0)
        y, n = check_forward(llm, b, q, 0.7, y=out)
        full = out.as_strided((T, D + 5), (D + 5, 1), out.storage_offset() - 2)
        assert (full[:, :2] == 5).all() and (full[:, 2 + D:] == 5).all()
        got = check_backward(llm, b, q, 0.7, dw_pre=flat_g[1:1 + D], dw_post=flat_g[1 + D:1 + 2 * D],
                             **({"dgate": flat_g[2 + 2 * D:2 + 3 * D]} if gate == "channel" else {}))
        assert flat_g[0] == 0 and (flat_g[2 + 3 * D:] == 0).all() and flat_g[1 + 2 * D] == 0
        # added once more: twice the sums (rounded again)
        llm.residual_norm_backward(b["dn"], b["dy"], b["y"], b["h"], **q, scale=0.7, dw_pre=got.dw_pre, dw_post=got.dw_post,
                                   **({"dgate": got.dgate} if gate == "channel" else {}), accumulate=True)
        want, tol = R.residual_backward(a["dn"], a["dy"], a["y"], a["h"], **p, scale=0.7)
        R.close(got.dw_pre, 2 * want["dw_pre"], 2 * tol["dw_pre"], "dw_pre twice")
        if gate == "channel":
            R.close(got.dgate, 2 * want["dgate"], 2 * tol["dgate"], "dgate twice")
        # outputs in place of inputs that nobody needs any more
        xx, hh = b["x"].clone(), b["h"].clone()
        y2, n2 = llm.residual_norm(xx, hh, **q, scale=0.7, y=xx, n=hh)
        y1, n1 = llm.residual_norm(b["x"].clone(), b["h"].clone(), **q, scale=0.7)
        assert torch.equal(y1, y2) and torch.equal(n1, n2)
        dyy, hh, dnn = b["dy"].clone(), b["h"].clone(), b["dn"].clone()
        g1 = llm.residual_norm_backward(dnn, dyy, b["y"], hh, **q, scale=0.7)
        g1 = [None if t is None else t.clone() for t in g1]
        qq = dict(q)
        if gate == "element":
            qq["gate"] = q["gate"].clone()
        g2 = llm.residual_norm_backward(dnn, dyy, b["y"], hh, **qq, scale=0.7, dx=dyy, dh=hh, **({"dgate": qq["gate"]} if gate == "element" else {}))
        for u, v in zip(g1, g2):
            assert u is None and v is None or torch.equal(u, v)
        dyy, hh = b["dy"].clone(), b["h"].clone()
        g3 = llm.residual_norm_backward(dnn, dyy, b["y"], hh, **q, scale=0.7, dx=dnn)
        for u, v in zip(g1, g3):
            assert u is None and v is None or torch.equal(u, v)


def test_zero_rows_and_no_tokens(llm):
    """A row of zeros has rms sqrt(eps): finite everywhere; without tokens the sums are zero (or stay, when added to)."""
    for D in (48, 1000, 4096):
        a, p = make(4, D, "bf16", "channel", True, 3)
        for k in ("x", "h", "y"):
            a[k][1] = 0
        check_forward(llm, a, p, 0.7)
        check_backward(llm, a, p, 0.7)
        e = {k: v[:0] for k, v in a.items()}
        y, n = llm.residual_norm(e["x"], e["h"], **p)
        assert y.shape == n.shape == (0, D)
        r = llm.residual_norm_backward(e["dn"], e["dy"], e["y"], e["h"], **p)
        assert (r.dw_pre == 0).all() and (r.dw_post == 0).all() and (r.dgate == 0).all()
        keep = torch.ones(D, device=DEV)
        r = llm.residual_norm_backward(e["dn"], e["dy"], e["y"], e["h"], **p, dw_pre=keep, accumulate=True)
        assert (keep == 1).all() and (r.dw_post == 0).all()


def test_nan_and_infinity_stay_in_their_rows(llm):
    for D in (100, 2048):
        a, p = make(5, D, "f32", "none", True, 4)
        a["h"][2, 3] = float("nan")
        a["x"][4, 1] = float("inf")
        y, n = llm.residual_norm(a["x"], a["h"], **p)
        assert torch.isnan(n[2]).all() and torch.isfinite(n[[0, 1, 3]]).all() and not torch.isfinite(y[4, 1])


@pytest.mark.parametrize("gate", ["none", "channel", "element"])
@pytest.mark.parametrize("post", [False, True], ids=["plain", "post"])
def test_gradients_against_differences(llm, gate, post):
    """d/ds of <n, dn> + <y, dy> along random directions of every input, from the forward pass alone."""
    T, D = 5, 72
    a, p = make(T, D, "f32", gate, post, 17)
    kw = dict(scale=0.7)
    y, n = llm.residual_norm(a["x"], a["h"], **p, **kw)
    r = llm.residual_norm_backward(a["dn"], a["dy"], y, a["h"], **p, **kw)

    def value(x, h, q):
        y, n = llm.residual_norm(x, h, **q, **kw)
        return float((n.double() * a["dn"].double()).sum() + (y.double() * a["dy"].double()).sum())

    grads = {"x": r.dx, "h": r.dh, "w_pre": r.dw_pre, "w_post": r.dw_post, "gate": r.dgate}
    step = 1e-2
    for name, got in grads.items():
        base = {"x": a["x"], "h": a["h"], **p}
        if base[name] is None:
            assert got is None
            continue
        v = torch.randn(base[name].shape, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV)
        ends = []
        for s in (step, -step):
            b = dict(base)
            b[name] = base[name] + s * v
            ends.append(value(b["x"], b["h"], {k: b[k] for k in ("w_pre", "w_post", "gate")}))
        slope = float((got.double() * v.double()).sum())
        # the value's terms are about 0.1 sqrt(360) = 2 in sum, each with an error of 1e-6 (over the step: 2e-4 at most); the third
        # derivative adds about step^2 of the slope's own scale
        assert abs((ends[0] - ends[1]) / (2 * step) - slope) <= 1e-3 + 1e-3 * abs(slope), name


def test_many_rows_and_streams_give_equal_bits(llm):
    a, p = make(2500, 512, "bf16", "channel", True, 8)
    one = check_backward(llm, a, p, 0.7)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        two = llm.residual_norm_backward(a["dn"], a["dy"], a["y"], a["h"], **p, scale=0.7)
    s.synchronize()
    for u, v in zip(one, two):
        assert torch.equal(u, v)


def test_rows_beyond_two_gigaelements(llm):
    """The last row starts more than 2^31 elements behind the first."""
    T, D, ld = 3, 1030, 1_200_000_000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    a, p = make(T, D, "bf16", "channel", True, 6)
    store = torch.empty((T - 1) * ld + D, dtype=torch.bfloat16, device=DEV)
    far = store.as_strided((T, D), (ld, 1))
    far.copy_(a["x"])
    y, n = llm.residual_norm(far, a["h"], **p, scale=0.7, y=far)
    wy, wn, ty, tn = R.residual(a["x"], a["h"], **p, scale=0.7)
    R.close(y, wy, ty, "y")
    R.close(n, wn, tn, "n")
    far.copy_(a["y"])
    check_backward(llm, a | {"y": far}, p, 0.7)
    del store, far, y
    torch.cuda.empty_cache()


def test_in_a_captured_graph(llm):
    """All operators of a step captured once and replayed on new values."""
    from paper_2308_15164_b200 import llm as L

    T, D, V = 130, 256, 1000
    a, p = make(T, D, "bf16", "channel", True, 9)
    w = (torch.randn(D, V, device=DEV) * D ** -0.5).bfloat16()
    lab = torch.randint(0, V, (T,), device=DEV, dtype=torch.int32)
    adv, wt, old = torch.randn(T, device=DEV), torch.full((T,), 1.0 / T, device=DEV), torch.full((T,), -7.0, device=DEV)
    x, h = a["x"].clone(), a["h"].clone()

    def step():
        y, n = L.residual_norm(x, h, **p, scale=0.7)
        c = L.ckpt8_quantize(n)
        r = L.policy_loss(n @ w, lab, old, adv, wt)
        g = L.residual_norm_backward(r.dlogits @ w.t(), None, y, h, **p, scale=0.7)
        return [r.loss, r.logp, L.ckpt8_wgrad(c, r.dlogits), *g]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (1, 2):
        b, _ = make(T, D, "bf16", "channel", True, 20 + seed)
        x.copy_(b["x"])
        h.copy_(b["h"])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for u, v in zip(got, step()):
            assert torch.equal(u, v)
    L.check()


@pytest.mark.parametrize("dtype,T,D", [("f32", 310, 8192), ("f32", 301, 7001), ("bf16", 700, 5000), ("bf16", 610, 3500), ("f32", 1203, 1537), ("bf16", 305, 8192)])
@pytest.mark.parametrize("gate", ["channel", "element"])
def test_several_rows_per_cta_at_every_split_of_a_row(llm, dtype, T, D, gate):
    a, p = make(T, D, dtype, gate, True, 29)
    check_forward(llm, a, p, 0.7)
    check_backward(llm, a, p, 0.7, dy=True)
    check_backward(llm, a, p, 0.7, dy=False)


@pytest.mark.parametrize("gate", ["none", "channel", "element"])
def test_inner_products_that_cancel(llm, gate):
    """dn w_pre nearly along y: dY is a small difference of large terms, and so is its product with h."""
    a, p = make(40, 1024, "f32", gate, True, 31)
    p["w_pre"] = p["w_pre"].abs() + 0.1
    a["dn"] = a["y"] / p["w_pre"] * (1 + 0.01 * a["dn"])
    check_backward(llm, a, p, 0.7, dy=False)
    check_backward(llm, a, p, 0.7, dy=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(9003, 100), (9600, 257), (7301, 512), (12000, 8), (20001, 33)])
@pytest.mark.parametrize("gate,post", [("none", False), ("channel", True), ("element", True)])
def test_many_narrow_rows(llm, dtype, T, D, gate, post):
    a, p = make(T, D, dtype, gate, post, 37)
    check_forward(llm, a, p, 0.7)
    check_backward(llm, a, p, 0.7, dy=True)
    for k in ("x", "h", "y", "dn", "dy"):             # rows at a distance of D + 3
        wide = torch.full((T, D + 3), float("nan"), dtype=a[k].dtype, device=DEV)
        wide[:, :D] = a[k]
        a[k] = wide[:, :D]
    if gate == "element":
        wide = torch.full((T, D + 3), float("nan"), dtype=p["gate"].dtype, device=DEV)
        wide[:, :D] = p["gate"]
        p["gate"] = wide[:, :D]
    out = [torch.empty(T, D + 3, dtype=a["x"].dtype, device=DEV)[:, :D] for _ in range(3)]
    check_forward(llm, a, p, 0.7, y=out[0], n=out[1])
    check_backward(llm, a, p, 0.7, dy=False, dx=out[0], dh=out[1], dgate=out[2] if gate == "element" else None)
