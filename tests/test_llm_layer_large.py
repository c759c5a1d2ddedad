"""Matrices of more than 2^31 elements: what lies behind the offset that 32 bits hold is what a call on those rows alone gives."""

import pytest
import torch

from tests import llm_layers_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16
T, W = 70000, 32768                  # 2.3e9 elements


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def big(rows=T, width=W, dtype=BF):
    x = torch.empty(rows, width, device=DEV, dtype=dtype)
    part = torch.randn(1000, width, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(dtype)
    for i in range(0, rows, 1000):
        x[i:i + 1000] = part[: min(1000, rows - i)]
    return x


def test_layer_norm(llm):
    x, w = big(width=16000), torch.ones(16000, device=DEV)
    x = torch.cat((x, x))[: 140000]                       # 2.24e9 elements
    n = llm.layer_norm(x, w)
    assert torch.equal(n[-5:], llm.layer_norm(x[-5:], w)) and torch.equal(n[135000], n[0])
    del n
    g = llm.layer_norm_backward(x, x, w, bias=False)
    want = llm.layer_norm_backward(x[-5:], x[-5:], w, bias=False).dx
    assert torch.equal(g.dx[-5:], want)


def test_embedding(llm):
    table = torch.zeros(T, W, device=DEV)
    table[-1], table[-2] = 1.5, 2.5
    ids = torch.tensor([T - 1, 0, T - 2, T, T - 1], dtype=torch.int32, device=DEV)
    y = llm.embed(ids, table, dtype=torch.float32)
    assert y[:, 0].tolist() == [1.5, 0.0, 2.5, 0.0, 1.5] and y[:, -1].tolist() == [1.5, 0.0, 2.5, 0.0, 1.5]
    dy = torch.ones(5, W, device=DEV)
    llm.embed_backward(dy, ids, T, out=table)
    assert table[:, 0].sum() == 4 and table[-1].eq(2).all() and table[-2].eq(1).all() and table[0].eq(1).all() and table[1:100].eq(0).all()
    many = torch.full((3000,), T - 3, dtype=torch.int32, device=DEV)
    llm.embed_backward(torch.ones(3000, W, device=DEV, dtype=BF), many, T, out=table, accumulate=True)
    assert table[-3].eq(3000).all() and table[-1].eq(2).all()


def test_linear(llm):
    K = 16
    x, w = big(T, K), big(K, W)
    y = llm.linear(x, w).y
    assert torch.equal(y[-300:], llm.linear(x[-300:], w).y)
    dx = llm.linear_dgrad(y, w)
    # a call on 300 rows alone cuts the 32768 products of an element into parts and rounds elsewhere: against the definition instead
    R.close(dx[-300:], *R.dgrad(y[-300:], w, "none", None, None))
    del y, dx
    a, b = big(K, 50000), big(K, 50000)
    dw = llm.linear_wgrad(a, b).dw                        # 2.5e9 elements
    assert torch.equal(dw[-256:, -256:], llm.linear_wgrad(a[:, -256:].contiguous(), b[:, -256:].contiguous()).dw)


def test_recurrence(llm):
    x = big()
    offsets = torch.tensor([0, 7, T - 40, T - 9, T], dtype=torch.int32, device=DEV)
    r = llm.gated_recurrence(x, x, offsets)
    alone = llm.gated_recurrence(x[-9:], x[-9:])
    # the same nine rows in a tile of their own: the products inside a warp's rows may be taken apart elsewhere
    assert torch.allclose(r.y[-9:].float(), alone.y.float(), rtol=2.0 ** -7, atol=1e-5) and torch.allclose(r.last[3:], alone.last, rtol=1e-5, atol=1e-6)
    del r
    y = llm.gated_recurrence(x, x, offsets).y
    b = llm.gated_recurrence_backward(x, x, x, y, offsets)
    one = llm.gated_recurrence_backward(x[-9:], x[-9:], x[-9:], y[-9:])
    assert torch.allclose(b.dx[-9:].float(), one.dx.float(), rtol=2.0 ** -7, atol=1e-5) and torch.allclose(b.dg[-9:].float(), one.dg.float(), rtol=2.0 ** -7, atol=1e-4)
