"""Embedding lookup and its gradient against their definitions in 64 bits."""

import pytest
import torch

from tests import llm_layers_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def ids_of(T, V, seed, how="mixed"):
    g = gen(seed)
    if how == "one":
        return torch.full((T,), V // 2, dtype=torch.int32, device=DEV)
    ids = (torch.rand(T, generator=g, device=DEV) ** 4 * V).to(torch.int32).clamp(max=V - 1)      # some far more often than others
    if how == "none":
        ids.fill_(-1)
    elif how == "mixed":
        ids[::7] = -1
        ids[3::11] = V
        ids[5::23] = torch.iinfo(torch.int32).min
        ids[6::29] = torch.iinfo(torch.int32).max
    return ids


@pytest.mark.parametrize("T,V,W", [(1, 1, 1), (1, 5, 8), (3, 7, 5), (33, 100, 64), (257, 1000, 129), (70, 300, 2048), (41, 50, 5000), (5000, 90, 16)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lookup(llm, T, V, W, dtype):
    table = torch.randn(V, W, generator=gen(1), device=DEV)
    ids = ids_of(T, V, T)
    y = llm.embed(ids, table, scale=1.7, dtype=DT[dtype])
    assert y.dtype == DT[dtype]
    R.close(y, R.embed(ids, table, float(torch.tensor(1.7))), torch.zeros(()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift,pad", [(0, 3), (1, 0), (4, 8), (3, 5)])
def test_lookup_of_slices(llm, dtype, shift, pad):
    """Rows of a wider buffer, from an address that is not 16-byte aligned; what lies beside them stays."""
    V, W, T = 60, 40, 37
    whole = torch.randn(V * (W + pad) + shift, generator=gen(2), device=DEV)
    table = whole[shift:].view(V, W + pad)[:, :W]
    ids = ids_of(T, V, 5)
    buf = torch.full((T * (W + pad) + shift,), 7.0, device=DEV, dtype=DT[dtype])
    y = buf[shift:].view(T, W + pad)[:, :W]
    out = llm.embed(ids, table, scale=0.5, dtype=DT[dtype], y=y)
    assert out.data_ptr() == y.data_ptr()
    R.close(y, R.embed(ids, table, 0.5), torch.zeros(()))
    assert (buf[:shift] == 7).all() and (buf[shift:].view(T, W + pad)[:, W:] == 7).all()


SIZES = [(1, 1, 1), (1, 9, 8), (2, 9, 3), (31, 40, 7), (32, 40, 8), (33, 3, 16), (64, 1, 24), (65, 300, 33), (777, 200, 129), (2000, 256, 64), (513, 70000, 4),
         (8192, 500, 8), (8193, 5000, 8), (20000, 66000, 12), (300, 64, 4104), (100, 12, 9000)]


@pytest.mark.parametrize("T,V,W", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient(llm, T, V, W, dtype):
    dy = torch.randn(T, W, generator=gen(T), device=DEV).to(DT[dtype])
    ids = ids_of(T, V, T + V)
    want, tol = R.embed_backward(dy, ids, V, float(torch.tensor(1.3)))
    spoiled = torch.where(((ids < 0) | (ids >= V))[:, None], torch.full((), float("nan"), device=DEV, dtype=dy.dtype), dy)     # rows of padding are not read
    got = llm.embed_backward(spoiled, ids, V, scale=1.3)
    R.close(got, want, tol)
    assert torch.equal(llm.embed_backward(dy, ids, V, scale=1.3), got)
    base = torch.randn(V, W, generator=gen(3), device=DEV)
    acc = base.clone()
    llm.embed_backward(dy, ids, V, scale=1.3, out=acc, accumulate=True)
    there = torch.zeros(V, dtype=torch.bool, device=DEV)
    there[ids[(ids >= 0) & (ids < V)].long()] = True
    assert torch.equal(acc[~there], base[~there])
    R.close(acc, R.d(base) + want, tol + 2 * R.U32 * (R.d(base).abs() + want.abs()))


@pytest.mark.parametrize("how", ["one", "none", "plain"])
@pytest.mark.parametrize("T", [1, 32, 33, 1000, 9000, 40000])
def test_gradient_of_crowded_rows(llm, how, T):
    V, W = 37, 24
    dy = torch.randn(T, W, generator=gen(T), device=DEV)
    ids = ids_of(T, V, T, how)
    R.close(llm.embed_backward(dy, ids, V), *R.embed_backward(dy, ids, V, 1.0))


@pytest.mark.parametrize("T", [1, 200, 5000, 20000])
@pytest.mark.parametrize("V,W", [(1, 1), (1, 2), (2, 1), (3, 1)])
def test_tiny_tables_of_padding_alone(llm, T, V, W):
    """Every row is written, however few there are and however the tokens are sorted."""
    out = torch.full((V, W), 7.0, device=DEV)
    llm.embed_backward(torch.ones(T, W, device=DEV), torch.full((T,), -1, dtype=torch.int32, device=DEV), V, out=out)
    assert (out == 0).all()


def test_many_tokens(llm):
    """More blocks of the sort than one, all passes."""
    T, V, W = 300001, 152064, 1
    dy = torch.randn(T, W, generator=gen(1), device=DEV)
    ids = torch.randint(-3, V + 3, (T,), generator=gen(2), device=DEV, dtype=torch.int32)
    R.close(llm.embed_backward(dy, ids, V), *R.embed_backward(dy, ids, V, 1.0))


@pytest.mark.parametrize("T,V,W,dtype", [(30000, 40, 2048, "bf16"), (20000, 3, 1500, "f32"), (60000, 500, 520, "bf16"), (3000, 2900, 1030, "bf16"), (16384, 77, 40, "f32"), (16385, 77, 40, "f32")])
def test_long_runs_of_wide_rows(llm, T, V, W, dtype):
    """Chunks of more than sixteen tokens, runs over many of them; the sort by one cluster and by launches."""
    dy = torch.randn(T, W, generator=gen(T), device=DEV).to(DT[dtype])
    ids = ids_of(T, V, 11)
    at = torch.where((ids >= 0) & (ids < V), ids, V).long()
    want = torch.zeros(V + 1, W, dtype=torch.float64, device=DEV).index_add_(0, at, dy.double())[:-1]
    size = torch.zeros(V + 1, W, dtype=torch.float64, device=DEV).index_add_(0, at, dy.double().abs())[:-1]
    # a chunk's sum has at most 256 additions, the groups of a join add up the chunks in turn: some thousand at most, as bounded in the reference
    tol = (torch.bincount(at, minlength=V + 1)[:-1, None] + 2) * R.U32 * size
    got = llm.embed_backward(dy, ids, V)
    R.close(got, want.cpu(), tol.cpu())
    acc = torch.ones_like(got)
    llm.embed_backward(dy, ids, V, out=acc, accumulate=True)
    R.close(acc, (1 + want).cpu(), (tol + 2 * R.U32 * (1 + want.abs())).cpu())
    assert torch.equal(llm.embed_backward(dy, ids, V), got)


@pytest.mark.parametrize("shift,pad", [(0, 4), (1, 0), (2, 3)])
def test_gradient_into_a_slice(llm, shift, pad):
    T, V, W = 200, 50, 40
    dy = torch.randn(T, W + pad, generator=gen(4), device=DEV).bfloat16()[:, :W]
    ids = ids_of(T, V, 9)
    buf = torch.full((V * (W + pad) + shift,), 5.0, device=DEV)
    out = buf[shift:].view(V, W + pad)[:, :W]
    llm.embed_backward(dy, ids, V, out=out)
    R.close(out, *R.embed_backward(dy, ids, V, 1.0))
    assert (buf[:shift] == 5).all() and (buf[shift:].view(V, W + pad)[:, W:] == 5).all()


def test_no_tokens(llm):
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    assert llm.embed(none, torch.ones(4, 6, device=DEV)).shape == (0, 6)
    out = torch.full((4, 6), 3.0, device=DEV)
    llm.embed_backward(torch.zeros(0, 6, device=DEV), none, 4, out=out, accumulate=True)
    assert (out == 3).all()
    llm.embed_backward(torch.zeros(0, 6, device=DEV), none, 4, out=out)
    assert (out == 0).all()


def test_against_differences(llm):
    """The gradient of a sum of products by differences of the lookup."""
    T, V, W = 9, 5, 4
    table, ids = torch.randn(V, W, generator=gen(1), device=DEV), ids_of(T, V, 3)
    dy = torch.randn(T, W, generator=gen(2), device=DEV)
    f = lambda t: (R.d(llm.embed(ids, t, scale=2.0, dtype=torch.float32)) * R.d(dy)).sum()  # noqa: E731
    got = llm.embed_backward(dy, ids, V, scale=2.0)
    for i in range(V):
        for j in range(W):
            step = torch.zeros_like(table)
            step[i, j] = 0.5
            # linear: the difference is exact but for the roundings of the lookups, |2 table| 2^-24 for each of at most T tokens
            assert abs(float(f(table + step) - f(table - step)) - float(got[i, j])) < T * 16 * R.U32 * 8
