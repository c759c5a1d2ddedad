"""8-bit activation checkpoints: packing bit for bit, unpacking, and the weight gradient taken from them."""

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


def randn(seed, *s):
    return torch.randn(*s, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


def check_pack(llm, x):
    c = llm.ckpt8_quantize(x)
    q, e = R.pack(x)
    assert torch.equal(c.e.cpu().long(), e) and torch.equal(c.q.cpu().to(R.D), q)
    want = R.unpack(q, e, x.shape[1])
    for dt in DT.values():
        got = R.d(llm.ckpt8_dequantize(c, dt))
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    return c


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(1, 1), (3, 7), (2, 31), (5, 32), (4, 33), (7, 100), (64, 256), (33, 1000), (2, 4096), (515, 1537)])
def test_pack_and_unpack_are_exact(llm, T, D, dtype):
    x = randn(T + D, T, D) * torch.exp(3 * randn(1, T, 1))
    x[:, ::17] *= 50
    x[0, : D // 2] = 0
    check_pack(llm, x.to(DT[dtype]))
    big = torch.full((T, D + 5), float("nan"), device=DEV, dtype=DT[dtype])
    big[:, 1:1 + D] = x
    check_pack(llm, big[:, 1:1 + D])                               # rows that no 16-byte load can start at
    c = llm.ckpt8_quantize(x.to(DT[dtype]))
    out = torch.full((T, D + 3), 4.0, device=DEV, dtype=torch.bfloat16)
    llm.ckpt8_dequantize(c, torch.bfloat16, out=out[:, 1:1 + D])
    assert (out[:, 0] == 4).all() and (out[:, 1 + D:] == 4).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pack_at_the_edges_of_the_format(llm, dtype):
    """Blocks whose maximum sits at a power's limit, ties, subnormal, huge, infinite and NaN blocks, zeros of either sign."""
    b = torch.zeros(14, 32, device=DEV)
    b[0, 0] = 127.0
    b[1, 0] = 127.5
    b[2, :5] = torch.tensor([127.0, 0.5, 1.5, -2.5, 2.4999])       # ties go to even
    b[3, :] = -0.0
    b[4, 3] = 1e-40
    b[5, 3] = 3.3e38
    b[5, 4] = -3.3e38
    b[6, 7] = float("inf")
    b[7, 7] = float("nan")
    b[8, 7] = float("-inf")
    b[9, :] = 2.0 ** -126
    b[10, 0] = 127.0 * 2.0 ** -127
    b[11, 0] = 128.0 * 2.0 ** -127
    b[12, :3] = torch.tensor([2.0 ** -133, -(2.0 ** -128), 3 * 2.0 ** -128])
    b[13, 0] = -127.0
    x = b.to(DT[dtype])
    c = check_pack(llm, x)
    assert c.e[6, 0] == 255 and c.e[7, 0] == 255 and c.e[8, 0] == 255 and c.e[0, 0] == 127 and c.e[3, 0] == 0
    assert torch.isnan(llm.ckpt8_dequantize(c, torch.float32)[6:9]).all()


def test_every_exponent(llm):
    x = torch.zeros(255, 32, device=DEV)
    x[:, 5] = torch.exp2(torch.arange(255, device=DEV).double() - 127).float()
    x[:, 6] = -x[:, 5] * 0.37
    check_pack(llm, x)


def wgrad_want(q, e, width, dy):
    x, dd = R.unpack(q.cpu(), e.cpu(), width), R.d(dy)
    want = x.t() @ dd
    steps = -(-q.shape[0] // 16) + 32
    # products of bf16 numbers are exact in fp32; an accumulation of `steps` groups loses at most one unit of the running sum each
    return want, (x.abs().t() @ dd.abs()) * (steps * 2.0 ** -23)


SHAPES = [(1, 1, 1), (1, 33, 5), (3, 32, 8), (16, 128, 256), (63, 100, 40), (64, 128, 256), (65, 129, 257), (200, 31, 300), (515, 1000, 1111), (1024, 256, 512),
          (2000, 160, 72), (130, 700, 1024), (4096, 128, 128), (77, 2500, 3000)]


@pytest.mark.parametrize("T,D,N", SHAPES)
def test_weight_gradient(llm, T, D, N):
    x = randn(T * 7 + D, T, D) * torch.exp(randn(2, T, 1))
    dy = (0.1 * randn(N, T, N)).bfloat16()
    c = llm.ckpt8_quantize(x)
    want, tol = wgrad_want(c.q, c.e, D, dy)
    got = llm.ckpt8_wgrad(c, dy)
    llm.check()
    R.close(got, want, tol, "dw")
    again = llm.ckpt8_wgrad(c, dy)
    assert torch.equal(got, again)
    # into a slice of a flat gradient that starts anywhere, stored and added
    flat = torch.full((D * N + 5,), 3.0, device=DEV)
    view = flat[3:3 + D * N].view(D, N)
    llm.ckpt8_wgrad(c, dy, out=view)
    assert torch.equal(view, got) and (flat[:3] == 3).all() and (flat[3 + D * N:] == 3).all()
    llm.ckpt8_wgrad(c, dy, out=view, accumulate=True)
    assert torch.equal(view, got + got) and (flat[:3] == 3).all() and (flat[3 + D * N:] == 3).all()
    # dy and dw with gaps between rows, dy starting at any element
    wide = torch.full((T, N + 11), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 3:3 + N] = dy
    out = torch.full((D, N + 6), 9.0, device=DEV)
    llm.ckpt8_wgrad(c, wide[:, 3:3 + N], out=out[:, 2:2 + N])
    assert torch.equal(out[:, 2:2 + N], got) and (out[:, :2] == 9).all() and (out[:, 2 + N:] == 9).all()
    pad = torch.full((T, (N + 15) // 8 * 8), float("nan"), dtype=torch.bfloat16, device=DEV)
    pad[:, :N] = dy
    assert torch.equal(llm.ckpt8_wgrad(c, pad[:, :N]), got)
    llm.check()


def test_weight_gradient_of_extreme_blocks(llm):
    """Blocks near the ends of the exponent range, blocks of zeros, and a NaN block, which reaches its own columns only."""
    T, D, N = 70, 160, 24
    x = randn(1, T, D)
    x[:, 32:64] *= 1e30
    x[:, 64:96] *= 1e-36
    x[:, 96:128] = 0
    dy = (0.1 * randn(2, T, N)).bfloat16()
    c = llm.ckpt8_quantize(x)
    want, tol = wgrad_want(c.q, c.e, D, dy)
    got = llm.ckpt8_wgrad(c, dy)
    R.close(got, want, tol, "dw")
    x[5, 130] = float("nan")
    bad = llm.ckpt8_wgrad(llm.ckpt8_quantize(x), dy)
    assert torch.isnan(bad[128:]).all() and torch.equal(bad[:128], got[:128])


def test_weight_gradient_without_tokens(llm):
    c = llm.ckpt8_quantize(torch.zeros(0, 40, device=DEV))
    dy = torch.zeros(0, 12, dtype=torch.bfloat16, device=DEV)
    assert (llm.ckpt8_wgrad(c, dy) == 0).all()
    keep = torch.ones(40, 12, device=DEV)
    llm.ckpt8_wgrad(c, dy, out=keep, accumulate=True)
    assert (keep == 1).all()
    assert llm.ckpt8_dequantize(c).shape == (0, 40)


def test_long_contraction(llm):
    """Precision over many tokens: against 64 bits, relative to the whole result."""
    T, D, N = 16384, 128, 256
    c = llm.ckpt8_quantize(randn(1, T, D))
    dy = randn(2, T, N).bfloat16()
    got = llm.ckpt8_wgrad(c, dy)
    want, tol = wgrad_want(c.q, c.e, D, dy)
    R.close(got, want, tol, "dw")


def test_streams(llm):
    T, D, N = 900, 300, 500
    x, dy = randn(1, T, D), randn(2, T, N).bfloat16()
    a = llm.ckpt8_wgrad(llm.ckpt8_quantize(x), dy)
    ss = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for s in ss:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs.append(llm.ckpt8_wgrad(llm.ckpt8_quantize(x), dy))
    torch.cuda.synchronize()
    assert all(torch.equal(o, a) for o in outs)


def test_rows_beyond_two_gigaelements_and_slices_of_a_checkpoint(llm):
    T, D, ld = 3, 1030, 1_200_000_000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    store = torch.empty((T - 1) * ld + D, dtype=torch.bfloat16, device=DEV)
    far = store.as_strided((T, D), (ld, 1))
    x = randn(4, T, D).bfloat16()
    far.copy_(x)
    c = check_pack(llm, far)
    want = llm.ckpt8_dequantize(c, torch.bfloat16)
    llm.ckpt8_dequantize(c, torch.bfloat16, out=far)
    assert torch.equal(far, want)
    del store, far
    torch.cuda.empty_cache()
    part = llm.Ckpt8(c.q[1:], c.e[1:], D)                # the exponents of a slice start at any byte
    assert torch.equal(llm.ckpt8_dequantize(part, torch.bfloat16), want[1:])
    dy = randn(5, T, 40).bfloat16()
    got = llm.ckpt8_wgrad(part, dy[1:])
    w, tol = wgrad_want(c.q[1:], c.e[1:], D, dy[1:])
    R.close(got, w, tol, "dw")
