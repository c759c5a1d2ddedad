"""The weight gradient from 8-bit activations where its operand is converted before the product (many tokens and output
columns): sizes, alignments, precision relative to the norm of the result."""

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def llm():
    from paper_2308_15164_b200 import llm

    return llm


def randn(seed, *s):
    return torch.randn(*s, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


def want_of(c, dy):
    """In 64 bits on the GPU (the products are large), from the values that the checkpoint stands for."""
    s = torch.exp2(c.e.double() - 127.0)
    s = torch.where(c.e == 255, torch.full_like(s, float("nan")), s)
    x = (c.q.double().view(c.q.shape[0], -1, 32) * s[..., None]).view(c.q.shape[0], -1)[:, :c.width]
    return x.t() @ dy.double()


def off_by(got, want):
    return float((got.double() - want).norm() / want.norm())


# Products of bf16 numbers are exact in fp32.  What is added up in one accumulator loses low bits at every addition: 2.8e-6 of
# the result's norm over 512 additions (8192 tokens) was measured, 5.5e-9 each; sums of 16 runs of 64 tokens (64 additions) leave
# 3.5e-7; adding up the sums in fp32 2^-24 each time.  Bound: half as much again.
FEW = 5e-7

# whole tiles and cut ones (1100 x 4000 x 1300: 96 tiles on 74 pairs; 8192 x 2048 x 2600: 88), cut ones only, one row or column
# beyond a tile, runs of tokens that end inside 64, sizes that no 16-byte boundary divides
SHAPES = [(1025, 300, 600), (1025, 100, 513), (1100, 1000, 1111), (2048, 1024, 1111), (1500, 2500, 3000), (2085, 700, 1025), (1100, 4000, 1300), (8192, 2048, 2600),
          (4097, 33, 514), (1088, 257, 768), (9000, 64, 1000)]


@pytest.mark.parametrize("T,D,N", SHAPES)
def test_operand_converted_before_the_product(llm, T, D, N):
    c = llm.ckpt8_quantize(randn(T + D, T, D) * torch.exp(randn(2, T, 1)))
    dy = (0.1 * randn(N, T, N)).bfloat16()
    want = want_of(c, dy)
    got = llm.ckpt8_wgrad(c, dy)
    llm.check()
    assert off_by(got, want) <= FEW
    # element by element: 64 additions lose at most a unit of a sum that grows to the magnitudes' sum, 32 * 2^-23 of it, then the sums in fp32
    x = llm.ckpt8_dequantize(c, torch.float32).double().abs()
    bound = x.t() @ dy.double().abs() * (4e-6 + T / 1024 * 2.0 ** -24)
    assert ((got.double() - want).abs() <= bound).all()
    for _ in range(3):                                            # calls in a row, and equal bits
        again = llm.ckpt8_wgrad(c, dy)
    assert torch.equal(got, again)
    # a slice of a flat gradient, stored and added to
    flat = torch.full((D * N + 5,), 3.0, device=DEV)
    view = flat[3:3 + D * N].view(D, N)
    llm.ckpt8_wgrad(c, dy, out=view)
    assert torch.equal(view, got)
    llm.ckpt8_wgrad(c, dy, out=view, accumulate=True)
    assert torch.equal(view, got + got) and (flat[:3] == 3).all() and (flat[3 + D * N:] == 3).all()
    # dy whose rows start anywhere (packed before the product), dw with gaps between rows
    wide = torch.full((T, N + 11), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 3:3 + N] = dy
    out = torch.full((D, N + 6), 9.0, device=DEV)
    llm.ckpt8_wgrad(c, wide[:, 3:3 + N], out=out[:, 2:2 + N])
    assert torch.equal(out[:, 2:2 + N], got) and (out[:, :2] == 9).all() and (out[:, 2 + N:] == 9).all()
    # and at 16-byte boundaries with gaps
    pad = torch.full((T, (N + 15) // 8 * 8), float("nan"), dtype=torch.bfloat16, device=DEV)
    pad[:, :N] = dy
    assert torch.equal(llm.ckpt8_wgrad(c, pad[:, :N]), got)
    llm.check()


def test_blocks_at_the_ends_of_the_range_and_a_nan_block(llm):
    T, D, N = 1300, 300, 700
    x = randn(1, T, D)
    x[:, 32:64] *= 1e30
    x[:, 64:96] *= 1e-30
    x[:, 96:128] = 0
    dy = (0.1 * randn(2, T, N)).bfloat16()
    c = llm.ckpt8_quantize(x)
    want, got = want_of(c, dy), llm.ckpt8_wgrad(c, dy)
    for a in range(0, D, 32):
        if a != 96:
            assert off_by(got[a:a + 32], want[a:a + 32]) <= FEW, a
    assert (got[96:128] == 0).all()
    x[1290, 130] = float("nan")
    bad = llm.ckpt8_wgrad(llm.ckpt8_quantize(x), dy)
    assert torch.isnan(bad[128:160]).all() and torch.equal(bad[:128], got[:128]) and torch.equal(bad[160:], got[160:])
