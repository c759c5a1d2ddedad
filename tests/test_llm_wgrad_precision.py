"""Precision of the weight gradient from 8-bit activations over many tokens, relative to the norm of the result."""

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
# the result's norm over 512 additions (8192 tokens) was measured, 5.5e-9 each; sums of at most 32 runs of 64 tokens (128 additions)
# leave 7e-7; adding up the sums in fp32 2^-24 each time.  Bound: half as much again.
MANY = 1.1e-6


@pytest.mark.parametrize("T,D,N", [(8192, 128, 256), (8192, 1000, 512), (32768, 512, 300), (8192, 9728, 512), (16384, 18944, 256), (8200, 6000, 130), (70000, 100, 64)])
def test_many_tokens_and_few_output_columns(llm, T, D, N):
    """Converted in the kernel: tiles that are cut along the tokens, and more tiles than pairs of SMs, which are not."""
    c = llm.ckpt8_quantize(randn(1, T, D))
    dy = randn(2, T, N).bfloat16()
    got = llm.ckpt8_wgrad(c, dy)
    want = want_of(c, dy)
    assert off_by(got, want) <= MANY
    keep = randn(3, D, N)
    out = keep.clone()
    llm.ckpt8_wgrad(c, dy, out=out, accumulate=True)
    assert off_by(out, want + keep.double()) <= MANY
    assert torch.equal(llm.ckpt8_wgrad(c, dy), got)
    llm.check()


@pytest.mark.parametrize("T,D,N", [(1, 19000, 200), (1000, 10000, 300), (2048, 18944, 256), (700, 9728, 512), (130, 40000, 40)])
def test_more_tiles_than_pairs_of_multiprocessors(llm, T, D, N):
    """Few tokens and output columns, many input columns: several tiles for each pair, whole ones and what is left of them."""
    c = llm.ckpt8_quantize(randn(4, T, D))
    dy = randn(5, T, N).bfloat16()
    got = llm.ckpt8_wgrad(c, dy)
    assert off_by(got, want_of(c, dy)) <= MANY
    flat = torch.full((D * N + 5,), 3.0, device=DEV)
    view = flat[3:3 + D * N].view(D, N)
    llm.ckpt8_wgrad(c, dy, out=view)
    assert torch.equal(view, got)
    llm.ckpt8_wgrad(c, dy, out=view, accumulate=True)
    assert torch.equal(view, got + got) and (flat[:3] == 3).all() and (flat[3 + D * N:] == 3).all()
    llm.check()
