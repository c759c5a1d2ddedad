"""What the language-model operators refuse because they could not do it right, and workspaces that stay within bounds.  Nothing
here needs a GPU: every call returns from its checks."""

import pytest

from tests.test_llm_refusals import B, P, backward, forward, policy, preference  # noqa: F401  (B: the fixture)


@pytest.mark.parametrize("call", [policy, preference])
@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2)])
def test_rows_whose_bytes_pass_32_bits(B, call, dtype, size):  # noqa: F811
    """A row's bytes are counted in 32 bits, in chunks of up to 16 KB."""
    for V in ((1 << 32) // size, (1 << 32) // size - 1, ((1 << 32) - (1 << 14)) // size + 1, (1 << 31) - 1 if size == 2 else 1 << 30):
        assert call(B, V=V, ld=V, ld_d=V, dtype=dtype) == B.ELIMIT
        assert b"vocab" in B.lib.abs_last_error(None)
    for V in (((1 << 32) - (1 << 16)) // size, 1 << 20):                  # refused for something that is looked at later
        assert call(B, V=V, ld=V, ld_d=V, dtype=dtype, n=0) == B.ENOMEM


def test_tokens_whose_steps_pass_31_bits(B):  # noqa: F811
    """An answer's rows are counted in 32 bits, in steps of 512."""
    for T in ((1 << 31) - 1, (1 << 31) - 512):
        assert preference(B, T=T) == B.ELIMIT
    assert preference(B, T=(1 << 31) - 513, n=0) == B.ENOMEM


@pytest.mark.parametrize("D,N", [(4096, 512), (128, 256), (100, 64), (18944, 256)])
def test_partial_sums_do_not_grow_with_the_tokens(B, D, N):  # noqa: F811
    """The weight gradient's workspace for few output columns: partial sums of at most one tile for each pair of SMs."""
    for T in (4096, 1 << 17, 1 << 20, 1 << 24):
        assert B.lib.abs_ckpt8_wgrad_workspace(T, D, N, P, N) <= 74 * 256 * 256 * 4


@pytest.mark.parametrize("kw,text", [
    (dict(dx=2 * P, dh=3 * P, dgate=2 * P), b"two outputs"), (dict(dx=2 * P, dh=2 * P, dgate=4 * P), b"two outputs"), (dict(dx=2 * P, dh=3 * P, dgate=3 * P), b"two outputs"),
    (dict(dx=2 * P, dh=3 * P, dgate=4 * P, dw_pre=5 * P, dw_post=5 * P), b"two outputs"),
    # dh is formed from h when dx and dgate of the row are written already
    (dict(h=2 * P, dx=2 * P, dh=3 * P, dgate=4 * P), b"must not be h"), (dict(h=4 * P, dx=2 * P, dh=3 * P, dgate=4 * P), b"must not be h"),
    (dict(h=2 * P, kind=1, dx=2 * P, dh=3 * P, dgate=4 * P), b"must not be h")])
def test_outputs_that_would_spoil_each_other(B, kw, text):  # noqa: F811
    assert backward(B, **(dict(dw_pre=6 * P, dw_post=7 * P) | kw)) == B.EINVAL
    assert text in B.lib.abs_last_error(None)


def test_two_outputs_of_the_join_at_one_place(B):  # noqa: F811
    assert forward(B, y=2 * P, n=2 * P) == B.EINVAL and b"two outputs" in B.lib.abs_last_error(None)
