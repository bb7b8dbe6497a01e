"""More refusals of the C ABI for the products of a language model and what is done to their rows, before anything touches a device."""

import ctypes as C

import pytest

from paper_2101_11714_amd import binding as B

F32, BF16, F16 = 0, 1, 2


def rows(data=64, ld=16, type=F32):
    return C.byref(B.TTRows(data, ld, type))


def toks(data=64, L=5, bits=64):
    return C.byref(B.TTTokens(data, L, bits))


@pytest.mark.parametrize("scale", [1e-37, 1e-45, 0.99e-36, 1.01e30])
def test_scales_that_32_bits_cannot_bear_are_refused(scale):
    l = B.lib()
    assert l.tt_token_logprob_fwd(rows(), toks(), scale, 64, 64, 64, 0, None, 64, None, 5, 16, None, 0, None) == -3
    assert l.tt_token_logprob_bwd(rows(), toks(), scale, 64, 64, 64, 64, rows(), 5, 16, None) == -3
    assert b"scale" in l.tt_last_error()
