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


def heads(data=64, ld=64, ld_head=16, n=4, type=F32):
    return C.byref(B.TTHeads(data, ld, ld_head, n, type))


@pytest.mark.parametrize("q_type,k_type,q,k", [(F32, F32, 64, 64), (F32, F32, 64, 124), (BF16, F32, 4096, 4096 - 60), (F16, BF16, 64, 94)])
@pytest.mark.parametrize("n_rows,accumulate", [(5000, 0), (5000, 1), (1, 1), (0, 0)])
def test_one_array_does_not_take_the_gradients_of_both_weights(q_type, k_type, q, k, n_rows, accumulate):
    # (queries and keys are summed apart: one of the sums would be lost)
    l = B.lib()
    need = l.tt_qk_norm_rotate_bwd_workspace_bytes(n_rows, 4, 4, 16)
    call = lambda a, b: l.tt_qk_norm_rotate_bwd(heads(), heads(), heads(), heads(), None, 1, 1e-6, None, F32, None, F32, heads(), heads(), a, q_type, b, k_type, accumulate, n_rows, 16, 256, need, None)  # noqa: E731
    assert call(q, k) == -3 and b"overlap" in l.tt_last_error()
