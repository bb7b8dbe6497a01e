"""Refusals of the operators at a language model's way in that test_lm_cpu.py does not have: none of these calls reaches a launch."""

import ctypes as C

from paper_2101_11714_amd import binding as B


def rows(type=0, ld=1 << 20):
    return C.byref(B.TTRows(64, ld, type))


def test_arrays_of_2_to_the_40_elements_are_refused():
    l = B.lib()
    tokens = lambda L: C.byref(B.TTTokens(64, L, 64))  # noqa: E731
    drop = C.byref(B.TTDropout(64, 0, 0.5))
    n, N = 1 << 25, 1 << 15
    assert l.tt_token_fwd(rows(), 10, N, tokens(n), 1.0, None, rows(), None) == -6
    assert l.tt_token_fwd(rows(), n, N, tokens(10), 1.0, None, rows(), None) == -6
    for f, tail in ((l.tt_token_bwd, (0,)), (l.tt_token_bwd_sgd, (0.1,))):
        assert f(tokens(n), rows(ld=0), 1.0, None, rows(), 10, N, *tail, 256, 1 << 60, None) == -6
        assert f(tokens(10), rows(), 1.0, None, rows(), n, N, *tail, 256, 1 << 60, None) == -6
    assert l.tt_dropout_fwd(rows(), None, drop, rows(), n, N, None) == -6
    assert l.tt_dropout_bwd(rows(), drop, rows(), n, N, None) == -6
    assert l.tt_add_rms_norm_fwd(rows(), None, None, None, 0, 1e-6, None, rows(), None, None, 0, n, N, None) == -6
    assert l.tt_add_rms_norm_bwd(rows(), rows(), 64, None, 0, None, None, rows(), None, None, 0, 0, n, N, None, 0, None) == -6
    assert b"2^40" in l.tt_last_error()
