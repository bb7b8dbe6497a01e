"""More refusals of the C ABI for the products of a language model and what is done to their rows, before anything touches a device."""

import ctypes as C
import random

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


# A workspace of no bytes at an odd address: refused for its size where one is needed, else for its address; no call here reaches a launch.
def needed(call):
    l = B.lib()
    rc = call()
    text = l.tt_last_error().decode()
    if rc == -3:
        assert "aligned" in text, text
        return 0
    assert rc == -4, (rc, text)
    return int(text.split("workspace of ")[1].split(" bytes")[0])


def linear_needs(n, K, N, type, lead=0):
    l = B.lib()
    return needed(lambda: l.tt_linear_fwd(rows(ld=K + lead, type=type), rows(ld=K + lead, type=type), None, F32, 0, None, None, rows(ld=N, type=type), n, K, N, 8, 0, None))


def gradients_need(n, K, N, type, lead=0, act=0, x=True, w=True, b=True, w_type=F32):
    l = B.lib()
    return needed(lambda: l.tt_linear_bwd(rows(ld=N + lead, type=type), rows(ld=K + lead, type=type), rows(ld=K + lead, type=type), rows(ld=N, type=type), act, rows(ld=K, type=type) if x else None,
                                          rows(ld=K, type=w_type) if w else None, 64 if b else None, F32, 0, n, K, N, 8, 0, None))


def test_calls_ask_for_what_they_use():
    # one part, whole chunks, no activation: nothing goes through a workspace
    for type in (F32, BF16, F16):
        assert linear_needs(8192, 4096, 16384, type) == 0 and linear_needs(4096, 1024, 4096, type) == 0
        assert gradients_need(8192, 4096, 4096, type, b=False) == 0
    # an activation's gradient and the bands of the bias, and no more
    assert 2 * 8192 * 4096 <= gradients_need(8192, 4096, 4096, BF16, act=4) <= 2 * 8192 * 4096 + 4 * 256 * 4096 + 1024
    # copies of what is not whole
    assert 0 < linear_needs(4096, 1021, 4096, BF16) <= 2 * 2 * 4096 * 1024 + 1024
    # parts of a long sum
    assert linear_needs(100, 8192, 64, F32) >= 2 * 4 * 100 * 64


def test_what_a_query_says_is_enough_for_every_call():
    l = B.lib()
    rng = random.Random(5)
    for i in range(3000):
        size = lambda most: max(1, int(2 ** rng.uniform(0, most)) // rng.choice([1, 1, 8]) * rng.choice([1, 8]))  # noqa: E731
        n, K, N = size(15), size(15), size(15)
        type, act = rng.choice([F32, BF16, F16]), rng.choice([0, 4])
        lead = rng.choice([0, 0, 3, 8])
        most = n + rng.choice([0, 1, 100, 5000])
        whole = type != F32 and lead % 8 == 0 and K % 8 == 0
        if n * K * N:
            assert linear_needs(n, K, N, type, lead) <= l.tt_linear_fwd_workspace_bytes(most, K, N, type, int(whole)), (n, most, K, N, type, lead)
            x, w = rng.random() < 0.7, rng.random() < 0.7
            need = gradients_need(n, K, N, type, lead, act, x, w, rng.random() < 0.7)
            assert need <= l.tt_linear_bwd_workspace_bytes(most, K, N, type, act, int(whole and N % 8 == 0)), (n, most, K, N, type, lead, act, x, w)
