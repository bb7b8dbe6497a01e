"""Host side of the operators at a language model's way in: refusals of the C ABI before anything touches a device, sizes of
workspaces, and pins of the plain implementations that the kernels are tested against."""

import ctypes as C

import numpy as np
import pytest
import torch

import lm_util as R
from paper_2101_11714_amd import binding as B

F32, BF16, F16, E4M3 = 0, 1, 2, 3


def rows(data=64, ld=16, type=F32):
    return C.byref(B.TTRows(data, ld, type))


def toks(data=64, L=5, bits=64):
    return C.byref(B.TTTokens(data, L, bits))


def drop(state=64, site=0, p=0.5):
    return C.byref(B.TTDropout(state, site, p))


def test_struct_layouts_match_the_header():
    assert C.sizeof(B.TTRows) == 24 and B.TTRows.ld.offset == 8 and B.TTRows.type.offset == 16
    assert C.sizeof(B.TTTokens) == 24 and B.TTTokens.L.offset == 8 and B.TTTokens.bits.offset == 16
    assert C.sizeof(B.TTDropout) == 16 and B.TTDropout.site.offset == 8 and B.TTDropout.p.offset == 12


# (no call here may reach a launch: each is refused, or has nothing to do)
def test_token_calls_check_their_arguments():
    l = B.lib()
    good = lambda **k: (k.get("table", rows()), k.get("num_rows", 10), k.get("N", 16), k.get("tokens", toks()), 1.0, k.get("drop"), k.get("out", rows()), None)  # noqa: E731
    for code, k in [(-1, dict(tokens=None)), (-1, dict(tokens=toks(data=None))), (-3, dict(tokens=toks(L=-1))), (-3, dict(tokens=toks(bits=16))), (-6, dict(tokens=toks(L=2**31))),
                    (-3, dict(tokens=toks(data=60))), (-1, dict(table=None)), (-1, dict(table=rows(data=None))), (-6, dict(table=rows(type=E4M3))), (-6, dict(table=rows(type=9))),
                    (-3, dict(table=rows(data=66))), (-3, dict(table=rows(ld=-1))), (-6, dict(table=rows(ld=2**31 + 1))), (-3, dict(num_rows=-1)), (-6, dict(num_rows=2**31)), (-3, dict(N=-1)),
                    (-6, dict(N=2**20 + 1, out=rows(ld=2**21))), (-1, dict(out=None)), (-3, dict(out=rows(ld=15))), (-3, dict(out=rows(ld=0))), (-1, dict(drop=drop(state=None))),
                    (-3, dict(drop=drop(state=60))), (-3, dict(drop=drop(p=-0.1))), (-3, dict(drop=drop(p=1.1))), (-3, dict(drop=drop(p=float("nan"))))]:
        assert l.tt_token_fwd(*good(**k)) == code, k
        assert len(l.tt_last_error()) > 0
    assert l.tt_token_fwd(*good(tokens=toks(data=None, L=0))) == 0
    assert l.tt_token_fwd(*good(N=0)) == 0
    assert l.tt_token_bwd_workspace_bytes(5, 10, 16) == 0      # few tokens need none
    need = l.tt_token_bwd_workspace_bytes(2000, 10, 16)
    assert need > 0
    for f, tail in ((l.tt_token_bwd, (0,)), (l.tt_token_bwd_sgd, (0.1,))):
        args = lambda **k: (k.get("tokens", toks(L=2000)), k.get("grad", rows()), 1.0, k.get("drop"), k.get("table", rows()), k.get("num_rows", 10), k.get("N", 16), *tail,  # noqa: E731
                            k.get("ws", 256), k.get("bytes", need), None)
        for code, k in [(-1, dict(tokens=None)), (-6, dict(tokens=toks(L=2**28))), (-1, dict(grad=None)), (-6, dict(grad=rows(type=E4M3))), (-3, dict(table=rows(ld=0))), (-1, dict(table=None)),
                        (-3, dict(num_rows=-1)), (-6, dict(N=2**20 + 1, table=rows(ld=2**21))), (-4, dict(ws=None)), (-4, dict(bytes=need - 1)), (-3, dict(ws=8)), (-1, dict(drop=drop(state=None)))]:
            assert f(*args(**k)) == code, k
        assert f(*args(num_rows=0)) == 0
    assert l.tt_token_bwd(toks(data=None, L=0), rows(), 1.0, None, rows(), 10, 16, 1, None, 0, None) == 0


def test_dropout_calls_check_their_arguments():
    l = B.lib()
    for code, args in [(-1, (None, None, drop(), rows(), 5, 16, None)), (-1, (rows(), None, None, rows(), 5, 16, None)), (-1, (rows(), None, drop(), None, 5, 16, None)),
                       (-6, (rows(), None, drop(), rows(type=BF16), 5, 16, None)), (-6, (rows(), rows(type=F16), drop(), rows(), 5, 16, None)), (-3, (rows(), None, drop(), rows(), -5, 16, None)),
                       (-3, (rows(), None, drop(p=2.0), rows(), 5, 16, None)), (-3, (rows(), rows(data=65), drop(), rows(), 5, 16, None)), (-3, (rows(), None, drop(), rows(ld=8), 5, 16, None)),
                       (0, (rows(), None, drop(), rows(), 0, 16, None)), (0, (rows(), None, drop(), rows(), 5, 0, None))]:
        assert l.tt_dropout_fwd(*args) == code
        if args[1] is None:
            assert l.tt_dropout_bwd(args[0], *args[2:]) == code


def test_norm_calls_check_their_arguments():
    l = B.lib()
    fwd = lambda **k: (k.get("x", rows()), k.get("res"), k.get("drop"), k.get("w"), k.get("wt", F32), k.get("eps", 1e-6), k.get("sum"), k.get("out", rows()), k.get("rstd"),  # noqa: E731
                       k.get("scales"), k.get("group", 0), k.get("rows", 5), k.get("N", 16), None)
    for code, k in [(-1, dict(x=None)), (-1, dict(out=None)), (-6, dict(x=rows(type=E4M3))), (-6, dict(out=rows(type=BF16))), (-6, dict(res=rows(type=BF16))), (-6, dict(x=rows(type=BF16), out=rows(type=BF16), res=rows(type=F16))),
                    (-6, dict(sum=rows(type=F16))), (-6, dict(res=rows(), sum=rows(type=BF16))), (-3, dict(eps=-1.0)), (-3, dict(eps=float("nan"))), (-6, dict(N=32769, out=rows(ld=40000))), (-3, dict(N=0)), (-3, dict(rows=-1)),
                    (-6, dict(w=64, wt=E4M3)), (-3, dict(w=66)), (-3, dict(rstd=66)), (-3, dict(scales=rows())), (-3, dict(group=128)), (-1, dict(out=rows(type=E4M3))),
                    (-6, dict(out=rows(type=E4M3), scales=rows(ld=1), group=16)), (-6, dict(out=rows(type=E4M3), scales=rows(ld=1, type=BF16))), (-3, dict(out=rows(type=E4M3), scales=rows(ld=0))),
                    (-1, dict(drop=drop(state=None))), (-6, dict(N=16000, out=rows(ld=16000), rows=2**30))]:
        assert l.tt_add_rms_norm_fwd(*fwd(**k)) == code, k
    assert l.tt_add_rms_norm_fwd(*fwd(rows=0)) == 0
    assert l.tt_add_rms_norm_bwd_workspace_bytes(5, 16) == 0      # few rows need none
    need = l.tt_add_rms_norm_bwd_workspace_bytes(5000, 16)
    bwd = lambda **k: (k.get("dy", rows()), k.get("h", rows()), k.get("rstd", 64), k.get("w"), k.get("wt", F32), k.get("ds"), k.get("drop"), k.get("dx", rows()), k.get("dr"),  # noqa: E731
                       k.get("dw", 64), k.get("dwt", F32), 0, k.get("rows", 5000), k.get("N", 16), k.get("ws", 256), k.get("bytes", need), None)
    for code, k in [(-1, dict(dy=None)), (-1, dict(h=None)), (-1, dict(rstd=None)), (-6, dict(h=rows(type=BF16))), (-6, dict(ds=rows(type=BF16))), (-6, dict(dr=rows(type=F16))), (-6, dict(dx=rows(type=F16))),
                    (-6, dict(dw=64, dwt=E4M3)), (-4, dict(ws=None)), (-4, dict(bytes=need - 4)), (-3, dict(ws=24)), (-3, dict(rstd=65)), (-6, dict(N=32769, dx=rows(ld=40000))), (-1, dict(drop=drop(state=None)))]:
        assert l.tt_add_rms_norm_bwd(*bwd(**k)) == code, k
    assert l.tt_add_rms_norm_bwd(*bwd(dx=None, dw=None)) == 0
    assert l.tt_add_rms_norm_bwd(*bwd(rows=0, dw=None)) == 0


def test_workspaces_are_enough_for_shorter_calls():
    l = B.lib()
    lengths = [1, 2, 2047, 2048, 2049, 16_383, 16_384, 16_385, 65_536, 131_072, 131_073, 1_000_000, 2**28 - 1]
    for N in (1, 7, 64, 4096):
        sizes = [l.tt_token_bwd_workspace_bytes(L, 1000, N) for L in lengths]
        assert sizes[0] == 0 and sizes[-1] > 0 and sizes == sorted(sizes), (N, sizes)
        sizes = [l.tt_add_rms_norm_bwd_workspace_bytes(L, N) for L in lengths]
        assert sizes[0] == 0 and sizes[-1] > 0 and sizes == sorted(sizes), (N, sizes)
    assert l.tt_token_bwd_workspace_bytes(2**28, 10, 8) == 0 and l.tt_token_bwd_workspace_bytes(0, 10, 8) == 0 and l.tt_token_bwd_workspace_bytes(8, 10, 2**20 + 1) == 0
    assert l.tt_token_bwd_workspace_bytes(8, 2**31, 8) == 0 and l.tt_token_bwd_workspace_bytes(8, 0, 8) == 0
    assert l.tt_add_rms_norm_bwd_workspace_bytes(8, 32769) == 0


# ---- the plain implementations -------------------------------------------------------------------------------------------


def test_generator_gives_the_published_words():
    # the known answers of the generator's authors for 4 x 32 bits and ten rounds
    ff = 0xFFFFFFFF
    assert R.philox(0, 0, 0, 0) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert R.philox(ff << 32 | ff, ff, ff, ff << 32 | ff) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert R.philox(0x85a308d3243f6a88, 0x13198a2e, 0x03707344, 0x299f31d0a4093822) == [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]
    many = R.philox_blocks(2**32 - 2, 4, 9, 12, 0x123456789ABCDEF)
    assert [list(map(int, w)) for w in many] == [R.philox(2**32 - 2 + i, 9, 12, 0x123456789ABCDEF) for i in range(4)]


def test_mask_follows_the_words():
    state = np.array([0x123456789ABCDEF, 7])
    keep, factor = R.keep_mask(5, 19, 0.3, state, 2)
    q = 19661                                               # 0.3 * 65536 = 19660.8
    assert abs(factor * (65536 - q) - 65536) < 1e-9
    for r in range(5):
        for c in range(19):
            word = R.philox(r * 3 + c // 8, 2, 7, 0x123456789ABCDEF)[(c % 8) // 2]
            assert keep[r, c] == (((word >> 16) if c % 2 else (word & 0xFFFF)) >= q)


def test_plain_gradients_are_autograd_s():
    g = torch.Generator().manual_seed(1)
    d = (0.25, torch.tensor([5, 6]), 1)
    x, r, w = (torch.randn(s, generator=g, dtype=torch.float64, requires_grad=True) for s in ((6, 21), (6, 21), (21,)))
    G, S = torch.randn((6, 21), generator=g, dtype=torch.float64), torch.randn((6, 21), generator=g, dtype=torch.float64)
    keep, factor = R.keep_mask(6, 21, 0.25, d[1].numpy(), 1)
    h = r + x * torch.from_numpy(keep) * factor
    rstd = (h.square().mean(1) + 1e-4).rsqrt()
    y = h * rstd[:, None] * w
    ((y * G).sum() + (h * S).sum()).backward()
    ph, prstd, py, _ = R.norm_fwd(x, r, w, 1e-4, d)
    assert np.allclose(ph, h.detach()) and np.allclose(py, y.detach()) and np.allclose(prstd, rstd.detach())
    dx, dres, dw, _, _ = R.norm_bwd(G, h, rstd, w, S, d)
    assert np.allclose(dx, x.grad) and np.allclose(dres, r.grad) and np.allclose(dw, w.grad)
    table = torch.randn((9, 21), generator=g, dtype=torch.float64, requires_grad=True)
    tokens = torch.tensor([3, 3, -1, 8, 9, 0])
    there = (tokens >= 0) & (tokens < 9)
    out = torch.where(there[:, None], table[tokens.clamp(0, 8)] * 1.5, 0) * torch.from_numpy(keep) * factor
    (out * G).sum().backward()
    assert np.allclose(R.token_fwd(table, tokens, 1.5, d), out.detach())
    assert np.allclose(R.token_bwd(tokens, G, 9, 1.5, d)[0], table.grad)


@pytest.mark.parametrize("p,q", [(0.0, 0), (2.0 ** -18, 0), (2.0 ** -16, 1), (0.5, 32768), (1.0, 65536)])
def test_shares_are_rounded_to_16_bits(p, q):
    _, factor = R.keep_mask(1, 8, p, np.array([1, 2]), 0)
    assert factor == (65536.0 / (65536 - q) if q < 65536 else 0.0)
