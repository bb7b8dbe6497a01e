"""Matrix product with its epilogue, norm and rotation of queries and keys and log probabilities of tokens against plain implementations in
64 bits (products_util.py).

Bounds.  A value is rounded once to its type (unit roundoff u) after sums in 32 bits.  A sum of n products is off by at most 2 n 2^-24 of the sum
of the products' magnitudes, whatever its order (the matrix cores cut off what they align, up to a whole step for each addition)."""

import math

import numpy as np
import pytest
import torch

import products_util as P
from lm_util import U32, UNIT, TINY, assert_within, f64, rows_of
from paper_2101_11714_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def room(rows, N, dtype, lead=0, shift=0):
    """Rows to write into, with a guard value before, between and behind them."""
    flat = torch.full((shift + rows * (N + lead) + 8,), 7.0, dtype=torch.float32, device="cuda:0").to(dtype)
    return torch.as_strided(flat, (rows, N), (N + lead, 1), shift), flat


def assert_guard(view, flat):
    m = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(m, view.shape, view.stride(), view.storage_offset()).fill_(False)
    assert bool((flat.float()[m] == 7.0).all())


def vector(g, n, dtype, mean=0.0):
    return (torch.randn(n, generator=g) * 0.3 + mean).to(dtype).to("cuda:0")


# ---- matrix product ---------------------------------------------------------------------------------------------------

# rows, K, N: one of everything, edges of tiles and of steps, few rows over a long sum, wide and narrow
PRODUCTS = [(1, 1, 1), (1, 7, 3), (2, 8, 8), (5, 33, 17), (16, 64, 64), (17, 65, 129), (31, 128, 100), (32, 256, 256), (33, 31, 8), (64, 64, 128), (100, 200, 300), (127, 96, 127), (128, 128, 128),
            (129, 129, 129), (257, 72, 40), (256, 512, 384), (3, 4096, 40), (1, 5000, 130), (300, 1000, 16), (40, 8, 1000), (513, 640, 257), (1025, 40, 520), (65, 96, 72), (200, 1096, 328), (3000, 264, 1400), (2056, 72, 3592)]


def output_bound(y, z, mag, n, u, tiny):
    """What an output may be off: its sum, an activation of slope up to 1.2 with a few roundings of its own, the last rounding."""
    return 1.2 * 2 * (n + 4) * U32 * mag + 16 * U32 * (np.abs(z) + np.abs(y)) + u * np.abs(y) + tiny + 1e-37


@pytest.mark.parametrize("rows,K,N", PRODUCTS)
@pytest.mark.parametrize("type", TYPES)
def test_linear_fwd(rows, K, N, type):
    g = gen(rows + K + N)
    for kind, bias, residual, pre, out, lead, shift in [("none", None, False, False, type, 0, 0), ("gelu_tanh", F32, False, True, type, 8, 0), ("silu", type, True, True, F32, 3, 1),
                                                        ("gelu", BF16, True, False, type, 1, 3), ("relu", F16, False, True, F32, 0, 0)]:
        x, w = rows_of(g, rows, K, type, lead, shift), rows_of(g, N, K, type, lead, 0, K ** -0.5)
        b = None if bias is None else vector(g, N, bias)
        r = rows_of(g, rows, N, out, lead, shift) if residual else None
        y, flat = room(rows, N, out, lead, shift)
        z, zflat = room(rows, N, type, lead) if pre else (None, None)
        assert B.tt_linear_fwd(x, w, y, bias=b, activation=kind, residual=r, pre=z) is y
        want, wz, mag = P.linear_fwd(x, w, b, kind, r)
        off = 1.2 * 2 * (K + 4) * U32 * mag + 16 * U32 * (np.abs(wz) + np.abs(want)) + (0 if r is None else U32 * np.abs(f64(r)))
        assert_within(y, want, off + UNIT[out] * (np.abs(want) + off) + TINY[out], (kind, "out"))
        assert_guard(y, flat)
        if pre:
            off = 2 * (K + 4) * U32 * mag
            assert_within(z, wz, off + UNIT[type] * (np.abs(wz) + off) + TINY[type], (kind, "pre"))
            assert_guard(z, zflat)


def test_linear_in_place_leading_dimensions_and_repeated_rows():
    g = gen(1)
    x, w = rows_of(g, 24, 48, BF16), rows_of(g, 40, 48, BF16, 0, 0, 0.1)
    r = rows_of(g, 24, 40, F32)
    want, z, mag = P.linear_fwd(x, w, None, "none", r)
    out = r.clone()
    B.tt_linear_fwd(x.view(2, 3, 4, 48), w, out.view(2, 3, 4, 40), residual=out.view(2, 3, 4, 40))
    assert_within(out, want, 2 * 52 * U32 * mag + 4 * U32 * np.abs(want), "in place")
    one = x[:1].expand(24, 48)                               # a row that repeats
    want, z, mag = P.linear_fwd(one, w, None, "none", None)
    out = torch.empty((24, 40), dtype=BF16, device="cuda:0")
    B.tt_linear_fwd(one, w, out)
    assert_within(out, want, 2 * 52 * U32 * mag + UNIT[BF16] * 1.01 * np.abs(want) + TINY[BF16], "repeated")
    same = w[:1].expand(40, 48)
    want, z, mag = P.linear_fwd(x, same, None, "none", None)
    B.tt_linear_fwd(x, same, out)
    assert_within(out, want, 2 * 52 * U32 * mag + UNIT[BF16] * 1.01 * np.abs(want) + TINY[BF16], "repeated weight")


def test_linear_without_columns_is_its_bias():
    b, r = vector(gen(2), 10, F32), vector(gen(3), 50, F32).view(5, 10)
    out = torch.empty((5, 10), device="cuda:0")
    B.tt_linear_fwd(torch.empty((5, 0), device="cuda:0"), torch.empty((10, 0), device="cuda:0"), out, bias=b, activation="relu", residual=r)
    assert torch.equal(out, b.relu() + r)


@pytest.mark.parametrize("rows,K,N", PRODUCTS)
@pytest.mark.parametrize("type", TYPES)
def test_linear_bwd(rows, K, N, type):
    g = gen(rows + K + N)
    for kind, wtype, btype, add, lead, shift in [("none", F32, F32, True, 0, 0), ("silu", type, type, False, 8, 0), ("gelu_tanh", type, F32, True, 3, 1), ("gelu", type, BF16, False, 0, 1), ("relu", F32, None, False, 1, 0),
                                                 ("none", type, F16, False, 16, 0)]:
        x, w = rows_of(g, rows, K, type, lead, shift), rows_of(g, N, K, type, lead, 0, K ** -0.5)
        dy, pre = rows_of(g, rows, N, type, lead, shift), rows_of(g, rows, N, type, lead)
        dx, fx = room(rows, K, type, lead, shift)
        dw, fw = room(N, K, wtype, lead, shift)
        db = None if btype is None else vector(g, N, btype)
        if add:
            dw.copy_(rows_of(g, N, K, wtype))
        w0, b0 = f64(dw) * add, 0 if db is None else f64(db) * add
        B.tt_linear_bwd(dy, x, w, dx, dw, grad_bias=db, pre=None if kind == "none" else pre, activation=kind, accumulate=add)
        wx, ww, wb, mx, mw, mb = P.linear_bwd(dy, x, w, pre, kind)
        # The gradient in front of an activation is rounded to its type.  The slope is a sum of up to two terms of at most 1.2 each, which near its
        # zero cancel: it is off by eight roundings of the terms, 10 2^-24 as such, however small it is, and its product with dy by one more.
        r = 0 if kind == "none" else UNIT[type] + 2 * U32
        tiny = 0 if kind == "none" else TINY[type]
        term = np.abs(f64(dy)) * (0 if kind in ("none", "relu") else 10 * U32) + tiny
        ax, aw, ab = term @ np.abs(f64(w)), term.T @ np.abs(f64(x)), term.sum(0)
        off = (2 * (N + 4) * U32 + r) * mx * 1.01 + ax
        assert_within(dx, wx, off + UNIT[type] * (np.abs(wx) + off) + TINY[type], (kind, "x"))
        off = (2 * (rows + 4) * U32 + r) * mw * 1.01 + aw + 2 * U32 * np.abs(w0)
        assert_within(dw, ww + w0, off + UNIT[wtype] * (np.abs(ww + w0) + off) + TINY[wtype], (kind, "weight"))
        if db is not None:
            off = (2 * (rows + 4) * U32 + 2 * U32) * mb + ab + 2 * U32 * np.abs(b0)
            assert_within(db, wb + b0, off + UNIT[btype] * (np.abs(wb + b0) + off) + TINY[btype], (kind, "bias"))
        assert_guard(dx, fx)
        assert_guard(dw, fw)


def test_linear_bwd_of_parts_and_of_nothing():
    g = gen(5)
    x, w, dy = rows_of(g, 50, 70, BF16), rows_of(g, 90, 70, BF16), rows_of(g, 50, 90, BF16)
    full = [torch.empty((50, 70), dtype=BF16, device="cuda:0"), torch.empty((90, 70), dtype=F32, device="cuda:0"), torch.empty(90, device="cuda:0")]
    B.tt_linear_bwd(dy, x, w, full[0], full[1], grad_bias=full[2])
    for want in range(3):
        got = [torch.empty_like(t) if i == want else None for i, t in enumerate(full)]
        B.tt_linear_bwd(dy, x if want == 1 else None, w if want == 0 else None, got[0], got[1], grad_bias=got[2])
        assert torch.equal(got[want], full[want])
    # no rows: gradients of nothing, or nothing to add
    empty = lambda n: torch.empty((0, n), dtype=BF16, device="cuda:0")  # noqa: E731
    B.tt_linear_bwd(empty(90), empty(70), w, empty(70), full[1], grad_bias=full[2], accumulate=True)
    assert full[1].any() and full[2].any()
    B.tt_linear_bwd(empty(90), empty(70), w, empty(70), full[1], grad_bias=full[2])
    assert not full[1].any() and not full[2].any()


def test_linear_gradients_are_differences():
    # sum of dy * y along a direction, from both sides, in 32 bits with steps that a quotient of differences bears
    g = gen(6)
    x, w, b = rows_of(g, 20, 36, F32), rows_of(g, 28, 36, F32, 0, 0, 0.2), vector(g, 28, F32)
    dy = rows_of(g, 20, 28, F32)
    for kind in ("silu", "gelu", "gelu_tanh"):
        pre, out = torch.empty((20, 28), device="cuda:0"), torch.empty((20, 28), device="cuda:0")
        value = lambda x, w, b: float((B.tt_linear_fwd(x, w, out, bias=b, activation=kind, pre=pre).double() * dy.double()).sum())  # noqa: E731
        value(x, w, b)
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
        B.tt_linear_bwd(dy, x, w, dx, dw, grad_bias=db, pre=pre.clone(), activation=kind)
        for i, (at, grad) in enumerate([(x, dx), (w, dw), (b, db)]):
            v = torch.randn(at.shape, generator=g).to("cuda:0")
            step = 2.0 ** -7
            args = [x, w, b]
            up, down = list(args), list(args)
            up[i], down[i] = at + step * v, at - step * v
            slope = (value(*up) - value(*down)) / (2 * step)
            want = float((grad.double() * v.double()).sum())
            size = float((grad.double().square() * v.double().square()).sum().sqrt())
            # third differences: step^2 / 6 times a third derivative, of the order of the terms themselves
            assert abs(slope - want) <= 100 * step ** 2 * size + 1e-3 * size, (kind, i, slope, want)


# ---- norm and rotation -------------------------------------------------------------------------------------------------

# rows, heads of q and k, D, rotated columns, sections of axes, neighbours
HEADS = [(1, 1, 1, 2, 2, (1,), False), (3, 2, 1, 6, 4, (2,), True), (5, 4, 2, 16, 16, (8,), False), (7, 3, 1, 17, 16, (3, 5), False), (9, 8, 2, 64, 64, (32,), True), (33, 4, 4, 80, 80, (8, 16, 16), False),
         (20, 5, 1, 72, 72, (12, 12, 12), True), (65, 16, 2, 128, 128, (64,), False), (130, 2, 2, 128, 32, (16,), False), (17, 1, 1, 256, 128, (24, 20, 20), True), (4, 2, 1, 512, 512, (256,), False),
         (6, 2, 1, 511, 500, (50, 0, 100, 100), False), (300, 3, 0, 40, 40, (20,), False), (11, 2, 2, 33, 0, (0,), False), (2, 40, 8, 96, 96, (0, 48), False), (1, 64, 8, 128, 128, (64,), True)]


def rotation_of(g, rows, rot, sections, neighbours, bits=torch.int64, far=1000):
    positions = torch.randint(-3, far, (len(sections), rows), generator=g).to(bits).to("cuda:0")
    freqs = (10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / max(rot, 1))).float().to("cuda:0")
    return B.Rotation(positions, freqs, sections, neighbours)


def heads_of(g, rows, heads, D, type, ways):
    """Heads as parts of wider rows."""
    lead, gap, shift = ways
    flat = torch.empty(shift + rows * (heads * (D + gap) + lead) + 8, dtype=type, device="cuda:0")
    flat.copy_(torch.randn(flat.numel(), generator=g))
    return torch.as_strided(flat, (rows, heads, D), (heads * (D + gap) + lead, D + gap, 1), shift)


# cosines and sines: the fraction of a turn from 64 bits, the series' rest and roundings in 32 bits
TURN = 6 * U32


@pytest.mark.parametrize("rows,hq,hk,D,rot,sections,neighbours", HEADS)
@pytest.mark.parametrize("type", TYPES)
def test_rotate_fwd(rows, hq, hk, D, rot, sections, neighbours, type):
    g = gen(rows + D)
    for norm, wtype, turned, ways, bits, in_place in [(True, type, True, (0, 0, 0), torch.int64, False), (False, None, True, (3, 1, 1), torch.int32, False), (True, None, False, (8, 0, 0), torch.int64, False),
                                                      (True, F32, True, (16, 8, 0), torch.int32, True)]:
        q = heads_of(g, rows, hq, D, type, ways)
        k = heads_of(g, rows, hk, D, type, ways) if hk else None
        r = rotation_of(g, rows, rot, sections, neighbours, bits) if turned else None
        wq, wk = (None if wtype is None else vector(g, D, wtype, 1.0) for _ in range(2))
        want = [P.rotate_fwd(q, wq, r, norm, 1e-5), P.rotate_fwd(k, wk, r, norm, 1e-5) if hk else None]
        qo, ko = (q, k) if in_place else (torch.empty_like(q), torch.empty_like(k) if hk else None)
        B.tt_qk_norm_rotate_fwd(q, k, qo, ko, r, norm=norm, q_weight=wq, k_weight=wk, eps=1e-5)
        for got, w in ((qo, want[0]), (ko, want[1])):
            if got is None:
                continue
            y, mag = w
            off = (TURN + (D + 12) * U32 * norm) * mag
            assert_within(got, y, off + UNIT[type] * (np.abs(y) + off) + TINY[type], (norm, turned))


@pytest.mark.parametrize("rows,hq,hk,D,rot,sections,neighbours", HEADS)
@pytest.mark.parametrize("type", TYPES)
def test_rotate_bwd(rows, hq, hk, D, rot, sections, neighbours, type):
    g = gen(rows + D)
    for norm, wtype, gtype, turned, ways, add, in_place in [(True, type, F32, True, (0, 0, 0), False, False), (False, None, None, True, (3, 1, 1), False, False), (True, None, BF16, False, (8, 0, 0), True, False),
                                                            (True, F32, F16, True, (1, 8, 3), False, True), (True, F32, None, True, (0, 0, 0), False, False)]:
        q = heads_of(g, rows, hq, D, type, ways)
        gq = heads_of(g, rows, hq, D, type, ways)
        k, gk = (heads_of(g, rows, hk, D, type, ways) for _ in range(2)) if hk else (None, None)
        r = rotation_of(g, rows, rot, sections, neighbours) if turned else None
        wq, wk = (None if wtype is None else vector(g, D, wtype, 1.0) for _ in range(2))
        dwq, dwk = (None if gtype is None else vector(g, D, gtype) for _ in range(2))
        before = [None if t is None else f64(t) * add for t in (dwq, dwk)]
        if not hk:
            dwk = None
        want = [P.rotate_bwd(gq, q, wq, r, norm, 1e-5), P.rotate_bwd(gk, k, wk, r, norm, 1e-5) if hk else None]
        dq, dk = (gq, gk) if in_place else (torch.empty_like(gq), torch.empty_like(gk) if hk else None)
        B.tt_qk_norm_rotate_bwd(gq, gk, q if norm else None, k if norm else None, dq, dk, r, norm=norm, q_weight=wq, k_weight=wk, grad_q_weight=dwq, grad_k_weight=dwk, eps=1e-5, accumulate=add)
        for got, dw, w, b, n in ((dq, dwq, want[0], before[0], rows * hq), (dk, dwk, want[1], before[1], rows * hk)):
            if got is None:
                continue
            dx, wdw, mx, mw = w
            off = (TURN + (2 * D + 24) * U32 * norm) * mx
            assert_within(got, dx, off + UNIT[type] * (np.abs(dx) + off) + TINY[type], (norm, turned, "x"))
            if dw is not None:
                off = (TURN + (n + D + 24) * U32) * mw + 2 * U32 * np.abs(b)
                assert_within(dw, wdw + b, off + UNIT[gtype] * (np.abs(wdw + b) + off) + TINY[gtype], (norm, turned, "weight"))


def test_far_positions():
    # angles of 10^9 turns: a product of 32 bits would have no digit of the angle left
    positions = torch.tensor([0, 1, 10**6, 2**31 - 1, 2**40 + 12345, -(2**40), 2**52 - 1], device="cuda:0")
    q = torch.randn((7, 2, 64), generator=gen(8)).to("cuda:0")
    freqs = torch.tensor([0.9 ** i for i in range(32)], dtype=torch.float32, device="cuda:0")
    out = torch.empty_like(q)
    r = B.Rotation(positions[:6], freqs, (32,))
    B.tt_qk_norm_rotate_fwd(q[:6], None, out[:6], None, r, norm=False)
    # in whole numbers: the angle's turns to 2^-60, from a rational pi
    from fractions import Fraction
    two_pi = Fraction(2 * 31415926535897932384626433832795028841971693993751, 10**49)
    x = f64(q)
    for i in range(6):
        for j in range(32):
            turns = Fraction(int(positions[i])) * Fraction(float(freqs[j])) / two_pi
            a = float(turns - round(turns)) * 2 * math.pi
            # the product with 1 / (2 pi) has three roundings of 53 bits before the fraction is taken
            off = 2 * math.pi * abs(float(turns)) * 2.0 ** -51 + TURN
            for c, want in ((j, x[i, :, j] * math.cos(a) - x[i, :, 32 + j] * math.sin(a)), (32 + j, x[i, :, 32 + j] * math.cos(a) + x[i, :, j] * math.sin(a))):
                size = np.abs(x[i, :, j]) + np.abs(x[i, :, 32 + j])
                assert (np.abs(f64(out)[i, :, c] - want) <= (off + 2 * U32) * size).all(), (i, j, c)


def test_rows_of_zeros_under_a_norm():
    q = torch.zeros((3, 2, 32), device="cuda:0")
    out, w = torch.empty_like(q), torch.ones(32, device="cuda:0")
    B.tt_qk_norm_rotate_fwd(q, None, out, None, None, q_weight=w, eps=1e-6)
    assert not out.any()
    g = torch.ones_like(q)
    dw = torch.empty(32, device="cuda:0")
    B.tt_qk_norm_rotate_bwd(g, None, q, None, out, None, None, q_weight=w, grad_q_weight=dw, eps=1e-6)
    assert torch.allclose(out, torch.full_like(out, 1000.0)) and not dw.any()


# ---- log probabilities ---------------------------------------------------------------------------------------------------

LOGITS = [(1, 1, 1), (1, 2, 2), (3, 7, 4), (2, 8, 8), (5, 9, 3), (4, 64, 64), (33, 100, 5), (7, 1000, 20), (600, 257, 1), (515, 4096, 0), (3, 4097, 32), (2, 50257, 20), (24, 32768, 20), (1, 131072, 64), (513, 1001, 7)]


def logits_of(g, rows, V, type, kind, lead=0, shift=0):
    x = rows_of(g, rows, V, type, lead, shift, 2.5)
    if kind == "banned":
        x.masked_fill_((torch.rand((rows, V), generator=g) < 0.4).to("cuda:0"), float("-inf"))
        x[rows // 2] = float("-inf")                         # a row of nothing
    elif kind == "least":                                    # masks of the type's lowest value
        x.masked_fill_((torch.rand((rows, V), generator=g) < 0.4).to("cuda:0"), torch.finfo(type).min)
        x[rows // 2] = torch.finfo(type).min
    elif kind == "equal":
        x.fill_(0.5)
    elif kind == "few":                                      # many ties
        x.copy_(torch.randint(-3, 3, (rows, V), generator=g).to(type).to("cuda:0"))
    return x


def logprob_bounds(x, scale, V):
    """(of lse and logprob, of the entropy): sums of V positive terms, each an exponential of a difference whose product with scale is rounded."""
    z = f64(x) * scale
    fine = np.isfinite(z)
    size = np.abs(np.where(fine & (z > -1e30), z, 0)).max(1) + 1
    return U32 * (4 * size + 24 + min(V, 4096)), U32 * (size + math.log(V + 1)) * (24 + min(V, 4096))


@pytest.mark.parametrize("rows,V,k", LOGITS)
@pytest.mark.parametrize("type", TYPES)
def test_logprob_fwd(rows, V, k, type):
    g = gen(rows + V)
    for kind, scale, ids, lead, shift in [("plain", 1.0, torch.int64, 0, 0), ("banned", 0.7, torch.int32, 3, 1), ("equal", 1.0, torch.int64, 0, 0), ("few", 1.3, torch.int64, 8, 0), ("least", 1.0, torch.int32, 1, 0)]:
        scale = float(np.float32(scale))                     # (what the call takes)
        x = logits_of(g, rows, V, type, kind, lead, shift)
        tokens = torch.randint(-2, V + 2, (rows,), generator=g).to(ids).to("cuda:0")
        lp, lse, ent = (torch.full((rows,), 7.0, device="cuda:0") for _ in range(3))
        top = torch.empty((rows, k), dtype=ids, device="cuda:0") if k else None
        best = torch.empty((rows, k), device="cuda:0") if k else None
        B.tt_token_logprob_fwd(x, tokens, lp, lse, entropy=ent, top_ids=top, top_logprobs=best, scale=scale)
        wlp, wlse, went, wids, wbest = P.logprob_fwd(x, tokens, scale, k)
        off, off_h = logprob_bounds(x, scale, V)
        for got, want, by in ((lp, wlp, off), (lse, wlse, off), (ent, went, off_h)):
            got = f64(got)
            big = np.isfinite(want) & (np.abs(want) > 1e30)
            assert np.array_equal(np.isinf(got) & ~big, np.isinf(want) & ~big), kind
            fine = np.isfinite(want) & ~big
            got, want = (np.where(np.isinf(t), 0, t) for t in (got, want))
            assert (np.abs(got - want)[fine] <= by[fine] + 2 * U32 * np.abs(want)[fine]).all(), (kind, np.abs(got - want)[fine].max())
            assert (np.abs(got - want)[big] <= 4 * U32 * np.abs(want)[big]).all()
        if k:
            assert np.array_equal(top.cpu().numpy(), wids), kind
            got = f64(best)
            assert np.array_equal(np.isinf(got), np.isinf(wbest))
            fine = np.isfinite(wbest)
            got, wbest = (np.where(np.isinf(t), 0, t) for t in (got, wbest))
            assert (np.abs(got - wbest)[fine] <= (off[:, None] + 4 * U32 * np.abs(np.where(fine, wbest, 0)))[fine]).all(), kind


def test_many_equal_logits_are_ranked_by_their_columns():
    # more candidates than a workgroup lists, wherever the larger ones lie
    V = 120_000
    for rows in (2, 600):
        x = torch.zeros((rows, V), dtype=BF16, device="cuda:0")
        x[0, 70_000:] = 1.0
        x[1, 5:119_000:7] = 2.0
        x[-1, -1] = 3.0
        lse = torch.empty(rows, device="cuda:0")
        top = torch.empty((rows, 64), dtype=torch.int64, device="cuda:0")
        B.tt_token_logprob_fwd(x, None, None, lse, top_ids=top)
        want = P.logprob_fwd(x[:2], None, 1.0, 64)[3]
        assert np.array_equal(top[:2].cpu().numpy(), want)
        if rows > 2:
            assert top[2].tolist() == list(range(64)) and top[-1].tolist() == [V - 1] + list(range(63))


def test_contiguous_peaks_and_rising_logits():
    # the largest logits all in one thread's places, or in the last ones that are looked at
    for V, make in [(40_000, lambda t: t), (40_000, lambda t: -t), (131_072, lambda t: (t % 4096 < 90).float() * t)]:
        x = make(torch.arange(V, dtype=torch.float32))[None].repeat(3, 1).to("cuda:0") / 1000
        top, lse = torch.empty((3, 64), dtype=torch.int32, device="cuda:0"), torch.empty(3, device="cuda:0")
        B.tt_token_logprob_fwd(x, None, None, lse, top_ids=top)
        assert np.array_equal(top.cpu().numpy(), P.logprob_fwd(x, None, 1.0, 64)[3])


def test_rows_that_are_not_finite():
    x = torch.zeros((5, 300), device="cuda:0")
    x[0, 17] = float("nan")
    x[1, 200] = float("inf")
    x[2, 5] = -float("nan")
    x[3] = float("-inf")
    tokens = torch.tensor([0, 200, 5, 3, 2], device="cuda:0")
    lp, lse, ent, best = torch.empty(5, device="cuda:0"), torch.empty(5, device="cuda:0"), torch.empty(5, device="cuda:0"), torch.empty((5, 3), device="cuda:0")
    ids = torch.empty((5, 3), dtype=torch.int64, device="cuda:0")
    B.tt_token_logprob_fwd(x, tokens, lp, lse, entropy=ent, top_ids=ids, top_logprobs=best)
    for t in (lp, lse, ent):
        assert t[:3].isnan().all() and not t[3:].isnan().any()
    assert ids[:, 0].tolist() == [17, 200, 5, -1, 0] and ids[3].tolist() == [-1] * 3 and best[:3].isnan().all()
    assert lse[3] == -math.inf and lp[3] == -math.inf and ent[3] == 0 and (best[3] == -math.inf).all()
    assert abs(float(ent[4]) - math.log(300)) < 1e-5
    out = torch.empty_like(x)
    one = torch.ones(5, device="cuda:0")
    B.tt_token_logprob_bwd(x, tokens, lse, one, out, entropy=ent, grad_entropy=one)
    assert not out[3].any() and out[4].isfinite().all() and out[0].isnan().any()


@pytest.mark.parametrize("rows,V,k", LOGITS)
@pytest.mark.parametrize("type", TYPES)
def test_logprob_bwd(rows, V, k, type):
    g = gen(rows + V)
    for kind, scale, ids, lead, shift, gl, ge, in_place in [("plain", 1.0, torch.int64, 0, 0, True, False, False), ("banned", 0.7, torch.int32, 3, 1, True, True, False), ("few", 1.3, torch.int64, 8, 0, False, True, True),
                                                            ("equal", 1.0, torch.int64, 0, 0, True, True, False)]:
        scale = float(np.float32(scale))                     # (what the call takes)
        x = logits_of(g, rows, V, type, kind, lead, shift)
        tokens = torch.randint(-2, V + 2, (rows,), generator=g).to(ids).to("cuda:0")
        _, wlse, went, _, _ = P.logprob_fwd(x, tokens, scale, 0)
        lse, ent = (torch.from_numpy(t).float().to("cuda:0") for t in (wlse, went))
        a, b = (vector(g, rows, F32) for _ in range(2))
        a, b = a if gl else None, b if ge else None
        want, mag, log_p = P.logprob_bwd(x, tokens, scale, lse, ent, a, b)
        out, flat = (x, None) if in_place else room(rows, V, type, lead, shift)
        B.tt_token_logprob_bwd(x, tokens if gl else None, lse, a, out, entropy=ent if ge else None, grad_entropy=b, scale=scale)
        # the exponential's argument is rounded twice; the magnitudes' other roundings
        off = mag * U32 * (4 * np.abs(log_p) + 16) + scale * (0 if b is None else np.abs(f64(b))[:, None] * U32 * 4 * np.exp(np.where(mag > 0, log_p, 0)) * (np.abs(log_p) + np.abs(f64(ent))[:, None]))
        # (exponentials below 2^-126 may be cut to 0)
        assert_within(out, want, off + UNIT[type] * (np.abs(want) + off) + TINY[type] + 2.0 ** -120, kind)
        if flat is not None:
            assert_guard(out, flat)


def test_logprob_gradient_is_a_difference():
    g = gen(9)
    x = rows_of(g, 6, 50, F32)
    tokens = torch.tensor([1, 4, -1, 49, 50, 0], device="cuda:0")
    a, b = vector(g, 6, F32), vector(g, 6, F32)
    lp, lse, ent = (torch.empty(6, device="cuda:0") for _ in range(3))

    def value(x):
        B.tt_token_logprob_fwd(x, tokens, lp, lse, entropy=ent, scale=1.5)
        return float((lp.double() * a.double() + ent.double() * b.double()).sum())

    value(x)
    out = torch.empty_like(x)
    B.tt_token_logprob_bwd(x, tokens, lse, a, out, entropy=ent, grad_entropy=b, scale=1.5)
    for _ in range(5):
        v = torch.randn(x.shape, generator=g).to("cuda:0")
        step = 2.0 ** -6
        slope = (value(x + step * v) - value(x - step * v)) / (2 * step)
        want = float((out.double() * v.double()).sum())
        # rounding: a few 2^-24 of values up to 10 over the step; third differences of the order of step^2
        assert abs(slope - want) <= 6 * 10 * 8 * U32 / step + 20 * step ** 2, (slope, want)


# ---- streams, graphs, workspaces, refusals -----------------------------------------------------------------------------------


def test_runs_are_bit_identical_and_other_streams_wait_for_nothing():
    g = gen(10)
    x, w, b = rows_of(g, 40, 4096, BF16), rows_of(g, 512, 4096, BF16, 0, 0, 0.02), vector(g, 512, F32)
    dy = rows_of(g, 40, 512, BF16)
    tokens = torch.randint(0, 512, (40,), generator=g).to("cuda:0")

    def run():
        y, dx, dw, db = torch.empty((40, 512), device="cuda:0"), torch.empty_like(x), torch.empty((512, 4096), device="cuda:0"), torch.empty(512, device="cuda:0")
        B.tt_linear_fwd(x, w, y, bias=b, activation="silu")
        B.tt_linear_bwd(dy, x, w, dx, dw, grad_bias=db)
        lp, lse, ent = (torch.empty(40, device="cuda:0") for _ in range(3))
        B.tt_token_logprob_fwd(y, tokens, lp, lse, entropy=ent)
        q = torch.empty((40, 4, 128), device="cuda:0")
        gq = torch.empty(128, device="cuda:0")
        B.tt_qk_norm_rotate_bwd(y.view(40, 4, 128), None, y.view(40, 4, 128), None, q, None, None, grad_q_weight=gq)
        return [y, dx, dw, db, lp, lse, ent, q, gq]

    first = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = run()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, second))


def test_a_captured_run_replays_on_new_inputs():
    """Product, norm and rotation, product, log probabilities and their gradients, as a model calls them, in one graph."""
    g = gen(11)
    rows, dim, heads, D, V = 48, 256, 4, 64, 1000
    dev = "cuda:0"
    w1, w2, table = (rows_of(g, n, dim, BF16, 0, 0, 0.06) for n in (2 * heads * D, dim, V))
    x = rows_of(g, rows, dim, BF16)
    tokens = torch.randint(0, V, (rows,), generator=g).to(dev)
    r = rotation_of(g, rows, D, (32,), False)
    wn = vector(g, D, F32, 1.0)
    e = lambda *s, t=BF16: torch.empty(s, dtype=t, device=dev)  # noqa: E731
    qk, qo, ko, hidden, pre, logits, lp, lse, ent = e(rows, 2 * heads * D), e(rows, heads, D), e(rows, heads, D), e(rows, dim), e(rows, dim), e(rows, V, t=F32), e(rows, t=F32), e(rows, t=F32), e(rows, t=F32)
    ids, glog, logits16, gh, gt, gq, gk, gwq, gwk, gx, gw1 = (e(rows, 5, t=torch.int64), e(rows, V), e(rows, V), e(rows, dim), e(V, dim, t=F32), e(rows, heads, D), e(rows, heads, D), e(D, t=F32), e(D, t=F32), e(rows, dim),
                                                              e(2 * heads * D, dim, t=F32))
    one = torch.ones(rows, device=dev)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device=dev)
    q, k = qk[:, :heads * D].view(rows, heads, D), qk[:, heads * D:].view(rows, heads, D)

    def step():
        B.tt_linear_fwd(x, w1, qk, workspace=ws)
        B.tt_qk_norm_rotate_fwd(q, k, qo, ko, r, q_weight=wn, k_weight=wn)
        B.tt_linear_fwd(qo.view(rows, dim), w2, hidden, activation="gelu", pre=pre, residual=x, workspace=ws)
        B.tt_linear_fwd(hidden, table, logits16, workspace=ws)
        B.tt_token_logprob_fwd(logits16, tokens, lp, lse, entropy=ent, top_ids=ids, workspace=ws)
        B.tt_token_logprob_bwd(logits16, tokens, lse, one, glog)
        B.tt_linear_bwd(glog, hidden, table, gh, gt, workspace=ws)
        B.tt_linear_bwd(gh, qo.view(rows, dim), w2, gx, None, pre=pre, activation="gelu", workspace=ws)
        B.tt_qk_norm_rotate_bwd(gx.view(rows, heads, D), ko, q, k, gq, gk, r, q_weight=wn, k_weight=wn, grad_q_weight=gwq, grad_k_weight=gwk, workspace=ws)
        B.tt_linear_bwd(gq.view(rows, dim), x, None, None, gw1[:heads * D], workspace=ws)

    outs = [qk, qo, ko, hidden, logits16, lp, lse, ent, ids, glog, gh, gt, gx, gq, gk, gwq, gwk]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.copy_(rows_of(g, rows, dim, BF16))
        tokens.copy_(torch.randint(-1, V, (rows,), generator=g).to(dev))
        step()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, t) for p, t in zip(want, outs)), i
    # against the formulas, end to end: a row's logprob from its logits as they were stored
    wlp = P.logprob_fwd(logits16, tokens, 1.0, 5)
    assert np.abs(f64(lp) - wlp[0]).max() < 1e-4 and np.array_equal(ids.cpu().numpy(), wlp[3])


def test_a_recorded_call_without_its_workspace_is_refused():
    x, w = torch.zeros((100, 4096), device="cuda:0"), torch.zeros((64, 4096), device="cuda:0")
    out = torch.empty((100, 64), device="cuda:0")
    assert B.linear_fwd_workspace_bytes(100, 4096, 64, F32) > 0
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(B.TTError) as e:
        with torch.cuda.graph(graph):
            B.tt_linear_fwd(x, w, out)
    assert e.value.code == -4
    B.tt_linear_fwd(x, w, out)                               # (and outside of it goes on)


def test_refusals_of_the_binding():
    e = lambda *s, t=F32: torch.zeros(s, dtype=t, device="cuda:0")  # noqa: E731
    for f in [lambda: B.tt_linear_fwd(e(4, 8), e(6, 9), e(4, 6)), lambda: B.tt_linear_fwd(e(4, 8), e(6, 8), e(4, 7)), lambda: B.tt_linear_fwd(e(4, 8), e(6, 8), e(4, 6), bias=e(7)),
              lambda: B.tt_linear_fwd(e(8, 4).t(), e(6, 8), e(4, 6)), lambda: B.tt_linear_fwd(torch.zeros(4, 8), e(6, 8), e(4, 6)), lambda: B.tt_linear_bwd(e(4, 6), e(4, 8), e(6, 8), e(4, 8), e(6, 9)),
              lambda: B.tt_linear_bwd(e(4, 6), e(5, 8), None, None, e(6, 8)), lambda: B.tt_qk_norm_rotate_fwd(e(4, 2, 8), e(4, 2, 6), e(4, 2, 8), e(4, 2, 6)),
              lambda: B.tt_qk_norm_rotate_fwd(e(4, 2, 8), None, e(4, 2, 8), None, (torch.zeros(5, dtype=torch.int64, device="cuda:0"), e(4), (4,), False)),
              lambda: B.tt_qk_norm_rotate_fwd(e(4, 2, 8), None, e(4, 2, 8), None, (torch.zeros(4, dtype=torch.int16, device="cuda:0"), e(4), (4,), False)),
              lambda: B.tt_token_logprob_fwd(e(4, 8), torch.zeros(3, dtype=torch.int64, device="cuda:0"), e(4)), lambda: B.tt_token_logprob_fwd(e(4, 8), None, None, e(3)),
              lambda: B.tt_token_logprob_fwd(e(4, 80), None, None, e(4), top_ids=torch.zeros((4, 65), dtype=torch.int64, device="cuda:0")), lambda: B.tt_token_logprob_bwd(e(4, 8), None, e(4), None, e(4, 9))]:
        with pytest.raises((AssertionError, B.TTError)):
            f()
    with pytest.raises(ValueError):
        B.tt_linear_fwd(e(4, 8), e(6, 8), e(4, 6), activation="swish")
    with pytest.raises(B.TTError):
        B.tt_linear_fwd(e(4, 8), e(6, 8, t=BF16), e(4, 6))
    with pytest.raises(B.TTError):
        B.tt_qk_norm_rotate_fwd(e(4, 2, 8), None, e(4, 2, 8), None, (torch.zeros(4, dtype=torch.int64, device="cuda:0"), e(5), (5,), False))
