"""Gradients of log probabilities under masks of a type's lowest value, and scales at the end of their range, against the formulas in 64 bits.

Bounds.  A sum of V exponentials is off by at most (24 + V, up to 4,096 additions in a row) 2^-24 of itself, an exponential by 2^-24 of itself for each unit of its argument
(the argument is rounded up to four times), and a log probability by that of the sum and of its own size."""

import math

import numpy as np
import pytest
import torch

from lm_util import U32, UNIT, TINY, assert_within, f64, rows_of
from paper_2101_11714_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
DEV = "cuda:0"


def gen(seed):
    return torch.Generator().manual_seed(seed)


class Rows:
    """Of rows of logits in 64 bits, from each row's own maximum: log p, p, lse, entropy; 0 for p where a row has nothing."""

    def __init__(self, x, scale):
        d = f64(x)
        self.raw, self.scale = d, scale
        self.V = d.shape[1]
        top = d.max(1)
        self.none = top == -np.inf
        m = np.where(self.none, 0, top)[:, None]
        with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
            z = (d - m) * scale
            log_s = np.log(np.exp(z).sum(1))
            self.log_p = np.where(self.none[:, None], -np.inf, z - log_s[:, None])
        self.p = np.exp(self.log_p)
        self.size = np.where(self.p > 0, np.abs(np.where(self.p > 0, self.log_p, 0)), 0)
        self.entropy = (self.p * self.size).sum(1)
        self.lse = np.where(self.none, -np.inf, m[:, 0] * scale + log_s)

    def sum_bound(self):
        return U32 * (40 + min(self.V, 4096))

    def lse_bound(self):
        """Of an lse that is stored, where it is one of less than 2^12 in size: beyond that the row's own sum stands for it."""
        size = np.abs(np.where(np.abs(self.lse) <= 4200, self.lse, 0))
        return self.sum_bound() + U32 * 2 * size

    def entropy_bound(self):
        return self.sum_bound() * (70 + math.log(self.V + 1))

    def gradient(self, tokens, g, ge):
        """(gradient, how far it may be off before its last rounding)"""
        rows = self.raw.shape[0]
        t = tokens.cpu().numpy().reshape(-1).astype(np.int64)
        there = (t >= 0) & (t < self.V)
        gg = np.where(there, f64(g), 0)[:, None]
        hot = np.zeros_like(self.p)
        hot[np.nonzero(there)[0], t[there]] = 1
        b, h = f64(ge)[:, None], self.entropy[:, None]
        neg = np.where(self.p > 0, -self.size, 0)
        want = gg * (hot - self.p) - b * self.p * (neg + h)
        rel = self.lse_bound()[:, None] + U32 * (4 * self.size + 16)
        off = np.abs(gg) * (self.p * rel + 4 * U32 * (hot + self.p)) + np.abs(b) * self.p * ((self.size + h) * (rel + 8 * U32) + self.lse_bound()[:, None] + self.entropy_bound())
        dead = (self.raw == -np.inf) | self.none[:, None]
        # (exponentials below 2^-126 may be cut to 0: times |ge| (|log p| + entropy), up to 2^4 2^8)
        return np.where(dead, 0, want) * self.scale, (np.where(dead, 0, off) * 1.01 + 2.0 ** -114) * self.scale


def run(x, tokens, g, ge, scale, in_place, lse=None):
    """The gradient, with what the forward pass leaves (or with another lse)."""
    rows = x.shape[0]
    lp, own, ent = (torch.empty(rows, device=DEV) for _ in range(3))
    B.tt_token_logprob_fwd(x, tokens, lp, own, entropy=ent, scale=scale)
    out = x if in_place else torch.empty_like(x)
    B.tt_token_logprob_bwd(x, tokens, own if lse is None else lse, g, out, entropy=ent, grad_entropy=ge, scale=scale)
    return out, lp, own, ent


# rows, V: one piece of a row and many, whole vectors and odd ones, one column
SIZES = [(1, 2), (3, 7), (9, 64), (33, 100), (8, 4097), (8, 8192), (8, 50257), (300, 1001)]


@pytest.mark.parametrize("rows,V", SIZES)
@pytest.mark.parametrize("type", TYPES)
def test_columns_of_the_lowest_value_have_no_gradient_of_the_entropy(rows, V, type):
    gr = gen(rows + V)
    for scale, in_place, lead in [(1.0, False, 0), (1.3, True, 0), (1.3, False, 3), (0.7, False, 1)]:
        scale = float(np.float32(scale))
        x = rows_of(gr, rows, V, type, lead, 0, 2.5)
        mask = torch.rand((rows, V), generator=gr) < 0.4
        mask[:, V // 2] = False                              # (no row of nothing else)
        x.masked_fill_(mask.to(DEV), torch.finfo(type).min)
        tokens = torch.randint(-1, V, (rows,), generator=gr).to(DEV)
        g, ge = (torch.randn(rows, generator=gr).to(DEV) * 4 for _ in range(2))
        want, off = Rows(x, scale).gradient(tokens, g, ge)
        got, _, _, _ = run(x, tokens, g, ge, scale, in_place)
        assert_within(got, want, off + UNIT[type] * (np.abs(want) + off) + TINY[type], (scale, in_place))


def special_rows(gr, V, type):
    """Rows whose lse has lost the logarithm of the sum, or is no finite number, and others between them."""
    low, high = torch.finfo(type).min, torch.finfo(type).max
    x = torch.randn((11, V), generator=gr) * 2
    x[0] = low
    x[1] = low
    x[1, ::2] = -math.inf
    x[1, -1] = low
    x[2] = low
    x[2, V // 3] = low / 2
    x[3] += 30000.0                                          # (values as the type holds them)
    x[4] = high
    x[5] = -math.inf
    x[7] = -math.inf
    x[7, V // 2] = low
    x[8] = -x[3]
    x[9] = high
    x[9, V // 2:] = low
    return x.to(type).to(DEV)


@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 4097, 8192, 50257])
@pytest.mark.parametrize("type", TYPES)
def test_rows_of_the_lowest_value_have_even_probabilities(V, type):
    gr = gen(V)
    for scale, in_place in [(1.0, False), (1.3, False), (1.3, True), (0.7, True), (100.0, False)]:
        scale = float(np.float32(scale))
        x = special_rows(gr, V, type)
        rows = x.shape[0]
        tokens = torch.randint(0, V, (rows,), generator=gr).to(DEV)
        tokens[0] = 0
        g, ge = (torch.randn(rows, generator=gr).to(DEV) * 4 for _ in range(2))
        r = Rows(x, scale)
        want, off = r.gradient(tokens, g, ge)
        got, _, lse, ent = run(x, tokens, g, ge, scale, in_place)
        assert_within(got, want, off + UNIT[type] * (np.abs(want) + off) + TINY[type], (scale, in_place))
        assert (np.abs(f64(ent) - r.entropy) <= r.entropy_bound()).all()


@pytest.mark.parametrize("type", TYPES)
def test_many_rows_of_the_lowest_value(type):
    # as in a padded batch: half of the rows, each beside another one's pieces
    gr, rows, V = gen(1), 400, 9001
    x = rows_of(gr, rows, V, type, 0, 0, 2.0)
    x[::2] = torch.finfo(type).min
    x[::8] = -math.inf
    tokens = torch.randint(0, V, (rows,), generator=gr).to(DEV)
    g, ge = (torch.randn(rows, generator=gr).to(DEV) for _ in range(2))
    want, off = Rows(x, 1.0).gradient(tokens, g, ge)
    first, _, _, _ = run(x, tokens, g, ge, 1.0, False)
    got, _, _, _ = run(x, tokens, g, ge, 1.0, True)
    assert_within(got, want, off + UNIT[type] * (np.abs(want) + off) + TINY[type], "in place")
    assert torch.equal(first, got)


def test_an_lse_of_more_columns_than_the_row_has_is_taken_as_it_is():
    # halves of a vocabulary: p = exp(z - lse) with the lse of both
    gr, rows, V = gen(2), 12, 3001
    for offset, scale in [(0.0, 1.0), (20000.0, 1.0), (-30000.0, 1.3)]:
        scale = float(np.float32(scale))
        x = (torch.randn((rows, 2 * V), generator=gr) * 2 + offset).to(DEV)
        tokens = torch.randint(0, V, (rows,), generator=gr).to(DEV)
        g, ge = torch.randn(rows, generator=gr).to(DEV), torch.zeros(rows, device=DEV)
        whole = Rows(x, scale)
        lse = torch.from_numpy(whole.lse).float().to(DEV)
        out, _, _, _ = run(x[:, :V].contiguous(), tokens, g, ge, scale, False, lse)
        want, off = whole.gradient(tokens, g, ge)
        want, off = want[:, :V], off[:, :V]
        # (what the lse has lost as it is stored, and as much again for the product that it is taken from)
        off = off + 2 * U32 * np.abs(whole.lse)[:, None] * np.abs(f64(g))[:, None] * whole.p[:, :V] * scale * 1.01
        assert_within(out, want, off + UNIT[F32] * (np.abs(want) + off), offset)


@pytest.mark.parametrize("scale", [1e-36, 1e-30, 1e-20, 1e30])
@pytest.mark.parametrize("top", [0, 5])
def test_scales_at_the_ends_of_their_range(scale, top):
    # logits as far apart as that takes to tell them from each other
    gr, scale = gen(3), float(np.float32(scale))
    for rows, V, wide in [(3, 5, 3), (2, 1000, 3), (2, 20001, 3), (2, 20001, 0.5)]:
        x = torch.randn((rows, V), generator=gr).double() * wide / scale
        x = x.clamp(-3e38, 3e38).float().to(DEV)
        tokens = torch.randint(0, V, (rows,), generator=gr).to(DEV)
        lp, lse, ent = (torch.empty(rows, device=DEV) for _ in range(3))
        ids = torch.empty((rows, top), dtype=torch.int64, device=DEV) if top else None
        B.tt_token_logprob_fwd(x, tokens, lp, lse, entropy=ent, scale=scale, top_ids=ids)
        r = Rows(x, scale)
        for got, want, by in ((lse, r.lse, r.lse_bound()), (lp, r.log_p[np.arange(rows), tokens.cpu().numpy()], r.sum_bound()), (ent, r.entropy, r.entropy_bound())):
            assert_within(got, want, by + 8 * U32 * np.abs(want), (rows, V))


@pytest.mark.parametrize("V", [5, 1000, 9001])
def test_an_infinite_lse_that_is_not_the_row_s_is_taken_as_it_is(V):
    # +inf: no column has a probability; -inf: no gradient
    gr, rows = gen(V), 6
    x = (torch.randn((rows, V), generator=gr) * 2).to(DEV)
    x[3:] += 30000.0
    tokens = torch.randint(0, V, (rows,), generator=gr).to(DEV)
    g, ge = torch.randn(rows, generator=gr).to(DEV), torch.ones(rows, device=DEV)
    for value in (math.inf, -math.inf):
        out, _, _, _ = run(x, tokens, g, ge, 1.5, False, torch.full((rows,), value, device=DEV))
        want = torch.zeros_like(x)
        if value > 0:
            want[torch.arange(rows, device=DEV), tokens] = g * 1.5
        assert torch.equal(out, want), value
