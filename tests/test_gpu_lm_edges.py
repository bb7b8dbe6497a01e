"""Edges of the operators at a language model's way in: exact quotients and ties in 8 bits, values that are not finite, arrays at the
limits of a launch, and each rule's branches on both of its sides.  Plain implementations and bounds as in test_gpu_lm.py."""

import numpy as np
import pytest
import torch

import lm_util as R
from lm_util import U32
from paper_2101_11714_amd import binding as B
from test_gpu_lm import BF16, E4M3, F16, F32, assert_guard, check_grad, dropout_of, gen, room, tokens_of

pytestmark = pytest.mark.gpu


# ---- 8 bits -------------------------------------------------------------------------------------------------------------


def in_8_bits(y, group):
    """(values, scales) of rows y of 32 bits: scales max |y| / 448, values y / scale to the nearest even e4m3, both quotients rounded
    to 32 bits, on the host."""
    y = y.cpu()
    rows, N = y.shape
    width = group or N
    parts = [y[:, c:c + width] for c in range(0, N, width)]
    scales = torch.stack([p.abs().amax(1) / torch.tensor(448.0) for p in parts], 1)
    q = torch.cat([(p / s[:, None]).to(E4M3) for p, s in zip(parts, scales.unbind(1))], 1)
    return q, scales


def assert_same_8_bits(x, w, group, eps):
    rows, N = x.shape
    y = torch.empty_like(x)
    q, scales = torch.empty_like(x, dtype=E4M3), torch.empty((rows, -(-N // group) if group else 1), device="cuda:0")
    B.tt_add_rms_norm_fwd(x, w, y, eps=eps)
    B.tt_add_rms_norm_fwd(x, w, q, scales=scales, group=group, eps=eps)
    want_q, want_s = in_8_bits(y, group)
    assert np.array_equal(scales.cpu().numpy(), want_s.numpy(), equal_nan=True)
    q, number = q.cpu(), ~torch.isnan(want_q.float())
    assert torch.equal(~torch.isnan(q.float()), number)
    assert torch.equal(q.view(torch.uint8)[number], want_q.view(torch.uint8)[number])     # (zeros with their signs)


@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -60, 2.0 ** -75])
def test_ties_in_8_bits_go_to_the_even_value(group, size):
    # With eps = 2^100 the mean square vanishes: y = 2^-50 x exactly.  Row c holds (times `size`) whole multiples of c, 448 c the largest in each group:
    # its scale is 2^-50 c and its quotients are the multiples, among them every value of e4m3 and every midpoint of two neighbours.
    vals = torch.arange(0, 127, dtype=torch.uint8).view(E4M3).float()
    points = torch.cat([vals, (vals[1:] + vals[:-1]) / 2])
    points = torch.cat([points, -points, torch.zeros(-2 * points.numel() % 31)]).view(-1, 31)
    row = torch.cat([torch.full((points.shape[0], 1), 448.0), points], 1).reshape(-1)      # (448 leads every 32 columns)
    c = torch.arange(1, 4097, 2).float()
    x = (c[:, None] * row * size).to("cuda:0")
    assert_same_8_bits(x, None, group, 2.0 ** 100)


@pytest.mark.parametrize("rows,N", [(300, 512), (37, 1001), (5, 8192), (1000, 40)])
@pytest.mark.parametrize("group", [0, 64])
def test_quotients_in_8_bits_are_rounded_once(rows, N, group):
    g = gen(rows + N)
    assert_same_8_bits(R.rows_of(g, rows, N, F32), torch.randn(N, generator=g).to("cuda:0"), group, 1e-6)


def test_quotients_in_8_bits_by_scales_that_are_not_finite():
    # y is infinite in a column of rows 0 and 1, NaN in all of row 2
    x = torch.randn((4, 128), generator=gen(3)).to("cuda:0")
    w = torch.ones(128, device="cuda:0")
    w[5], x[:, 5] = 3e38, 1e3
    x[0, 5], x[1, 5], x[2, 9] = 2.0 ** 60, -2.0 ** 60, float("nan")
    for group in (0, 32):
        assert_same_8_bits(x, w, group, 2.0 ** 100)


# ---- more rows than a launch takes along one dimension --------------------------------------------------------------------


def need(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip("%d GiB of free memory are needed" % gib)


def pieces(rows, n=1 << 26):
    return [slice(r, min(r + n, rows)) for r in range(0, rows, n)]


def test_dropout_of_2_to_the_32_vectors():
    # rows of three vectors of eight columns, in place; ones become 0 or 2
    need(60)
    rows, N = (1 << 32) // 3 + 1000, 17
    x = torch.ones((rows, N), dtype=BF16, device="cuda:0")
    d = dropout_of(0.5)
    B.tt_dropout_fwd(x, x, d)
    kept = 0
    for p in pieces(rows):
        zero, two = x[p] == 0, x[p] == 2
        assert bool((zero ^ two).all())
        kept += int(two.sum())
    assert abs(kept / (rows * N) - 0.5) < 6 * 0.5 / (rows * N) ** 0.5
    seed, step = (int(v) for v in d.state.cpu())
    for first in (0, (1 << 30) + 5, (1 << 32) // 3 - 50, rows - 100):   # (every vector is a block of the generator)
        words = R.philox_blocks(3 * first, 300, d.site, step, seed)
        draws = np.stack([words & 0xFFFF, words >> 16], 2).reshape(100, 24)[:, :N]
        assert np.array_equal(x[first:first + 100].float().cpu().numpy(), 2.0 * (draws >= 32768))


def test_lookup_of_2_to_the_33_vectors():
    need(140)
    rows, N, vocab = (1 << 33) // 5 + 1000, 33, 1021
    tokens = (torch.arange(rows, dtype=torch.int32, device="cuda:0") % 1024).sub_(2)         # (-1, 1021 and their like are none)
    table = R.rows_of(gen(5), vocab, N, BF16)
    out = torch.empty((rows, N), dtype=BF16, device="cuda:0")
    B.tt_token_fwd(table, tokens, out)
    padded = torch.cat([torch.zeros((2, N), dtype=BF16, device="cuda:0"), table, torch.zeros((1, N), dtype=BF16, device="cuda:0")])
    whole = padded.repeat(1 << 14, 1)
    for p in pieces(rows, whole.shape[0]):
        assert torch.equal(out[p], whole[:out[p].shape[0]])


@pytest.mark.parametrize("bits8", [False, True])
def test_norm_of_2_to_the_32_threads(bits8):
    # four threads a row; all rows are one and the same
    need(70)
    rows, N = (1 << 30) + 1000, 17
    row, w = R.rows_of(gen(6), 1, N, BF16), torch.randn(N, generator=gen(7)).to("cuda:0")
    first = torch.empty((1, N), dtype=E4M3 if bits8 else BF16, device="cuda:0")
    one = torch.empty((1, 1), device="cuda:0") if bits8 else None
    B.tt_add_rms_norm_fwd(row, w, first, scales=one)
    out = torch.zeros((rows, N), dtype=first.dtype, device="cuda:0")
    scales = torch.zeros((rows, 1), device="cuda:0") if bits8 else None
    B.tt_add_rms_norm_fwd(row.expand(rows, N), w, out, scales=scales)
    as_bits = torch.uint8 if bits8 else torch.int16
    for p in pieces(rows):
        assert bool((out[p].view(as_bits) == first.view(as_bits)).all())
        assert scales is None or bool((scales[p] == one).all())


# ---- refusals and values that are not finite -------------------------------------------------------------------------------


def test_norm_refuses_an_empty_array_for_its_roots():
    x = torch.ones((5, 16), device="cuda:0")
    with pytest.raises(AssertionError):
        B.tt_add_rms_norm_fwd(x, None, torch.empty_like(x), rstd=torch.empty(0, device="cuda:0"))
    B.tt_add_rms_norm_fwd(x[:0], None, x[:0].clone(), rstd=torch.empty(0, device="cuda:0"))


@pytest.mark.parametrize("L", [6, 140_000])
@pytest.mark.parametrize("scale", [float("inf"), float("nan"), -float("inf")])
def test_rows_of_no_token_are_zero_under_any_scale(L, scale):
    table = torch.ones((9, 64), device="cuda:0")
    tokens = tokens_of(gen(8), L, 9, "some")
    none = (tokens < 0) | (tokens >= 9)
    for t in (table, table[:0]):
        out = torch.full((L, 64), 7.0, device="cuda:0")
        B.tt_token_fwd(t, tokens, out, scale=scale)
        zero = none if t.shape[0] else torch.ones_like(none)
        assert bool((out[zero] == 0).all()) and not torch.isfinite(out[~zero]).any()


# ---- both sides of each rule ---------------------------------------------------------------------------------------------


@pytest.mark.parametrize("L", [1025, 3000, 8192, 8193])
@pytest.mark.parametrize("vocab", [1 << 18, (1 << 18) + 1, (1 << 18) + 77, (1 << 20) + 5])
def test_token_bwd_of_rows_whose_marks_another_kernel_clears(L, vocab):
    # the sort of one workgroup (up to 8,192 tokens) clears the bytes of 2^18 rows itself, that of several 2^20
    N, g = 3, gen(L + vocab)
    tokens, grad = tokens_of(g, L, vocab, "some"), R.rows_of(g, L, N, F32)
    tokens[:3] = torch.tensor([0, vocab - 1, vocab - 17])
    dirty = torch.full((B.token_bwd_workspace_bytes(L, vocab, N),), 255, dtype=torch.uint8, device="cuda:0")
    out, flat = room(vocab, N, F32, 1, 0)
    B.tt_token_bwd(tokens, grad, out, workspace=dirty)
    want, mag, most = R.token_bwd(tokens, grad, vocab, 1.0, None)
    R.assert_within(out, want, (most + 4) * U32 * mag)
    assert_guard(out, flat)


@pytest.mark.parametrize("L", [5, 60])
@pytest.mark.parametrize("N", [2048, 2056, 4100, 8200])
@pytest.mark.parametrize("kind", ["some", "one", "none"])
def test_token_bwd_without_a_sort_into_rows_of_several_pieces(L, N, kind):
    check_grad(L, 300, N, kind, F32, F32, torch.int64, 0.2, 1, 1, "write")
    check_grad(L, 300, N, kind, BF16, F16, torch.int32, None, 0, 0, "write")


@pytest.mark.parametrize("L,N,s,o", [(9_000, 1001, F16, BF16), (9_001, 1001, BF16, F32), (35_000, 1024, F32, BF16), (70_001, 1001, BF16, F32), (66_000, 1024, F16, F32),
                                     (140_000, 1003, F32, F16), (132_000, 1024, BF16, BF16)])
def test_large_lookups(L, N, s, o):
    # two vectors a thread, between types, odd widths, dropout: against lookups of few rows and dropout on its own
    g = gen(L + N)
    table, tokens = R.rows_of(g, 500, N, s, 3, 1), tokens_of(g, L, 500, "some")
    out, flat = room(L, N, o, 3, 1)
    B.tt_token_fwd(table, tokens, out, scale=1.5)
    assert_guard(out, flat)
    wide = torch.empty((L, N), device="cuda:0")
    for p in pieces(L, 1000):
        few = torch.empty((out[p].shape[0], N), dtype=o, device="cuda:0")
        assert torch.equal(B.tt_token_fwd(table, tokens[p], few, scale=1.5), out[p])
        B.tt_token_fwd(table, tokens[p], wide[p])
    d = dropout_of(0.25)
    B.tt_token_fwd(table, tokens, out, dropout=d)
    assert torch.equal(out, B.tt_dropout_fwd(wide, wide, d).to(o))
    assert_guard(out, flat)


@pytest.mark.parametrize("N", [777, 12001, 16400, 20001, 32768])
@pytest.mark.parametrize("T,H", [(BF16, BF16), (F16, F32), (F32, F32)])
def test_norm_gradients_in_place(N, T, H):
    g, rows = gen(N), 530
    dy, h, ds = R.rows_of(g, rows, N, T, 1, 1), R.rows_of(g, rows, N, H, 0, 0, 2.0), R.rows_of(g, rows, N, H, 3, 0)
    rstd, w, d = (h.double().square().mean(1) + 1e-6).rsqrt().float(), torch.randn(N, generator=g).to("cuda:0"), dropout_of(0.4)
    gx, gr, gw, same = torch.empty_like(dy), torch.empty_like(ds), torch.empty(N, device="cuda:0"), torch.empty(N, device="cuda:0")
    B.tt_add_rms_norm_bwd(dy, h, rstd, w, gx, gw, grad_sum=ds, grad_residual=gr, dropout=d)
    B.tt_add_rms_norm_bwd(dy, h, rstd, w, dy, same, grad_sum=ds, grad_residual=ds, dropout=d)
    assert torch.equal(dy, gx) and torch.equal(ds, gr) and torch.equal(same, gw)


@pytest.mark.parametrize("N", [777, 12001, 16400, 20001, 32768])
def test_norms_in_place(N):
    g, rows = gen(N), 530
    x, r, w = R.rows_of(g, rows, N, F16, 1, 1), R.rows_of(g, rows, N, F32, 3, 0), torch.randn(N, generator=g).to("cuda:0")
    out, hs = torch.empty_like(x), torch.empty_like(r)
    B.tt_add_rms_norm_fwd(x, w, out, residual=r, sum_out=hs)
    B.tt_add_rms_norm_fwd(x, w, x, residual=r, sum_out=r)
    assert torch.equal(x, out) and torch.equal(r, hs)


@pytest.mark.parametrize("E,N", [(16, 39_000), (32, 22_000), (64, 10_800)])
def test_token_bwd_of_runs_from_every_place_of_a_tile(E, N):
    # one run after the other of a length that is prime to E: their starts pass through every place of a tile of E sorted positions
    lengths = [E + 1] * E + [2 * E + 1] * E + [3] * E + [1] * E
    vocab, L = len(lengths), sum(lengths)
    vectors = L * -(-N // 8)
    assert {16: 1 << 22, 32: 1 << 23, 64: 1 << 24}[E] <= vectors < {16: 1 << 23, 32: 1 << 24, 64: 1 << 60}[E]     # (what the rule takes tiles of E for)
    tokens = torch.repeat_interleave(torch.arange(vocab), torch.tensor(lengths))[torch.randperm(L, generator=gen(E))].to("cuda:0")
    grad = torch.randn((L, N), generator=torch.Generator(device="cuda:0").manual_seed(3), device="cuda:0")
    out = torch.empty((vocab, N), device="cuda:0")
    B.tt_token_bwd(tokens, grad, out)
    zeros = lambda: torch.zeros((vocab, N), dtype=torch.float64, device="cuda:0")  # noqa: E731
    want, mag = zeros().index_add_(0, tokens, grad.double()), zeros().index_add_(0, tokens, grad.abs().double())
    assert bool(((out.double() - want).abs() <= (max(lengths) + 6) * U32 * mag).all())
