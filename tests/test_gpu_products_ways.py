"""Every way that a product or a row of logits can go (products_util.py has the formulas): few rows by one kernel or by tiles, tiles of either size, parts of
the sums, operands that are copied first, pieces of a row; workspaces of exactly the size asked for, far positions in memory, graphs that share a workspace.

Bounds as in test_gpu_products.py: a sum of n products is off by at most 2 n 2^-24 of the sum of their magnitudes, and rounded once."""

import numpy as np
import pytest
import torch

import products_util as P
from lm_util import U32, UNIT, TINY, assert_within, f64, rows_of
from paper_2101_11714_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
DEV = "cuda:0"


def gen(seed):
    return torch.Generator().manual_seed(seed)


class Sums:
    """On the device in 64 bits: a matrix product and the sum of its terms' magnitudes."""

    def __init__(self, a, b):
        a, b = a.double(), b.double()
        self.want, self.mag = (a @ b).cpu().numpy(), (a.abs() @ b.abs()).cpu().numpy()

    def hold(self, got, n, what, add=None):
        want = self.want if add is None else self.want + f64(add)
        off = 2 * (n + 4) * U32 * self.mag + (0 if add is None else U32 * np.abs(f64(add)))
        t = got.dtype
        assert_within(got, want, off + UNIT[t] * (np.abs(want) + off) + TINY[t], what)


def exact_room(size):
    """A workspace of `size` bytes of NaN, and what follows it."""
    size = int(size)
    mem = torch.full(((size + 255) // 256 * 256 + 1024,), 255, dtype=torch.uint8, device=DEV)
    return mem[:size] if size else None, mem[size:]


# rows, K, N: few rows over short and long sums, to narrow and wide outputs; large tiles alone and in parts, small ones; whole chunks and odd rows
WAYS = [(1, 512, 300), (1, 16384, 24), (16, 8192, 40), (17, 640, 9000), (32, 512, 8200), (33, 1000, 8192), (40, 64, 8200), (64, 8192, 72), (64, 8191, 72), (48, 4104, 130), (65, 8192, 64), (130, 5001, 70), (700, 2048, 520),
        (1500, 4096, 600), (260, 16384, 264), (2048, 512, 2048), (2049, 136, 2047), (4200, 64, 4200), (64, 20000, 16)]


@pytest.mark.parametrize("rows,K,N", WAYS)
@pytest.mark.parametrize("type", TYPES)
def test_products_of_every_way_in_exactly_their_workspaces(rows, K, N, type):
    g = gen(rows + K + N)
    for lead, shift in [(0, 0), (3, 1)] if K * N < 2 ** 22 else [(0, 0)]:
        x, w, dy = rows_of(g, rows, K, type, lead, shift), rows_of(g, N, K, type, 0, 0, K ** -0.5), rows_of(g, rows, N, type, lead, 0)
        whole = lead == 0 and shift == 0 and K % 8 == 0
        ws, behind = exact_room(B.linear_fwd_workspace_bytes(rows, K, N, type, whole))
        y = torch.empty((rows, N), dtype=type, device=DEV)
        B.tt_linear_fwd(x, w, y, workspace=ws)
        Sums(x, w.t()).hold(y, K, "out")
        assert bool((behind == 255).all())
        ws, behind = exact_room(B.linear_bwd_workspace_bytes(rows, K, N, type, whole=whole and N % 8 == 0))
        dx, dw, db = torch.empty((rows, K), dtype=type, device=DEV), rows_of(g, N, K, F32), torch.empty(N, device=DEV)
        dw0 = dw.clone()
        B.tt_linear_bwd(dy, x, w, dx, None, workspace=ws)
        Sums(dy, w).hold(dx, N, "x alone")
        dx.zero_()
        db0 = db.zero_().clone()
        B.tt_linear_bwd(dy, x, w, dx, dw, grad_bias=db, accumulate=True, workspace=ws)
        Sums(dy, w).hold(dx, N, "x")
        Sums(dy.t(), x).hold(dw, rows, "weight", dw0)
        Sums(torch.ones((1, rows), device=DEV), dy).hold(db[None], rows, "bias", db0[None])
        assert bool((behind == 255).all())


def test_one_operand_is_copied_and_the_other_is_not():
    g = gen(1)
    for x_ways, w_ways in [((0, 0), (4, 0)), ((5, 3), (0, 0)), ((0, 8), (8, 0)), ((0, 4), (0, 0))]:
        x, w, dy = rows_of(g, 200, 96, BF16, *x_ways), rows_of(g, 72, 96, BF16, *w_ways), rows_of(g, 200, 72, BF16)
        y, dx, dw = torch.empty((200, 72), device=DEV), torch.empty((200, 96), dtype=BF16, device=DEV), torch.empty((72, 96), device=DEV)
        B.tt_linear_fwd(x, w, y)
        Sums(x, w.t()).hold(y, 96, "out")
        B.tt_linear_bwd(dy, x, w, dx, dw)
        Sums(dy, w).hold(dx, 72, "x")
        Sums(dy.t(), x).hold(dw, 200, "weight")


@pytest.mark.parametrize("type", TYPES)
def test_a_row_that_repeats_stands_for_many(type):
    # (a stride of 0: nothing follows the row in memory)
    g = gen(2)
    for rows, K, N in [(20, 70, 33), (100, 129, 65), (300, 64, 72), (5, 3, 2)]:
        one, w, dy = rows_of(g, 1, K, type)[:, :K].clone().expand(rows, K), rows_of(g, 1, K, type).clone().expand(N, K), rows_of(g, 1, N, type).clone().expand(rows, N)
        y, dx, dw = torch.empty((rows, N), dtype=type, device=DEV), torch.empty((rows, K), dtype=type, device=DEV), torch.empty((N, K), device=DEV)
        B.tt_linear_fwd(one, w, y)
        Sums(one, w.t()).hold(y, K, "out")
        B.tt_linear_bwd(dy, one, w, dx, dw)
        Sums(dy, w).hold(dx, N, "x")
        Sums(dy.t(), one).hold(dw, rows, "weight")


@pytest.mark.parametrize("type,ld", [(BF16, 2 ** 22), (BF16, 2 ** 22 + 8), (F16, 2 ** 22 - 1), (F32, 2 ** 21 + 1)])
def test_rows_far_apart(type, ld):
    # places behind 4 GB, from one row to the next by strides that a tile's offsets can or cannot bear
    g, rows, K, N = gen(3), 700, 40, 24
    mem = torch.empty((rows - 1) * ld + K, dtype=type, device=DEV)
    x = torch.as_strided(mem, (rows, K), (ld, 1))
    x.copy_(rows_of(g, rows, K, type))
    w, dy = rows_of(g, N, K, type), rows_of(g, rows, N, type)
    y, dw = torch.empty((rows, N), dtype=type, device=DEV), torch.empty((N, K), device=DEV)
    B.tt_linear_fwd(x, w, y)
    Sums(x, w.t()).hold(y, K, "out")
    B.tt_linear_bwd(dy, x, None, None, dw)
    Sums(dy.t(), x).hold(dw, rows, "weight")
    few = torch.as_strided(mem, (9, K), (64 * ld, 1))
    out = torch.empty((9, N), dtype=type, device=DEV)
    B.tt_linear_fwd(few, w, out)
    Sums(few, w.t()).hold(out, K, "few")
    B.tt_linear_bwd(dy, None, w, x, None)                    # and written there
    Sums(dy, w).hold(x, N, "x")


def test_what_is_behind_a_row_is_not_read():
    # NaN between the rows and behind the last one: in odd rows, in copies, in tiles that end there
    g = gen(4)
    for type in TYPES:
        for rows, K, N in [(3, 13, 5), (40, 100, 70), (129, 65, 130), (300, 1001, 33)]:
            def padded(r, c):
                mem = torch.full((r * (c + 5) + 64,), float("nan"), dtype=type, device=DEV)
                v = torch.as_strided(mem, (r, c), (c + 5, 1), 8)
                v.copy_(rows_of(g, r, c, type))
                return v
            x, w, dy, pre = padded(rows, K), padded(N, K), padded(rows, N), padded(rows, N)
            y, dx, dw, db = torch.empty((rows, N), dtype=type, device=DEV), torch.empty((rows, K), dtype=type, device=DEV), torch.empty((N, K), device=DEV), torch.empty(N, device=DEV)
            B.tt_linear_fwd(x, w, y)
            Sums(x, w.t()).hold(y, K, "out")
            B.tt_linear_bwd(dy, x, w, dx, dw, grad_bias=db)
            Sums(dy, w).hold(dx, N, "x")
            Sums(dy.t(), x).hold(dw, rows, "weight")
            B.tt_linear_bwd(dy, x, w, dx, dw, grad_bias=db, pre=pre, activation="silu")
            assert all(bool(t.isfinite().all()) for t in (dx, dw, db))


@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "silu"])
def test_activations_of_single_values(kind):
    """A product with 1 leaves z as it is.  The functions have relative errors of z^2 2^-24 from the exponential's argument, z log2(e) or z^2 log2(e) / 2, each rounded
    twice (the tanh's argument, up to 2 (|z| + 0.045 |z|^3), four times), and of 16 2^-24 from the rest."""
    z = torch.cat([torch.linspace(-5, 5, 20001), torch.linspace(-1e-3, 1e-3, 101), torch.tensor([0.0, 1e-30, -1e-30, 30.0, 1e4, 3e38])]).to(DEV)[:, None]
    y, dx = torch.empty_like(z), torch.empty_like(z)
    one = torch.ones((1, 1), device=DEV)
    B.tt_linear_fwd(z, one, y, activation=kind)
    x = f64(z)
    args = {"gelu": x ** 2, "silu": np.abs(x), "gelu_tanh": 4 * 2 * (np.abs(x) + 0.045 * np.abs(x) ** 3)}[kind]
    rel = (np.where(np.abs(x) < 10, args, 0) + 16) * U32
    want = P.act(x, kind)
    # (the oracle's own 1 + erf or 1 + tanh is off by 2^-53)
    assert_within(y, want, rel * np.abs(want) + np.abs(x) * 2.0 ** -50 + 2.0 ** -126, kind)
    B.tt_linear_bwd(torch.ones_like(z), None, one, dx, None, pre=z, activation=kind)
    want = P.slope(x, kind)
    # (two terms of at most 1.2, which can cancel)
    assert_within(dx, want, (np.where(np.abs(x) < 10, np.minimum(args, 30), 0) * np.minimum(1, np.exp(-np.abs(x)) * 30) + 16) * 1.2 * U32, kind)


def test_two_graphs_share_a_workspace():
    g = gen(5)
    x, w, dy = rows_of(g, 130, 2049, BF16, 1), rows_of(g, 200, 2049, BF16, 0, 0, 0.02), rows_of(g, 130, 200, BF16)
    logits, tokens = rows_of(g, 4, 100_000, F32), torch.tensor([0, 5, 99_999, 7], device=DEV)
    ws = torch.empty(32 << 20, dtype=torch.uint8, device=DEV)
    y, dx, dw, lp, lse, ids = (torch.empty(s, dtype=t, device=DEV) for s, t in (((130, 200), BF16), ((130, 2049), BF16), ((200, 2049), F32), (4, F32), (4, F32), ((4, 9), torch.int64)))

    def one():
        B.tt_linear_fwd(x, w, y, activation="gelu", workspace=ws)
        B.tt_token_logprob_fwd(logits, tokens, lp, lse, top_ids=ids, workspace=ws)

    def two():
        B.tt_linear_bwd(dy, x, w, dx, dw, workspace=ws)

    one(), two()
    want = [t.clone() for t in (y, lp, lse, ids, dx, dw)]
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for graph, call in zip(graphs, (one, two)):
        with torch.cuda.graph(graph):
            call()
    for i in range(5):
        for t in (y, lp, lse, ids, dx, dw):
            t.zero_()
        for graph in graphs if i % 2 else graphs[::-1]:
            graph.replay()
        if i == 3:
            one()                                            # and the program's own calls between them
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, lp, lse, ids, dx, dw))), i


# rows, V, k: pieces in numbers below and above a wave's 64, one alternative and many, more alternatives than logits
PIECES = [(1, 1_000_000, 1), (1, 300_000, 3), (1, 300_000, 64), (2, 131_072, 20), (7, 50_257, 5), (24, 131_072, 20), (24, 131_072, 64), (511, 9_000, 2), (3, 16_400, 17), (2, 12_289, 64)]


@pytest.mark.parametrize("rows,V,k", PIECES)
@pytest.mark.parametrize("kind", ["normal", "steps", "banned", "late", "few"])
def test_alternatives_of_pieces(rows, V, k, kind):
    g = gen(rows + V + k)
    x = torch.randn((rows, V), generator=g)
    if kind == "steps":
        x = (x * 2).round()                                  # many equal ones, ranked by their columns
    elif kind == "banned":
        x[torch.rand((rows, V), generator=g) < 0.9] = -float("inf")
    elif kind == "late":
        x[:, -100:] += 20                                    # all of them in one piece
    elif kind == "few":
        keep = torch.randint(0, V, (rows, max(k // 2, 1)), generator=g)
        x = torch.full((rows, V), -float("inf")).scatter_(1, keep, x[:, :keep.shape[1]])
    x = x.to(DEV)
    size = B.token_logprob_fwd_workspace_bytes(rows, V, k)
    ws, behind = exact_room(size)
    top, best, lse = torch.empty((rows, k), dtype=torch.int64, device=DEV), torch.empty((rows, k), device=DEV), torch.empty(rows, device=DEV)
    B.tt_token_logprob_fwd(x, None, None, lse, top_ids=top, top_logprobs=best, workspace=ws)
    _, wlse, _, wids, wbest = P.logprob_fwd(x, None, 1.0, k)
    assert np.array_equal(top.cpu().numpy(), wids)
    there = np.isfinite(wbest)
    got = f64(best)
    assert np.array_equal(np.isfinite(got), there)
    # the sum is off by 2^-24 for each of the additions in a row, of which a thread, a wave and the pieces have few hundred, and 16 for the exponentials' arguments
    assert (np.abs(got[there] - wbest[there]) <= 1000 * U32 + 4 * U32 * np.abs(wbest[there])).all()
    assert bool((behind == 255).all())


def test_the_way_out_of_the_example():
    from paper_2101_11714_amd import token_block
    vocab, L = 300, 96
    answer = token_block.Answer(vocab, L, seed=3)
    g = gen(6)
    N = answer.head.shape[1]
    y, following = rows_of(g, L, N, F32), torch.randint(0, vocab, (L,), generator=g).to(DEV)
    lp = answer.forward(y, following)
    x, head = y.double().cpu().requires_grad_(True), answer.head.double().cpu().requires_grad_(True)
    want = torch.log_softmax(x @ head.t(), 1)[torch.arange(L), following.cpu()]
    (-want.mean()).backward()
    # logits of N products of about 1 / sqrt(N) and 1 are off by less than 2 N 2^-24, probabilities by that of themselves, and so are the gradients' terms; sums of L or vocab
    off = 2 * (N + 40) * U32 * float((x.detach().abs() @ head.detach().abs().t()).max())
    assert (lp.double().cpu() - want.detach()).abs().max() <= 2 * off + 16 * U32
    g_y = answer.backward(y, following)
    p = torch.softmax(x.detach() @ head.detach().t(), 1)
    terms = (p + torch.nn.functional.one_hot(following.cpu(), vocab)) / L
    for got, ref, mag in ((g_y, x.grad, terms @ head.detach().abs()), (answer.g_head, head.grad, terms.t() @ x.detach().abs())):
        assert_within(got, ref.numpy(), (mag * (2 * off + 2 * (vocab + 30) * U32)).numpy(), "gradient")
    ids, best = answer.likeliest(y[:7], 5)
    ref = torch.log_softmax(x[:7].detach() @ head.detach().t(), 1)
    assert (best.double().cpu() - ref.gather(1, ids.cpu())).abs().max() <= 2 * off + 16 * U32
    assert (best[:, :-1] >= best[:, 1:]).all() and (ref.max(1).values - best[:, 0].double().cpu()).abs().max() <= 2 * off + 16 * U32
    block, first, last = token_block.train(steps=12, vocab=200, L=512, loss="likelihood")
    assert block.answer.logprob.isfinite().all() and block.answer.head.isfinite().all()
    with pytest.raises(ValueError):
        token_block.train(steps=1, loss="other")
