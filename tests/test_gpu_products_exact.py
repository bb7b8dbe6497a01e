"""Products of small whole numbers, whose sums 32 bits hold exactly: a piece of an operand that lands in another place of a tile than its own, or a step that is
read before it has landed, shows as another number.  Then the bound that an epilogue holds around such sums."""

import numpy as np
import pytest
import torch

import products_util as P
from lm_util import TINY, UNIT, f64
from paper_2101_11714_amd import binding as B
from test_gpu_products import output_bound

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DEV = "cuda:0"

# tiles of 256 and of 128, in whole and in parts, edges in every direction; rows that are copied first; few rows
SIZES = [(512, 512, 512), (256, 64, 256), (1024, 4096, 256), (2048, 1024, 2048), (300, 1096, 328), (129, 8192, 72), (4096, 640, 4096), (515, 1003, 777), (64, 4096, 1000), (16, 2048, 4096)]


def whole_numbers(g, rows, N, type, most=3):
    return torch.randint(-most, most + 1, (rows, N), generator=g).to(type).to(DEV)


@pytest.mark.parametrize("rows,K,N", SIZES)
@pytest.mark.parametrize("type", [F32, BF16, F16])
def test_products_of_whole_numbers_are_exact(rows, K, N, type):
    for seed in range(3):
        g = torch.Generator().manual_seed(100 * seed + rows)
        x, w, dy = whole_numbers(g, rows, K, type), whole_numbers(g, N, K, type), whole_numbers(g, rows, N, type)
        y, dx, dw, db = (torch.full(s, 7.5, dtype=t, device=DEV) for s, t in (((rows, N), F32), ((rows, K), type), ((N, K), F32), ((N,), F32)))
        B.tt_linear_fwd(x, w, y)
        B.tt_linear_bwd(dy, x, w, dx, dw, grad_bias=db)
        a, b, c = x.double(), w.double(), dy.double()
        assert torch.equal(y.double(), a @ b.t()), seed
        assert torch.equal(dx, (c @ b).to(type)), seed
        assert torch.equal(dw.double(), c.t().contiguous() @ a), seed
        assert torch.equal(db.double(), c.sum(0)), seed


@pytest.mark.parametrize("kind", P.ACTS)
@pytest.mark.parametrize("type", [F32, BF16, F16])
def test_epilogues_hold_their_bound(kind, type):
    g = torch.Generator().manual_seed(7)
    for rows, K, N, out in [(300, 264, 136, type), (40, 96, 520, F32), (1000, 64, 1000, type)]:
        x, w = whole_numbers(g, rows, K, type), whole_numbers(g, N, K, type) / 64
        bias = (torch.randn(N, generator=g) * 0.3).to(DEV)
        y = torch.empty((rows, N), dtype=out, device=DEV)
        B.tt_linear_fwd(x, w, y, bias=bias, activation=kind)
        want, z, mag = P.linear_fwd(x, w, bias, kind, None)
        off = output_bound(want, z, mag, K, UNIT[out], TINY[out])
        assert (np.abs(f64(y) - want) <= off).all(), (rows, K, N)
