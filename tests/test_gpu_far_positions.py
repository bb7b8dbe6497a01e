"""Rotation by positions up to 2^52 in size: the angle's fraction of a turn against whole numbers of any length."""

import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from lm_util import U32, UNIT, TINY, f64
from paper_2101_11714_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DEV = "cuda:0"
TWO_PI = Fraction(2 * 31415926535897932384626433832795028841971693993751, 10**49)
# cosines and sines: the fraction of a turn to 2^-50, the series' rest and roundings in 32 bits
TURN = 6 * U32


def angle(position, freq):
    turns = Fraction(int(position)) * Fraction(float(freq)) / TWO_PI
    return float(turns - round(turns)) * 2 * math.pi


@pytest.mark.parametrize("type", [F32, BF16, F16])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("back", [False, True])
def test_the_farthest_positions_keep_their_angles(type, neighbours, back):
    positions = torch.tensor([2**52, 2**52 - 1, -(2**52), 2**51 + 12345, 3**32, 2**44 + 1, -(2**47) + 3, 10**15, 2**31 - 1, 1, 0], device=DEV)
    freqs = torch.tensor([1.0, 0.9999999, 0.7853982, 3.1415927, 1e-3, 0.1, 1e-7, 7.5], dtype=F32, device=DEV)
    rows, pairs = positions.numel(), freqs.numel()
    x = torch.randn((rows, 2, 2 * pairs + 3), generator=torch.Generator().manual_seed(1)).to(type).to(DEV)
    out = torch.empty_like(x)
    r = B.Rotation(positions, freqs, (pairs,), neighbours)
    if back:
        B.tt_qk_norm_rotate_bwd(x, None, None, None, out, None, r, norm=False)
    else:
        B.tt_qk_norm_rotate_fwd(x, None, out, None, r, norm=False)
    got, v = f64(out), f64(x)
    assert np.array_equal(got[:, :, 2 * pairs:], v[:, :, 2 * pairs:])
    for i in range(rows):
        for j in range(pairs):
            a = angle(positions[i], freqs[j]) * (-1 if back else 1)
            p, q = (2 * j, 2 * j + 1) if neighbours else (j, pairs + j)
            size = np.abs(v[i, :, p]) + np.abs(v[i, :, q])
            for c, want in ((p, v[i, :, p] * math.cos(a) - v[i, :, q] * math.sin(a)), (q, v[i, :, q] * math.cos(a) + v[i, :, p] * math.sin(a))):
                off = (TURN + 2 * U32) * size
                assert (np.abs(got[i, :, c] - want) <= off + UNIT[type] * (np.abs(want) + off) + TINY[type]).all(), (int(positions[i]), float(freqs[j]), c)


def test_several_axes_of_far_positions():
    positions = torch.tensor([[2**52 - 5, 3, 2**50 + 1], [7, 2**51 + 9, -(2**52)]], device=DEV)
    freqs = torch.tensor([1.0, 0.3, 0.01, 0.6, 0.02], dtype=F32, device=DEV)
    x = torch.randn((3, 1, 10), generator=torch.Generator().manual_seed(2)).to(DEV)
    out = torch.empty_like(x)
    B.tt_qk_norm_rotate_fwd(x, None, out, None, B.Rotation(positions, freqs, (3, 2)), norm=False)
    got, v = f64(out), f64(x)
    for i in range(3):
        for j in range(5):
            a = angle(positions[int(j >= 3), i], freqs[j])
            size = np.abs(v[i, 0, j]) + np.abs(v[i, 0, 5 + j])
            assert abs(got[i, 0, j] - (v[i, 0, j] * math.cos(a) - v[i, 0, 5 + j] * math.sin(a))) <= (TURN + 4 * U32) * size, (i, j)
