"""Plain implementations in 64 bits of the operators at a language model's way in, written from their formulas, and the bounds
that the tests hold the kernels to.  Everything here runs on the host."""

from __future__ import annotations

import numpy as np
import torch

# unit roundoffs: half the spacing of neighbouring values over their size
U32 = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half the spacing of the smallest values (below the normal range)
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def philox(block, site, step, seed, rounds=10):
    """Philox4x32: the four words of one block, in whole numbers of any length."""
    m = 0xFFFFFFFF
    c = [block & m, (block >> 32) & m, site & m, step & m]
    k = [seed & m, (seed >> 32) & m]
    for _ in range(rounds):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & m, (a >> 32) ^ c[3] ^ k[1], a & m]
        k = [(k[0] + 0x9E3779B9) & m, (k[1] + 0xBB67AE85) & m]
    return c


def philox_blocks(first, count, site, step, seed):
    """The same for blocks first .. first + count - 1, [count, 4]."""
    m, h = np.uint64(0xFFFFFFFF), np.uint64(32)
    b = np.arange(first, first + count, dtype=np.uint64)
    c = [b & m, b >> h, np.full(count, site, np.uint64), np.full(count, step & 0xFFFFFFFF, np.uint64)]
    k = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        x, y = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(y >> h) ^ c[1] ^ np.uint64(k[0]), y & m, (x >> h) ^ c[3] ^ np.uint64(k[1]), x & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1).astype(np.uint32)


def keep_mask(rows, N, p, state, site):
    """(kept [rows, N], factor)."""
    q = int(np.floor(float(np.float32(p)) * 65536 + 0.5))
    per = -(-N // 8)
    words = philox_blocks(0, rows * per, site, int(state[1]), int(state[0]) & 0xFFFFFFFFFFFFFFFF)
    draws = np.stack([words & 0xFFFF, words >> 16], 2).reshape(rows, per * 8)[:, :N]
    return draws >= q, 65536.0 / (65536 - q) if q < 65536 else 0.0


def drop(x, dropout):
    if dropout is None:
        return x
    p, state, site = dropout
    keep, factor = keep_mask(x.shape[0], x.shape[1], p, state.cpu().numpy(), site)
    with np.errstate(invalid="ignore"):
        return np.where(keep, x * factor, 0.0)


def f64(t):
    return t.detach().double().cpu().numpy()


def token_fwd(table, tokens, scale, dropout):
    tok = tokens.cpu().numpy().reshape(-1).astype(np.int64)
    there = (tok >= 0) & (tok < table.shape[0])
    rows = np.zeros((tok.size, table.shape[1]))
    t = f64(table)
    rows[there] = t[tok[there]]
    return drop(rows * scale, dropout)


def token_bwd(tokens, grad, num_rows, scale, dropout):
    """(gradient, sums of magnitudes, most terms of a row)."""
    tok = tokens.cpu().numpy().reshape(-1).astype(np.int64)
    there = (tok >= 0) & (tok < num_rows)
    g = drop(f64(grad), dropout) * scale
    out, mag = np.zeros((num_rows, g.shape[1])), np.zeros((num_rows, g.shape[1]))
    np.add.at(out, tok[there], g[there])
    np.add.at(mag, tok[there], np.abs(g[there]))
    most = int(np.bincount(tok[there]).max()) if there.any() else 0
    return out, mag, most


def norm_fwd(x, residual, weight, eps, dropout):
    """h, rstd, y, and the sum of the magnitudes that h is the sum of."""
    h = drop(f64(x), dropout)
    mag = np.abs(h)
    if residual is not None:
        h, mag = h + f64(residual), mag + np.abs(f64(residual))
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    w = np.ones(h.shape[1]) if weight is None else f64(weight).reshape(-1)
    return h, rstd, h * rstd[:, None] * w, mag


def norm_bwd(dy, h, rstd, weight, dsum, dropout):
    """dx, dresidual, dw and the magnitudes that bound their rounding: of dh, and of dw."""
    dy, h, r = f64(dy), f64(h), f64(rstd)[:, None]
    w = np.ones(h.shape[1]) if weight is None else f64(weight).reshape(-1)
    g = dy * w
    dh = r * (g - h * r ** 2 * (g * h).mean(1, keepdims=True))
    mag = np.abs(r * g) + np.abs(h) * r ** 3 * np.abs(g * h).mean(1, keepdims=True)
    if dsum is not None:
        dh, mag = dh + f64(dsum), mag + np.abs(f64(dsum))
    return drop(dh, dropout), dh, (dy * h * r).sum(0), mag, np.abs(dy * h * r).sum(0)


def assert_within(got, want, bound, what=""):
    got = f64(got).reshape(want.shape)
    assert np.isfinite(got).all(), what
    off = np.abs(got - want) - bound
    assert (off <= 0).all(), "%s: %d of %d values are off, the worst by %.3g more than %.3g (got %.9g, want %.9g)" % (
        what, int((off > 0).sum()), off.size, off.max(), np.broadcast_to(bound, off.shape).flat[off.argmax()], got.flat[off.argmax()], want.flat[off.argmax()])


def rows_of(gen, rows, N, dtype, lead=0, shift=0, size=1.0, device="cuda:0"):
    """[rows, N] normal values; the row stride is N + lead, and the first row starts `shift` elements into its allocation."""
    flat = torch.empty(shift + rows * (N + lead) + 8, dtype=dtype, device=device)
    flat.copy_(torch.randn(flat.numel(), generator=gen) * size)
    return torch.as_strided(flat, (rows, N), (N + lead, 1), shift)
