"""Plain implementations in 64 bits of the products of a language model and of what is done to their rows, written from the formulas.
Everything here runs on the host."""

from __future__ import annotations

import math

import numpy as np
import torch

from lm_util import f64

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
C, CUBE = math.sqrt(2 / math.pi), 0.044715


def erf(z):
    return torch.erf(torch.from_numpy(np.ascontiguousarray(z))).numpy()


def act(z, kind):
    if kind == "relu":
        return np.maximum(z, 0)
    if kind == "gelu":
        return z * (1 + erf(z / math.sqrt(2))) / 2
    if kind == "gelu_tanh":
        return z * (1 + np.tanh(C * (z + CUBE * z ** 3))) / 2
    if kind == "silu":
        with np.errstate(over="ignore"):
            return z / (1 + np.exp(-z))
    return z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).astype(np.float64)
    if kind == "gelu":
        return (1 + erf(z / math.sqrt(2))) / 2 + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        t = np.tanh(C * (z + CUBE * z ** 3))
        return (1 + t) / 2 + z * (1 - t * t) * C * (1 + 3 * CUBE * z * z) / 2
    if kind == "silu":
        with np.errstate(over="ignore"):
            p = 1 / (1 + np.exp(-z))
        return p * (1 + z * (1 - p))
    return np.ones_like(z)


def linear_fwd(x, w, bias, kind, residual):
    """y, z, and the sum of the magnitudes that z is the sum of."""
    x, w = f64(x), f64(w)
    z, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        b = f64(bias)
        z, mag = z + b, mag + np.abs(b)
    y = act(z, kind)
    return (y if residual is None else y + f64(residual)), z, mag


def linear_bwd(dy, x, w, pre, kind):
    """dx, dw, db and the sums of magnitudes behind each."""
    dy, x, w = f64(dy), f64(x), f64(w)
    dz = dy if kind == "none" else dy * slope(f64(pre), kind)
    a = np.abs(dz)
    return dz @ w, dz.T @ x, dz.sum(0), a @ np.abs(w), a.T @ np.abs(x), a.sum(0)


def angles(rotation, rows):
    """[rows, pairs]"""
    positions, freqs, sections, _ = rotation
    p, f = f64(positions).reshape(len(sections), rows), f64(freqs)
    axis = np.repeat(np.arange(len(sections)), sections)
    return p[axis].T * f


def turn(x, rotation, back=False):
    """x [rows, heads, D]"""
    if rotation is None:
        return x
    a = angles(rotation, x.shape[0])[:, None]
    pairs = a.shape[2]
    c, s = np.cos(a), np.sin(a) * (-1 if back else 1)
    i = np.arange(pairs)
    u, v = (2 * i, 2 * i + 1) if rotation[3] else (i, i + pairs)
    y = x.copy()
    y[..., u], y[..., v] = x[..., u] * c - x[..., v] * s, x[..., v] * c + x[..., u] * s
    return y


def paired(x, rotation):
    """What a turned column is a sum of, in magnitude: |u| + |v| of its pair."""
    if rotation is None:
        return np.abs(x)
    pairs = rotation[1].numel()
    i = np.arange(pairs)
    u, v = (2 * i, 2 * i + 1) if rotation[3] else (i, i + pairs)
    y = np.abs(x)
    both = y[..., u] + y[..., v]
    y[..., u], y[..., v] = both, both
    return y


def rotate_fwd(x, w, rotation, norm, eps):
    """(output, magnitudes), x [rows, heads, D]"""
    x = f64(x)
    if norm:
        x = x / np.sqrt((x * x).mean(2, keepdims=True) + eps) * (1 if w is None else f64(w))
    return turn(x, rotation), paired(x, rotation)


def rotate_bwd(dy, x, w, rotation, norm, eps):
    """dx, dw, magnitudes of dx and of dw."""
    dy = f64(dy)
    g, mag = turn(dy, rotation, True), paired(dy, rotation)
    if not norm:
        return g, None, mag, None
    x, w = f64(x), 1 if w is None else f64(w)
    r = 1 / np.sqrt((x * x).mean(2, keepdims=True) + eps)
    dx = r * (g * w - x * r ** 2 * (g * w * x).mean(2, keepdims=True))
    mag_x = r * (mag * np.abs(w) + np.abs(x) * r ** 2 * (mag * np.abs(w * x)).mean(2, keepdims=True))
    return dx, (g * x * r).sum((0, 1)), mag_x, (mag * np.abs(x) * r).sum((0, 1))


def logprob_fwd(logits, tokens, scale, k):
    """logprob, lse, entropy, ids, their log probabilities"""
    raw = f64(logits)
    rows, V = raw.shape
    z = raw * scale
    top = z.max(1)
    none = top == -np.inf
    m = np.where(none, 0, top)
    with np.errstate(divide="ignore", invalid="ignore"):
        log_s = np.log(np.exp(z - m[:, None]).sum(1))
        lse = np.where(none, -np.inf, m + log_s)
        # (from m and not from lse, which beside a type's lowest value has lost log_s in 64 bits as well)
        log_p = np.where(none[:, None], -np.inf, (z - m[:, None]) - log_s[:, None])
        p = np.exp(log_p)
        entropy = -np.where(p > 0, p * np.where(p > 0, log_p, 0), 0).sum(1)
    t = np.full(rows, -1) if tokens is None else tokens.cpu().numpy().reshape(-1).astype(np.int64)
    there = (t >= 0) & (t < V)
    logprob = np.where(there, log_p[np.arange(rows), np.where(there, t, 0)], 0.0)
    order = np.argsort(-raw, axis=1, kind="stable")[:, :k]
    ids, best = np.full((rows, k), -1), np.full((rows, k), -np.inf)
    n = order.shape[1]
    got = np.take_along_axis(log_p, order, 1)
    ids[:, :n], best[:, :n] = np.where(np.take_along_axis(raw, order, 1) == -np.inf, -1, order), got
    return logprob, lse, entropy, ids, best


def logprob_bwd(logits, tokens, scale, lse, entropy, g, ge):
    """(gradient, magnitudes)"""
    raw, lse = f64(logits), f64(lse).reshape(-1)
    rows, V = raw.shape
    with np.errstate(invalid="ignore"):
        log_p = raw * scale - lse[:, None]
    dead = (raw == -np.inf) | (lse == -np.inf)[:, None]
    log_p = np.where(dead, 0, log_p)
    p = np.where(dead, 0, np.exp(log_p))
    d, mag = np.zeros((rows, V)), np.zeros((rows, V))
    if g is not None:
        t = tokens.cpu().numpy().reshape(-1).astype(np.int64)
        there = (t >= 0) & (t < V)
        gg = np.where(there, f64(g).reshape(-1), 0)
        d -= gg[:, None] * p
        mag += np.abs(gg[:, None]) * p
        at = np.nonzero(there)[0]
        d[at, t[at]] += gg[at]
        mag[at, t[at]] += np.abs(gg[at])
    if ge is not None:
        h = f64(entropy).reshape(-1)[:, None]
        d -= f64(ge).reshape(-1)[:, None] * p * (log_p + h)
        mag += np.abs(f64(ge).reshape(-1)[:, None]) * p * (np.abs(log_p) + np.abs(h))
    return np.where(dead, 0, d) * scale, np.where(dead, 0, mag) * scale, log_p
