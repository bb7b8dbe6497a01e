"""The operators at a language model's way in, as timed cases: token embedding, dropout, residual addition + RMS norm.

Every case is one pass through one operator of ``paper_2101_11714_amd.binding``:

  embed         tt_token_fwd: rows of a table by token, scaled, with dropout or without.
  embed_grad    tt_token_bwd: the table's gradient, written whole or added to a gradient that is there.
  embed_sgd     tt_token_bwd_sgd: the step on the rows in use, in place.
  dropout       tt_dropout_fwd, alone or with the residual's addition.
  dropout_grad  tt_dropout_bwd.
  norm          tt_add_rms_norm_fwd: residual + dropout(x), its root-mean-square norm in the inputs' type or in 8 bits (e4m3)
                with a scale per row or per 128 columns.
  norm_grad     tt_add_rms_norm_bwd: gradients of x, of the residual and of the weight.

Random numbers come from Philox4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011), keyed by a seed and
a step that are inputs, so that every implementation keeps the same elements: block b = row * ceil(dim / 8) + column / 8,
counter (b low, b high, site, step), 16 bits per column, kept where they are at least q = round(65536 p).

With ``own`` false the operators are computed in their plain form: elementary torch operations in 32 bits, rounded once.
"""

import functools
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
SITE = 3                                                    # the dropout's number within its model
MOST8 = 448.0                                               # the largest e4m3 value


def _embed(rows, vocab, dim, type, out, zipf=1.0, pads=0.0, p=0.0, scale=1.0, ids="i64", lead=0):
    return {"kind": "embed", "rows": rows, "vocab": vocab, "dim": dim, "type": type, "out": out, "zipf": zipf, "pads": pads, "p": p,
            "scale": scale, "ids": ids, "lead": lead}


def _embed_grad(rows, vocab, dim, type, out, zipf=1.0, pads=0.0, p=0.0, scale=1.0, ids="i64", lead=0, add=False):
    return dict(_embed(rows, vocab, dim, type, out, zipf, pads, p, scale, ids, lead), kind="embed_grad", add=add)


def _embed_sgd(rows, vocab, dim, type, out, zipf=1.0, pads=0.0, p=0.0, scale=1.0, ids="i64", lead=0, lr=0.5):
    return dict(_embed(rows, vocab, dim, type, out, zipf, pads, p, scale, ids, lead), kind="embed_sgd", lr=lr)


def _dropout(kind, rows, dim, type, p, residual=False, lead=0):
    return {"kind": kind, "rows": rows, "dim": dim, "type": type, "p": p, "residual": residual, "lead": lead}


def _norm(rows, dim, type, stream, p=0.0, bits8="", lead=0):
    """stream: the type of the residual stream, "" for a norm of x alone; bits8: "", "row" or "group"."""
    return {"kind": "norm", "rows": rows, "dim": dim, "type": type, "stream": stream, "p": p, "bits8": bits8, "lead": lead}


def _norm_grad(rows, dim, type, stream, p=0.0, passed=True, lead=0):
    """passed: a gradient arrives through the residual stream as well."""
    return {"kind": "norm_grad", "rows": rows, "dim": dim, "type": type, "stream": stream, "p": p, "passed": passed, "lead": lead}


def listed():
    return [
        # Generation, one token for each of a few dozen sequences: all latency.
        dict(_embed(48, 32768, 1024, "bf16", "bf16", scale=32.0), name="embed_decode"),
        # A training batch of 32 sequences of 1,024 tokens with dropout.
        dict(_embed(32768, 131072, 4096, "bf16", "bf16", p=0.1), name="embed_train"),
        # A batch with padding, odd counts, an odd dimension, into the 32-bit residual stream.
        dict(_embed_grad(4093, 50001, 1001, "f16", "f32", pads=0.2, ids="i32"), name="embed_grad_ragged"),
        # The gradient of the training batch above in 32 bits: the largest pass.
        dict(_embed_grad(32768, 131072, 4096, "bf16", "f32", p=0.1), name="embed_grad_train"),
        # The step of an uncompressed table of this repository's dimension 64, used rows only.
        dict(_embed_sgd(16384, 1000000, 64, "f32", "f32", zipf=1.05), name="embed_sgd_dim64"),
        # Dropout and residual addition at the end of a small branch, an odd shape in 32 bits.
        dict(_dropout("dropout", 257, 777, "f32", 0.1, residual=True), name="dropout_small"),
        # The same at training size.
        dict(_dropout("dropout", 16384, 4096, "bf16", 0.1, residual=True), name="dropout_train"),
        # Its gradient, rows of a wider array.
        dict(_dropout("dropout_grad", 8192, 2048, "bf16", 0.2, lead=2048), name="dropout_grad_strided"),
        # Serving: seven sequences' next tokens, residual addition and norm into 8 bits for the following matrix product.
        dict(_norm(7, 8192, "bf16", "bf16", bits8="row"), name="norm_decode"),
        # Prefill: 8 bits with scales per 128 columns.
        dict(_norm(16384, 4096, "bf16", "bf16", bits8="group"), name="norm_prefill"),
        # Gradients at training size, dropout in the branch, residual stream in 32 bits.
        dict(_norm_grad(8192, 4096, "bf16", "f32", p=0.1), name="norm_grad_train"),
        # Rows of dimension 64, as a compressed table gives them, many of them, odd count.
        dict(_norm_grad(100003, 64, "f32", "f32"), name="norm_grad_dim64"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST = 1 << 26                                              # elements of a drawn case's largest array of rows


def _dim(rng):
    way = rng.random()
    if way < 0.4:
        return 1 << rng.randint(5, 13)
    if way < 0.7:
        return 640 * rng.randint(1, 12)
    return _log(rng, 16, 8192) | 1


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_sgd", "dropout", "dropout_grad", "norm", "norm_grad"])
    dim, type = _dim(rng), rng.choice(["f32", "bf16", "bf16", "f16"])
    rows = _log(rng, 1, min(65536, MOST // dim))
    p = rng.choice([0.0, 0.1, round(rng.uniform(0.01, 0.6), 3)])
    lead = rng.choice([0, 0, 8, 3])
    if kind.startswith("embed"):
        vocab = _log(rng, 1000, min(1_000_000, 4 * MOST // dim))
        out = rng.choice([type, "f32"])
        more = (rows, vocab, dim, type, out, round(rng.uniform(0.8, 1.2), 3), rng.choice([0.0, 0.0, 0.3]), p,
                rng.choice([1.0, round(math.sqrt(dim), 4)]), rng.choice(["i64", "i32"]), lead)
        if kind == "embed":
            return _embed(*more)
        return _embed_grad(*more, add=rng.random() < 0.3) if kind == "embed_grad" else _embed_sgd(*more)
    if kind.startswith("dropout"):
        return _dropout(kind, rows, dim, type, p or 0.1, kind == "dropout" and rng.random() < 0.5, lead)
    stream = rng.choice([type, "f32"])
    if kind == "norm":
        stream = rng.choice([stream, stream, ""])
        return _norm(rows, dim, type, stream, p if stream else 0.0, rng.choice(["", "row", "group"]), lead)
    return _norm_grad(rows, dim, type, stream, p, rng.random() < 0.7, lead)


# ---- inputs ---------------------------------------------------------------------------------------------------------


class _State:
    pass


def _normal(gen, rows, dim, type, lead=0, size=1.0):
    """A [rows, dim] array of normal values; with `lead`, the left part of wider rows."""
    wide = torch.empty((rows, dim + lead), dtype=TYPES[type], device=DEV).normal_(0.0, size, generator=gen)
    return wide[:, :dim]


def _room(rows, dim, type, lead=0):
    return torch.empty((rows, dim + lead), dtype=type if isinstance(type, torch.dtype) else TYPES[type], device=DEV)[:, :dim]


def _tokens(case, gen):
    """Tokens by a Zipf law over their numbers; the last part of each 512 positions is padding (-1)."""
    cdf = torch.arange(1, case["vocab"] + 1, dtype=torch.float64, device=DEV).pow_(-case["zipf"]).cumsum_(0)
    u = torch.rand(case["rows"], dtype=torch.float64, generator=gen, device=DEV) * cdf[-1]
    tokens = torch.searchsorted(cdf, u).clamp_(max=case["vocab"] - 1)
    at = torch.arange(case["rows"], device=DEV) % 512
    tokens = torch.where(at >= 512 * (1.0 - case["pads"]), -1, tokens)
    return tokens.to(torch.int32 if case["ids"] == "i32" else torch.int64)


def prepare(case, seed):
    s = _State()
    s.case, kind, rows, dim, lead = case, case["kind"], case["rows"], case["dim"], case["lead"]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s.rng = torch.tensor([seed * 0x9E3779B97F4A7C1 & 0x7FFFFFFFFFFFFFFF, 17 + seed % 1000], dtype=torch.int64, device=DEV)
    s.drop = (case["p"], s.rng, SITE) if case["p"] else None
    if kind.startswith("embed"):
        s.tokens = _tokens(case, gen)
        if kind == "embed":
            s.table = _normal(gen, case["vocab"], dim, case["type"], lead, 1.0 / math.sqrt(dim))
            s.out = _room(rows, dim, case["out"], lead)
            return s
        s.grad = _normal(gen, rows, dim, case["type"], lead, 0.25)
        if kind == "embed_grad":
            s.out = _normal(gen, case["vocab"], dim, case["out"], lead) if case["add"] else _room(case["vocab"], dim, case["out"], lead)
        else:
            s.table = _normal(gen, case["vocab"], dim, case["out"], lead)
        return s
    s.x = _normal(gen, rows, dim, case["type"], lead)       # (a gradient, for the backward passes)
    if kind.startswith("dropout"):
        s.residual = _normal(gen, rows, dim, case["type"], lead) if case["residual"] else None
        s.out = _room(rows, dim, case["type"], lead)
        return s
    stream = case["stream"]
    s.weight = torch.empty(dim, dtype=TYPES[case["type"]], device=DEV).normal_(1.0, 0.1, generator=gen)
    if kind == "norm":
        s.residual = _normal(gen, rows, dim, stream, lead, 2.0) if stream else None
        s.sum = _room(rows, dim, stream, lead) if stream else None
        s.out = _room(rows, dim, torch.float8_e4m3fn if case["bits8"] else case["type"], lead)
        groups = -(-dim // 128) if case["bits8"] == "group" else 1
        s.scales = _room(rows, groups, "f32") if case["bits8"] else None
        s.rstd = torch.empty(rows, dtype=torch.float32, device=DEV)
        return s
    s.h = _normal(gen, rows, dim, stream, lead, 2.0)
    s.rstd = (s.h.float().square().mean(1) + EPS).rsqrt()
    s.passed = _normal(gen, rows, dim, stream, lead) if case["passed"] else None
    s.gx = _room(rows, dim, case["type"], lead)
    s.gr = _room(rows, dim, stream, lead) if s.drop or stream != case["type"] else None
    s.gw = torch.empty(dim, dtype=torch.float32, device=DEV)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2101_11714_amd import binding as B
    case = s.case
    kind, drop = case["kind"], s.drop
    if kind == "embed":
        return B.tt_token_fwd(s.table, s.tokens, s.out, scale=case["scale"], dropout=drop)
    if kind == "embed_grad":
        return B.tt_token_bwd(s.tokens, s.grad, s.out, scale=case["scale"], dropout=drop, accumulate=case["add"])
    if kind == "embed_sgd":
        return B.tt_token_bwd_sgd(s.tokens, s.grad, s.table, case["lr"], scale=case["scale"], dropout=drop)
    if kind == "dropout":
        return B.tt_dropout_fwd(s.x, s.out, drop, residual=s.residual)
    if kind == "dropout_grad":
        return B.tt_dropout_bwd(s.x, s.out, drop)
    if kind == "norm":
        B.tt_add_rms_norm_fwd(s.x, s.weight, s.out, residual=s.residual, sum_out=s.sum, rstd=s.rstd, scales=s.scales,
                              group=128 if case["bits8"] == "group" else 0, eps=EPS, dropout=drop)
        return {"out": s.out, "scales": s.scales, "sum": s.sum, "rstd": s.rstd}
    B.tt_add_rms_norm_bwd(s.x, s.h, s.rstd, s.weight, s.gx, s.gw, grad_sum=s.passed, grad_residual=s.gr, dropout=drop)
    return {"x": s.gx, "residual": s.gr, "weight": s.gw}


LOW = 0xFFFFFFFF


def _kept(rows, dim, drop):
    """Which elements of a [rows, dim] array are kept, and the factor of those."""
    p, rng, site = drop
    q = int(math.floor(p * 65536 + 0.5))
    block = torch.arange(rows * -(-dim // 8), dtype=torch.int64, device=DEV)
    c0, c1, c2, c3 = block & LOW, block >> 32, torch.full_like(block, site), (rng[1] & LOW).expand_as(block)
    k0, k1 = rng[0] & LOW, (rng[0] >> 32) & LOW
    for _ in range(10):                                     # the generator's rounds
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & LOW) ^ c1 ^ k0, b & LOW, ((a >> 32) & LOW) ^ c3 ^ k1, a & LOW
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    words = torch.stack([c0, c1, c2, c3], 1)
    draws = torch.stack([words & 0xFFFF, words >> 16], 2).view(rows, -1)
    return draws[:, :dim] >= q, 65536.0 / (65536 - q) if q < 65536 else 0.0


def _dropped(x, drop):
    if drop is None:
        return x
    keep, factor = _kept(x.shape[0], x.shape[1], drop)
    return torch.where(keep, x * factor, 0.0)


def _plain(s):
    case = s.case
    kind = case["kind"]
    if kind == "embed":
        there = (s.tokens >= 0) & (s.tokens < case["vocab"])
        got = s.table[torch.where(there, s.tokens, 0).long()].float() * case["scale"]
        return _dropped(torch.where(there[:, None], got, 0.0), s.drop).to(s.out.dtype)
    if kind in ("embed_grad", "embed_sgd"):
        there = (s.tokens >= 0) & (s.tokens < case["vocab"])
        grad = torch.where(there[:, None], _dropped(s.grad.float(), s.drop) * case["scale"], 0.0)
        sums = torch.zeros((case["vocab"], case["dim"]), dtype=torch.float32, device=DEV)
        sums.index_add_(0, torch.where(there, s.tokens, 0).long(), grad)
        if kind == "embed_sgd":
            s.table.copy_(s.table.float() - case["lr"] * sums)
            return s.table
        if case["add"]:
            s.out.copy_(s.out.float() + sums)
            return s.out
        return sums.to(s.out.dtype)
    if kind == "dropout":
        got = _dropped(s.x.float(), s.drop)
        return (got if s.residual is None else got + s.residual.float()).to(s.x.dtype)
    if kind == "dropout_grad":
        return _dropped(s.x.float(), s.drop).to(s.x.dtype)
    weight = s.weight.float()
    if kind == "norm":
        h = _dropped(s.x.float(), s.drop)
        if s.residual is not None:
            h = h + s.residual.float()
        rstd = (h.square().mean(1) + EPS).rsqrt()
        y = h * rstd[:, None] * weight
        got = {"out": y, "scales": None, "sum": None if s.sum is None else h.to(s.sum.dtype), "rstd": rstd}
        if not case["bits8"]:
            return dict(got, out=y.to(s.out.dtype))
        width = 128 if case["bits8"] == "group" else case["dim"]
        groups = -(-case["dim"] // width)
        y = torch.nn.functional.pad(y, (0, groups * width - case["dim"])).view(case["rows"], groups, width)
        scales = y.abs().amax(2) / MOST8
        q = torch.where(scales[..., None] == 0, 0.0, y / scales[..., None]).view(case["rows"], -1)[:, :case["dim"]]
        return dict(got, out=q.to(torch.float8_e4m3fn), scales=scales)
    dy, h, rstd = s.x.float(), s.h.float(), s.rstd[:, None]
    g = dy * weight
    dh = rstd * (g - h * rstd.square() * (g * h).mean(1, keepdim=True))
    if s.passed is not None:
        dh = dh + s.passed.float()
    return {"x": _dropped(dh, s.drop).to(s.gx.dtype), "residual": None if s.gr is None else dh.to(s.gr.dtype), "weight": (dy * h * rstd).sum(0)}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------


def _philox(block, site, step, seed):
    """The four words of each block, [blocks, 4], on the host with 64-bit products."""
    low, high = np.uint64(LOW), np.uint64(32)
    x = [block & low, block >> high, np.full_like(block, site), np.full_like(block, step & LOW)]
    key = [np.uint64(seed & LOW), np.uint64(seed >> 32 & LOW)]
    for r in range(10):
        first, second = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [second >> high ^ x[1] ^ key[0], second & low, first >> high ^ x[3] ^ key[1], first & low]
        key = [key[0] + np.uint64(0x9E3779B9) & low, key[1] + np.uint64(0xBB67AE85) & low]
    return np.stack(x, 1).astype(np.uint32)


def _factors(s, rows, dim):
    """What dropout multiplies each element by, [rows, dim] in 64 bits."""
    if s.drop is None:
        return torch.ones((1, 1), dtype=torch.float64, device=DEV)
    seed, step = (int(v) for v in s.rng.cpu())
    q = int(round(s.drop[0] * 65536))
    per, parts = -(-dim // 8), []
    for r0 in range(0, rows, 4096):
        n = min(4096, rows - r0)
        words = _philox(np.arange(r0 * per, (r0 + n) * per, dtype=np.uint64), s.drop[2], step, seed)
        keep = words.view(np.uint16).reshape(n, per * 8)[:, :dim] >= q
        parts.append(torch.from_numpy(keep).to(DEV))
    return torch.cat(parts).double() * (65536.0 / (65536 - q))


def exact(case, seed):
    s = prepare(case, seed)
    kind, rows, dim = case["kind"], case["rows"], case["dim"]
    keep = _factors(s, rows, dim)
    if kind == "embed":
        out = torch.zeros((rows, dim), dtype=torch.float64, device=DEV)
        at = torch.nonzero(s.tokens >= 0)[:, 0]
        out[at] = s.table[s.tokens[at].long()].double()
        return out.mul_(case["scale"]).mul_(keep)
    if kind in ("embed_grad", "embed_sgd"):
        order = torch.argsort(s.tokens, stable=True)
        order = order[int((s.tokens < 0).sum()):]
        used, count = torch.unique_consecutive(s.tokens[order], return_counts=True)
        ends = count.cumsum(0)
        base = s.table if kind == "embed_sgd" else s.out if case["add"] else None
        factor = -case["lr"] * case["scale"] if kind == "embed_sgd" else case["scale"]
        total = torch.zeros((case["vocab"], dim), dtype=torch.float64, device=DEV) if base is None else base.double()
        for c0 in range(0, dim, 256):                       # differences of running sums, some columns at a time
            part = s.grad[:, c0:c0 + 256].double() * (keep[:, c0:c0 + 256] if s.drop else keep)
            run_ = torch.nn.functional.pad(part[order].cumsum(0), (0, 0, 1, 0))
            total[used.long(), c0:c0 + 256] += factor * (run_[ends] - run_[ends - count])
        return total
    if kind in ("dropout", "dropout_grad"):
        got = s.x.double() * keep
        return got if s.residual is None else got + s.residual.double()
    w = s.weight.double()
    if kind == "norm":
        h = s.x.double() * keep
        if s.residual is not None:
            h = h + s.residual.double()
        rstd = ((h * h).sum(1) / dim + EPS) ** -0.5
        y = h * rstd[:, None] * w
        got = {"out": y, "scales": None, "sum": None if s.sum is None else h, "rstd": rstd}
        if case["bits8"]:
            width = 128 if case["bits8"] == "group" else dim
            parts = [y[:, c:c + width].abs().max(1).values / MOST8 for c in range(0, dim, width)]
            got["scales"] = torch.stack(parts, 1)
            got["out"] = y / got["scales"].repeat_interleave(width, 1)[:, :dim]
        return got
    dy, h, rstd = s.x.double(), s.h.double(), s.rstd.double()[:, None]
    along = ((dy * w * h).sum(1, keepdim=True) / dim) * rstd ** 3
    dh = rstd * dy * w - h * along
    if s.passed is not None:
        dh = dh + s.passed.double()
    return {"x": dh * keep, "residual": None if s.gr is None else dh, "weight": (dy * (h * rstd)).sum(0)}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------


@functools.lru_cache(maxsize=None)
def _distinct(vocab, zipf, count):
    """The expected number of distinct tokens among `count`."""
    p = np.arange(1, vocab + 1, dtype=np.float64) ** (-zipf)
    return float(-np.expm1(-count * (p / p.sum())).sum())


def work(case):
    kind, rows, dim = case["kind"], case["rows"], case["dim"]
    n, size = rows * dim, SIZE[case["type"]]
    if kind.startswith("embed"):
        live = rows * (1.0 - case["pads"])
        used, ids, out = _distinct(case["vocab"], case["zipf"], live), (4 if case["ids"] == "i32" else 8) * rows, SIZE[case["out"]]
        if kind == "embed":
            return {"bytes": ids + used * dim * size + n * out, "flops": 2.0 * n}
        table = 2 * used if kind == "embed_sgd" or case["add"] else case["vocab"]
        return {"bytes": ids + live * dim * size + table * dim * out, "flops": 3.0 * n}
    if kind.startswith("dropout"):
        return {"bytes": n * size * (3 if case["residual"] else 2), "flops": 2.0 * n}
    stream = SIZE[case["stream"]] if case["stream"] else 0
    if kind == "norm":
        groups = 0 if not case["bits8"] else -(-dim // 128) if case["bits8"] == "group" else 1
        return {"bytes": n * (size + 2 * stream + (1 if case["bits8"] else size)) + rows * 4 * (1 + groups) + dim * size, "flops": 6.0 * n}
    two = case["p"] > 0 or case["stream"] != case["type"]
    return {"bytes": n * (2 * size + stream * (1 + two + case["passed"])) + 4 * rows + dim * (size + 4), "flops": 12.0 * n}
