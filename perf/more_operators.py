"""The products of a language model and what is done to their rows, as timed cases: a matrix product with its epilogue, norm and
rotation of queries and keys, log probabilities of tokens.

Every case is one pass through one operator of ``paper_2101_11714_amd.binding``:

  linear        tt_linear_fwd: act(x W^T + bias) + residual, the value before the activation kept for the gradient.
  linear_grad   tt_linear_bwd: gradients of x, of the weight (written or added) and of the bias.
  rotate        tt_qk_norm_rotate_fwd: every head's root-mean-square norm and the rotation by its row's position, whose pairs belong
                to one axis or to several (time, height, width); queries and keys in one call, parts of a wider row.
  rotate_grad   tt_qk_norm_rotate_bwd: gradients of queries, keys and of the norms' weights.
  logprob       tt_token_logprob_fwd: log probability of a given token per row of logits, entropy, the k likeliest alternatives.
  logprob_grad  tt_token_logprob_bwd: the gradient of the logits from those of the log probability and of the entropy.

With ``own`` false the operators are computed in their plain form: elementary torch operations in 32 bits (angles of positions in
64), rounded once.
"""

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
BASE = 10000.0                                              # of the rotation's frequencies


def _linear(rows, k, n, type, act="none", bias=True, residual=False, pre=False, out="", lead=0):
    """out: the output's and the residual's type, "" for x's."""
    return {"kind": "linear", "rows": rows, "k": k, "n": n, "type": type, "act": act, "bias": bias, "residual": residual, "pre": pre,
            "out": out or type, "lead": lead}


def _linear_grad(rows, k, n, type, act="none", bias=True, wtype="", add=False, lead=0):
    return {"kind": "linear_grad", "rows": rows, "k": k, "n": n, "type": type, "act": act, "bias": bias, "wtype": wtype or type, "add": add, "lead": lead}


def _rotate(rows, heads, kv, dim, type, norm=True, rot=0, axes=1, neighbours=False, far=0, lead=0):
    """rot: rotated columns of a head, 0 for all; neighbours: pairs of neighbouring columns, else of the halves; far: the first position."""
    return {"kind": "rotate", "rows": rows, "heads": heads, "kv": kv, "dim": dim, "type": type, "norm": norm, "rot": rot or dim, "axes": axes,
            "neighbours": neighbours, "far": far, "lead": lead}


def _rotate_grad(*a, **k):
    return dict(_rotate(*a, **k), kind="rotate_grad")


def _logprob(rows, vocab, type, entropy=True, top=0, scale=1.0, banned=0.0, pads=0.0, lead=0):
    """banned: the share of a row's logits that are -inf."""
    return {"kind": "logprob", "rows": rows, "vocab": vocab, "type": type, "entropy": entropy, "top": top, "scale": scale, "banned": banned,
            "pads": pads, "lead": lead}


def _logprob_grad(*a, **k):
    return dict(_logprob(*a, **k), kind="logprob_grad")


def listed():
    return [
        # Generation: the product at a branch's end for a few sequences' next tokens, with the residual.
        dict(_linear(5, 4096, 4096, "bf16", residual=True), name="linear_decode"),
        # Training: the first product of a feed-forward branch; the largest pass.
        dict(_linear(8192, 4096, 16384, "bf16", act="gelu_tanh", pre=True), name="linear_train"),
        # An odd shape in 32 bits, rows of wider arrays.
        dict(_linear(1001, 777, 1283, "f32", act="relu", residual=True, lead=3), name="linear_ragged"),
        # Gradients at a training batch's size, through an activation.
        dict(_linear_grad(8192, 4096, 4096, "bf16", act="silu"), name="linear_grad_train"),
        # Gradients of the way out, a table of the vocabulary's rows, added to a gradient in 32 bits.
        dict(_linear_grad(2048, 1024, 32768, "f16", bias=False, wtype="f32", add=True), name="linear_grad_out"),
        # Generation: two dozen sequences' next tokens at far positions.
        dict(_rotate(24, 32, 8, 128, "bf16", far=100000), name="rotate_decode"),
        # Prefill of a long prompt.
        dict(_rotate(16384, 32, 8, 128, "bf16"), name="rotate_prefill"),
        # An odd number of patches of a video: three axes, a smaller odd head, no norm, pairs of neighbours.
        dict(_rotate(9973, 16, 16, 72, "f16", norm=False, axes=3, neighbours=True), name="rotate_video"),
        # Gradients at a training batch's size.
        dict(_rotate_grad(8192, 32, 8, 128, "bf16"), name="rotate_grad_train"),
        # Serving: two dozen sequences' choices with twenty alternatives, a part of the vocabulary banned.
        dict(_logprob(24, 131072, "f32", top=20, scale=1.25, banned=0.1), name="logprob_serve"),
        # A training batch with padding, an odd vocabulary.
        dict(_logprob(4096, 50257, "bf16", pads=0.1), name="logprob_train"),
        # The gradient of a larger one.
        dict(_logprob_grad(4096, 131072, "bf16"), name="logprob_grad_train"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, most=8192):
    way = rng.random()
    if way < 0.4:
        return min(most, 1 << rng.randint(5, 13))
    if way < 0.7:
        return min(most, 640 * rng.randint(1, 12))
    return _log(rng, 16, most) | 1


MOST_FLOPS = 5.0e11                                         # of a drawn product
MOST = 1 << 26                                              # elements of a drawn case's heads
MOST_LOGITS = 1 << 28
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_grad", "rotate", "rotate_grad", "logprob", "logprob_grad"])
    type = rng.choice(["f32", "bf16", "bf16", "f16"])
    lead = rng.choice([0, 0, 8, 3])
    if kind.startswith("linear"):
        k, n = _width(rng), _width(rng, 16384)
        rows = _log(rng, 1, min(16384, MOST_FLOPS / (2 * k * n * (2 if kind == "linear_grad" else 1)) / (8 if type == "f32" else 1) + 1))
        act, bias = rng.choice(ACTS), rng.random() < 0.6
        if kind == "linear":
            return _linear(rows, k, n, type, act, bias, rng.random() < 0.4, act != "none" and rng.random() < 0.5, rng.choice(["", "f32"]), lead)
        return _linear_grad(rows, k, n, type, act, bias, rng.choice(["", "f32"]) if act == "none" else "", rng.random() < 0.3, lead)
    if kind.startswith("rotate"):
        kv = rng.choice([1, 2, 4, 8, 16])
        heads = kv * rng.choice([1, 2, 4, 5, 8]) if kv < 16 else 16
        dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 160, 192, 256, 2 * rng.randint(9, 120)])
        rows = _log(rng, 1, min(65536, MOST // (dim * (heads + kv))))
        rot = rng.choice([0, 0, 0, 2 * rng.randint(1, dim // 2)])
        return dict(_rotate(rows, heads, kv, dim, type, rng.random() < 0.6, rot, rng.choice([1, 1, 2, 3]), rng.random() < 0.4,
                            rng.choice([0, 0, _log(rng, 10, 10_000_000)]), lead), kind=kind)
    vocab = rng.choice([_log(rng, 500, 262144), _log(rng, 500, 262144) | 1, 32768, 131072])
    top = rng.choice([0, 1, 5, 20, 32]) if kind == "logprob" else 0
    rows = _log(rng, 1, min(512 if top else 16384, MOST_LOGITS // vocab))
    return dict(_logprob(rows, vocab, type, rng.random() < 0.6, top, rng.choice([1.0, round(rng.uniform(0.3, 2.0), 3)]),
                         rng.choice([0.0, 0.0, 0.3]), rng.choice([0.0, 0.2]), lead), kind=kind)


# ---- inputs ---------------------------------------------------------------------------------------------------------


class _State:
    pass


def _normal(gen, rows, dim, type, lead=0, size=1.0):
    """A [rows, dim] array of normal values; with `lead`, the left part of wider rows."""
    wide = torch.empty((rows, dim + lead), dtype=TYPES[type], device=DEV).normal_(0.0, size, generator=gen)
    return wide[:, :dim]


def _room(rows, dim, type, lead=0):
    return torch.empty((rows, dim + lead), dtype=TYPES[type], device=DEV)[:, :dim]


def _vector(n, type="f32"):
    return torch.empty(n, dtype=TYPES[type], device=DEV)


def _sections(case):
    """How many of a head's pairs belong to each axis: the last one has what is left."""
    pairs, axes = case["rot"] // 2, case["axes"]
    each = pairs // axes
    return [each] * (axes - 1) + [pairs - each * (axes - 1)]


def _positions(case):
    """[axes, rows]: one axis counts on, several walk through frames of 24 x 32 places."""
    at = torch.arange(case["rows"], dtype=torch.int64, device=DEV)
    if case["axes"] == 1:
        return (at + case["far"])[None]
    parts = [at // 768 + case["far"], at // 32 % 24, at % 32]
    return torch.stack(parts[:case["axes"]])


def _prepare_linear(s, case, gen):
    rows, k, n, type, lead = case["rows"], case["k"], case["n"], case["type"], case["lead"]
    s.weight = _normal(gen, n, k, type, lead, 1.0 / math.sqrt(k))
    s.x = _normal(gen, rows, k, type, lead)
    s.pre = None
    if case["kind"] == "linear":
        s.bias = _normal(gen, 1, n, type, 0, 0.5)[0] if case["bias"] else None
        s.residual = _normal(gen, rows, n, case["out"], lead, 2.0) if case["residual"] else None
        s.out = _room(rows, n, case["out"], lead)
        s.pre = _room(rows, n, type) if case["pre"] else None
        return s
    s.grad = _normal(gen, rows, n, type, lead, 0.25)
    if case["act"] != "none":
        s.pre = _normal(gen, rows, n, type)
    s.gx = _room(rows, k, type, lead)
    s.gw = _normal(gen, n, k, case["wtype"], lead) if case["add"] else _room(n, k, case["wtype"], lead)
    s.gb = None
    if case["bias"]:
        s.gb = _normal(gen, 1, n, "f32")[0] if case["add"] else _vector(n)
    return s


def _prepare_rotate(s, case, gen):
    rows, heads, kv, dim, type = case["rows"], case["heads"], case["kv"], case["dim"], case["type"]
    wide = _normal(gen, rows, (heads + 2 * kv) * dim, type, case["lead"], 1.5)           # queries, keys, values of a row
    s.q = wide[:, :heads * dim].unflatten(1, (heads, dim))
    s.k = wide[:, heads * dim:(heads + kv) * dim].unflatten(1, (kv, dim))
    s.positions = _positions(case)
    s.freqs = torch.tensor([BASE ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)], dtype=torch.float32, device=DEV)
    s.sections = _sections(case)
    s.wq = s.wk = s.gwq = s.gwk = None
    if case["norm"]:
        s.wq, s.wk = (_vector(dim, type).normal_(1.0, 0.2, generator=gen) for _ in range(2))
    s.q_out = torch.empty((rows, heads, dim), dtype=TYPES[type], device=DEV)
    s.k_out = torch.empty((rows, kv, dim), dtype=TYPES[type], device=DEV)
    if case["kind"] == "rotate_grad":
        s.gq = _normal(gen, rows, heads * dim, type, 0, 0.25).unflatten(1, (heads, dim))
        s.gk = _normal(gen, rows, kv * dim, type, 0, 0.25).unflatten(1, (kv, dim))
        if case["norm"]:
            s.gwq, s.gwk = _vector(dim), _vector(dim)
    return s


def _prepare_logprob(s, case, gen):
    rows, vocab, type = case["rows"], case["vocab"], case["type"]
    s.logits = _normal(gen, rows, vocab, type, case["lead"], 2.5)
    s.tokens = torch.randint(0, vocab, (rows,), generator=gen, device=DEV)
    if case["banned"]:
        for r0 in range(0, rows, 1024):
            part = s.logits[r0:r0 + 1024]
            part.masked_fill_(torch.rand(part.shape, generator=gen, device=DEV) < case["banned"], float("-inf"))
        s.logits.scatter_(1, s.tokens[:, None], 1.0)                                     # (a chosen token was not banned)
    if case["pads"]:
        s.tokens = torch.where(torch.rand(rows, generator=gen, device=DEV) < case["pads"], -1, s.tokens)
    s.lse, s.entropy = _vector(rows), _vector(rows) if case["entropy"] else None
    if case["kind"] == "logprob":
        s.logprob, s.top_ids, s.top = _vector(rows), None, None
        if case["top"]:
            s.top_ids = torch.empty((rows, case["top"]), dtype=torch.int64, device=DEV)
            s.top = _room(rows, case["top"], "f32")
        return s
    for r0 in range(0, rows, 1024):                         # what the forward pass has left
        z = s.logits[r0:r0 + 1024].double() * case["scale"]
        lse = torch.logsumexp(z, 1)
        s.lse[r0:r0 + 1024] = lse
        if case["entropy"]:
            log_p = z - lse[:, None]
            s.entropy[r0:r0 + 1024] = -torch.where(log_p > -math.inf, log_p.exp() * log_p, 0.0).sum(1)
    s.g, s.ge = (_vector(rows).normal_(0.0, 1.0, generator=gen) for _ in range(2))
    s.ge = s.ge if case["entropy"] else None
    s.out = _room(rows, vocab, type, case["lead"])
    return s


def prepare(case, seed):
    s = _State()
    s.case = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    make = {"linear": _prepare_linear, "rotate": _prepare_rotate, "logprob": _prepare_logprob}
    return make[case["kind"].split("_")[0]](s, case, gen)


# ---- one pass -------------------------------------------------------------------------------------------------------


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2101_11714_amd import binding as B
    case = s.case
    kind = case["kind"]
    if kind == "linear":
        B.tt_linear_fwd(s.x, s.weight, s.out, bias=s.bias, activation=case["act"], residual=s.residual, pre=s.pre)
        return {"out": s.out, "pre": s.pre}
    if kind == "linear_grad":
        B.tt_linear_bwd(s.grad, s.x, s.weight, s.gx, s.gw, grad_bias=s.gb, pre=s.pre, activation=case["act"], accumulate=case["add"])
        return {"x": s.gx, "weight": s.gw, "bias": s.gb}
    if kind.startswith("rotate"):
        rotation = B.Rotation(s.positions, s.freqs, s.sections, case["neighbours"])
        if kind == "rotate":
            B.tt_qk_norm_rotate_fwd(s.q, s.k, s.q_out, s.k_out, rotation, norm=case["norm"], q_weight=s.wq, k_weight=s.wk, eps=EPS)
            return {"q": s.q_out, "k": s.k_out}
        B.tt_qk_norm_rotate_bwd(s.gq, s.gk, s.q, s.k, s.q_out, s.k_out, rotation, norm=case["norm"], q_weight=s.wq, k_weight=s.wk, grad_q_weight=s.gwq,
                                grad_k_weight=s.gwk, eps=EPS)
        return {"q": s.q_out, "k": s.k_out, "q_weight": s.gwq, "k_weight": s.gwk}
    if kind == "logprob":
        B.tt_token_logprob_fwd(s.logits, s.tokens, s.logprob, s.lse, entropy=s.entropy, top_ids=s.top_ids, top_logprobs=s.top, scale=case["scale"])
        return {"logprob": s.logprob, "lse": s.lse, "entropy": s.entropy, "top_ids": s.top_ids, "top": s.top}
    return B.tt_token_logprob_bwd(s.logits, s.tokens, s.lse, s.g, s.out, entropy=s.entropy, grad_entropy=s.ge, scale=case["scale"])


TANH = math.sqrt(2.0 / math.pi)
CUBE = 0.044715


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "silu":
        return z / (1.0 + (-z).exp())
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(TANH * (z + CUBE * z * z * z)))
    return z


def _act_grad(z, act):
    if act == "relu":
        return torch.where(z > 0, 1.0, 0.0)
    if act == "silu":
        p = 1.0 / (1.0 + (-z).exp())
        return p * (1.0 + z * (1.0 - p))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * (-0.5 * z * z).exp() * math.sqrt(0.5 / math.pi)
    t = torch.tanh(TANH * (z + CUBE * z * z * z))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * TANH * (1.0 + 3.0 * CUBE * z * z)


def _angles(s):
    """Cosines and sines, [rows, pairs]: angles in 64 bits, taken to one turn."""
    axis = torch.repeat_interleave(torch.arange(s.case["axes"], device=DEV), torch.tensor(s.sections, device=DEV))
    angle = s.positions[axis].t().double() * s.freqs.double()
    angle = torch.remainder(angle, 2.0 * math.pi)
    return angle.cos().float(), angle.sin().float()


def _turned(x, cos, sin, case):
    """x [rows, heads, dim], its pairs turned."""
    rot, c, d = case["rot"], cos[:, None], sin[:, None]
    y = x.clone()
    if case["neighbours"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * d, b * c + a * d
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * d, b * c + a * d
    return y


def _plain(s):
    case = s.case
    kind = case["kind"]
    if kind == "linear":
        z = s.x.float() @ s.weight.float().t()
        if s.bias is not None:
            z = z + s.bias.float()
        y = _act(z, case["act"])
        if s.residual is not None:
            y = y + s.residual.float()
        return {"out": y.to(s.out.dtype), "pre": None if s.pre is None else z.to(s.pre.dtype)}
    if kind == "linear_grad":
        dz = s.grad.float()
        if s.pre is not None:
            dz = dz * _act_grad(s.pre.float(), case["act"])
        gw, gb = dz.t() @ s.x.float(), None if s.gb is None else dz.sum(0)
        if case["add"]:
            gw = gw + s.gw.float()
            s.gw.copy_(gw)
            if gb is not None:
                gb = gb + s.gb
                s.gb.copy_(gb)
        return {"x": (dz @ s.weight.float()).to(s.gx.dtype), "weight": gw.to(s.gw.dtype), "bias": gb}
    if kind.startswith("rotate"):
        cos, sin = _angles(s)
        out = {}
        for name, x, w, g in (("q", s.q, s.wq, getattr(s, "gq", None)), ("k", s.k, s.wk, getattr(s, "gk", None))):
            x = x.float()
            r = (x.square().mean(2, keepdim=True) + EPS).rsqrt() if case["norm"] else None
            if kind == "rotate":
                y = x * r * w.float() if case["norm"] else x
                out[name] = _turned(y, cos, sin, case).to(s.q.dtype)
                continue
            dy = _turned(g.float(), cos, -sin, case)
            out[name + "_weight"] = None
            if case["norm"]:
                out[name + "_weight"] = (dy * x * r).sum((0, 1))
                dy = dy * w.float()
                dy = r * (dy - x * r.square() * (dy * x).mean(2, keepdim=True))
            out[name] = dy.to(s.q.dtype)
        return {name: out[name] for name in (("q", "k") if kind == "rotate" else ("q", "k", "q_weight", "k_weight"))}
    z = s.logits.float() * case["scale"]
    there = (s.tokens >= 0) & (s.tokens < case["vocab"])
    at = torch.where(there, s.tokens, 0)
    if kind == "logprob":
        most = z.amax(1)
        e = (z - most[:, None]).exp()
        total = e.sum(1)
        lse = most + total.log()
        logprob = torch.where(there, z.gather(1, at[:, None])[:, 0] - lse, 0.0)
        entropy = None
        if case["entropy"]:
            entropy = total.log() - torch.where(e > 0, e * (z - most[:, None]), 0.0).sum(1) / total
        ids = top = None
        if case["top"]:
            top, ids = torch.sort(s.logits.float(), dim=1, descending=True, stable=True)
            top, ids = top[:, :case["top"]] * case["scale"] - lse[:, None], ids[:, :case["top"]]
        return {"logprob": logprob, "lse": lse, "entropy": entropy, "top_ids": ids, "top": top}
    log_p = z - s.lse[:, None]
    p = log_p.exp()
    g = torch.where(there, s.g, 0.0)
    d = -g[:, None] * p
    d.scatter_add_(1, at[:, None], g[:, None])
    if s.ge is not None:
        d = d - s.ge[:, None] * torch.where(p > 0, p * (log_p + s.entropy[:, None]), 0.0)
    return (d * case["scale"]).to(s.out.dtype)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------


def _product(a, b):
    """a b^T in 64 bits, some rows at a time."""
    b = b.double().t().contiguous()
    out = torch.empty((a.shape[0], b.shape[1]), dtype=torch.float64, device=DEV)
    for r0 in range(0, a.shape[0], 2048):
        torch.mm(a[r0:r0 + 2048].double(), b, out=out[r0:r0 + 2048])
    return out


def _normal_cdf(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def _exact_act(z, act, grad):
    """An activation, or its slope."""
    if act == "none":
        return torch.ones_like(z) if grad else z
    if act == "relu":
        return (z > 0).double() if grad else z.clamp(min=0)
    if act == "silu":
        p = torch.sigmoid(z)
        return p + z * p * torch.sigmoid(-z) if grad else z * p
    if act == "gelu":
        p = _normal_cdf(z)
        return p + z * torch.exp(-z ** 2 / 2) / math.sqrt(2 * math.pi) if grad else z * p
    u = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)                             # (1 + tanh(u / 2)) / 2 is the logistic function of u
    p = torch.sigmoid(u)
    return p + z * p * torch.sigmoid(-u) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z ** 2) if grad else z * p


def _exact_turn(x, s, back):
    """x [rows, heads, dim] in 64 bits: pairs as complex numbers, times e^(i angle)."""
    case = s.case
    rot, at = case["rot"], 0
    parts = []
    for axis, pairs in enumerate(s.sections):
        parts.append(s.positions[axis].double()[:, None] * s.freqs[at:at + pairs].double())
        at += pairs
    angle = torch.cat(parts, 1)
    turn = torch.polar(torch.ones_like(angle), -angle if back else angle)[:, None]
    part = x[..., :rot].unflatten(2, (rot // 2, 2)) if case["neighbours"] else x[..., :rot].unflatten(2, (2, rot // 2)).transpose(2, 3)
    z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
    z = z if case["neighbours"] else z.transpose(2, 3)
    return torch.cat([z.flatten(2), x[..., rot:]], 2)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "linear":
        z = _product(s.x, s.weight)
        if s.bias is not None:
            z += s.bias.double()
        y = _exact_act(z, case["act"], False)
        return {"out": y if s.residual is None else y + s.residual.double(), "pre": None if s.pre is None else z}
    if kind == "linear_grad":
        dz = s.grad.double()
        if s.pre is not None:
            dz = dz * _exact_act(s.pre.double(), case["act"], True)
        gw, gb = torch.mm(dz.t().contiguous(), s.x.double()), torch.mv(dz.t(), torch.ones(case["rows"], dtype=torch.float64, device=DEV))
        if case["add"]:
            gw += s.gw.double()
            if s.gb is not None:
                gb = gb + s.gb.double()
        return {"x": torch.mm(dz, s.weight.double()), "weight": gw, "bias": None if s.gb is None else gb}
    if kind.startswith("rotate"):
        out = {}
        for name in ("q", "k"):
            x, w = getattr(s, name).double(), getattr(s, "w" + name)
            rms = (torch.linalg.vector_norm(x, dim=2, keepdim=True) ** 2 / case["dim"] + EPS) ** 0.5
            if kind == "rotate":
                out[name] = _exact_turn(x / rms * w.double() if case["norm"] else x, s, False)
                continue
            g = _exact_turn(getattr(s, "g" + name).double(), s, True)
            out[name], out[name + "_weight"] = g, None
            if case["norm"]:
                unit = x / rms
                out[name + "_weight"] = (g * unit).flatten(0, 1).sum(0)
                g = g * w.double()
                out[name] = (g - unit * (g * unit).sum(2, keepdim=True) / case["dim"]) / rms
        return {name: out[name] for name in (("q", "k") if kind == "rotate" else ("q", "k", "q_weight", "k_weight"))}
    z = s.logits.double() * case["scale"]
    held = torch.nonzero(s.tokens >= 0)[:, 0]
    if kind == "logprob":
        log_p = torch.log_softmax(z, 1)
        best = z.argmax(1)
        lse = (z - log_p).gather(1, best[:, None])[:, 0]
        logprob = torch.zeros(case["rows"], dtype=torch.float64, device=DEV)
        logprob[held] = log_p[held, s.tokens[held]]
        entropy = torch.special.entr(log_p.exp()).sum(1) if case["entropy"] else None
        return {"logprob": logprob, "lse": lse, "entropy": entropy, "top_ids": None, "top": log_p.sort(1, descending=True)[0][:, :case["top"]] if case["top"] else None}
    p = (z - s.lse.double()[:, None]).exp()
    g = torch.zeros(case["rows"], dtype=torch.float64, device=DEV)
    g[held] = s.g.double()[held]
    d = p * -g[:, None]
    d[held, s.tokens[held]] += g[held]
    if s.ge is not None:
        d += s.ge.double()[:, None] * (torch.special.entr(p) - p * s.entropy.double()[:, None])
    return d * case["scale"]


# ---- what a pass cannot do without ------------------------------------------------------------------------------------


def work(case):
    kind, rows, size = case["kind"], case["rows"], SIZE[case["type"]]
    if kind == "linear":
        k, n, out = case["k"], case["n"], SIZE[case["out"]]
        bytes = (rows + n) * k * size + rows * n * (out * (1 + case["residual"]) + size * case["pre"]) + n * size * case["bias"]
        return {"bytes": bytes, "flops": 2.0 * rows * k * n}
    if kind == "linear_grad":
        k, n = case["k"], case["n"]
        bytes = (2 * rows + n) * k * size + n * k * SIZE[case["wtype"]] * (1 + case["add"]) + rows * n * size * (1 + (case["act"] != "none"))
        return {"bytes": bytes + 4 * n * case["bias"] * (1 + case["add"]), "flops": 4.0 * rows * k * n}
    if kind.startswith("rotate"):
        n, back = rows * (case["heads"] + case["kv"]) * case["dim"], kind == "rotate_grad"
        vectors = 2 * case["dim"] * (size + 4 * back) * case["norm"] + 2 * case["rot"]
        return {"bytes": n * size * (3 if back and case["norm"] else 2) + 8 * rows * case["axes"] + vectors, "flops": (10.0 if back else 7.0) * n}
    n = rows * case["vocab"]
    if kind == "logprob":
        return {"bytes": n * size + rows * (8 + 8 + 4 * case["entropy"] + 12 * case["top"]), "flops": 4.0 * n}
    return {"bytes": 2 * n * size + rows * (8 + 8 + 8 * case["entropy"]), "flops": 5.0 * n}
