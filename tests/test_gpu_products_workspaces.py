"""Products and gradients that use no workspace go without one, also while they are recorded; those that use one get by with exactly what they ask for."""

import numpy as np
import pytest
import torch

from lm_util import U32, UNIT, TINY, assert_within, f64, rows_of
from paper_2101_11714_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DEV = "cuda:0"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def hold(got, a, b, n, what):
    """got: a b, with sums of n terms in 32 bits."""
    a, b = a.double(), b.double()
    want, mag = (a @ b).cpu().numpy(), (a.abs() @ b.abs()).cpu().numpy()
    off, t = 2 * (n + 4) * U32 * mag, got.dtype
    assert_within(got, want, off + UNIT[t] * (np.abs(want) + off) + TINY[t], what)


@pytest.mark.parametrize("type", [F32, BF16, F16])
def test_recorded_calls_without_a_workspace_where_none_is_used(type):
    g = gen(1)
    rows, K, N = 4096, 1024, 4096
    assert B.linear_fwd_workspace_bytes(rows, K, N, type, True) > 0              # (fewer rows would have parts)
    x, w, y = rows_of(g, rows, K, type), rows_of(g, N, K, type, 0, 0, K ** -0.5), torch.empty((rows, N), dtype=type, device=DEV)
    x, w = x.contiguous(), w.contiguous()
    B.tt_linear_fwd(x, w, y)
    want = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.tt_linear_fwd(x, w, y)
    for i in range(3):
        y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i
    hold(y[:64], x[:64], w.t(), K, "out")


def asked(call):
    """The bytes that a call without a workspace asks for while it is recorded."""
    graph = torch.cuda.CUDAGraph()
    try:
        with torch.cuda.graph(graph):
            call(None)
    except B.TTError as e:
        assert e.code == -4
        return int(str(e).split("workspace of ")[1].split(" bytes")[0])
    return 0


@pytest.mark.parametrize("rows,K,N", [(100, 4096, 64), (700, 2048, 520), (700, 2047, 521), (260, 16384, 264), (2049, 136, 2047), (130, 5001, 70), (46, 1425, 495)])
@pytest.mark.parametrize("type", [F32, BF16, F16])
def test_workspaces_of_what_a_call_asks_for(rows, K, N, type):
    g = gen(rows)
    x, w, dy = rows_of(g, rows, K, type), rows_of(g, N, K, type, 0, 0, K ** -0.5), rows_of(g, rows, N, type)
    y, dx, dw, db = (torch.empty(s, dtype=t, device=DEV) for s, t in (((rows, N), type), ((rows, K), type), ((N, K), F32), (N, F32)))
    for name, call, most in [("out", lambda ws: B.tt_linear_fwd(x, w, y, workspace=ws), B.linear_fwd_workspace_bytes(rows, K, N, type)),
                             ("gradients", lambda ws: B.tt_linear_bwd(dy, x, w, dx, dw, grad_bias=db, workspace=ws), B.linear_bwd_workspace_bytes(rows, K, N, type))]:
        size = asked(call)
        assert size <= most
        mem = torch.full((size + 1024,), 255, dtype=torch.uint8, device=DEV)
        call(mem[:size] if size else None)
        assert bool((mem[size:] == 255).all()), name
        if size:
            with pytest.raises(B.TTError) as e:
                call(mem[:size - 256])
            assert e.value.code == -4
    hold(y, x, w.t(), K, "out")
    hold(dx, dy, w, N, "x")
    hold(dw, dy.t(), x, rows, "weight")
    hold(db[None], torch.ones((1, rows), device=DEV), dy, rows, "bias")
