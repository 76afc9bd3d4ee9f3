"""Embedding lookup and its gradient against 64 bits.

Tolerances.  Lookup: a float32 product (2^-24) rounded to bf16 (2^-8 of the value).  Gradient: m terms added up in fp32 one
after another, at most m roundings of 2^-24 of the partial sums, which are at most the sum of the magnitudes; the product with
the scale, and the rounding to the result's type (half a step) of the value."""
import math

import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
V0 = 1000


def _ctx(V, d, **kw):
    return B.Scd(B.make_config(**dict(dict(B=1, L=1, N=1, V=V, d=d), **kw)))


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("rows,V,d,scale", [(1, 1, 8, 1.0), (3, 7, 16, -2.5), (64, 1000, 1280, 35.8), (5, 50, 4104, 0.125),
                                            (1000, 333, 520, 1.0), (130, 70000, 64, 8.0), (0, 10, 8, 1.0)])
def test_lookup(rows, V, d, scale):
    g = _gen(rows + V)
    W = torch.randn(V, d, device="cuda", generator=g).to(torch.bfloat16)
    ids = torch.randint(0, V, (rows,), device="cuda", generator=g, dtype=torch.int32)
    if rows >= 3:
        ids[0], ids[1], ids[2] = -1, V, V - 1
    guard = torch.full((rows + 2, d), 7.0, dtype=torch.bfloat16, device="cuda")
    x = guard[1:rows + 1]
    _ctx(V, d).embed(ids, W, scale, x)
    there = (ids >= 0) & (ids < V)
    want = torch.where(there[:, None], W.double()[ids.clamp(0, V - 1).long()] * scale, 0.0)
    assert ((x.double() - want).abs() <= want.abs() * (HALF[torch.bfloat16] + 2.0 ** -23)).all()
    assert (guard[0] == 7).all() and (guard[-1] == 7).all()


def test_lookup_keeps_infinities_and_nan():
    W = torch.zeros(4, 8, device="cuda", dtype=torch.bfloat16)
    W[1, 3], W[2, 0], W[3, 7] = math.inf, math.nan, -math.inf
    x = torch.empty(4, 8, device="cuda", dtype=torch.bfloat16)
    _ctx(4, 8).embed(torch.arange(4, device="cuda", dtype=torch.int32), W, 2.0, x)
    assert torch.equal(x.float().nan_to_num(9.0), W.float().nan_to_num(9.0))


def _tokens(kind, rows, V, g):
    if kind == "one":
        return torch.full((rows,), V // 2, device="cuda", dtype=torch.int32)
    if kind == "none":
        return torch.full((rows,), -1, device="cuda", dtype=torch.int32)
    if kind == "distinct":
        return torch.randperm(V, device="cuda", generator=g)[:rows].to(torch.int32)
    if kind == "last":
        return torch.full((rows,), V - 1, device="cuda", dtype=torch.int32)
    ids = (torch.rand(rows, device="cuda", generator=g) ** 3 * V).int().clamp(max=V - 1)
    r = torch.rand(rows, device="cuda", generator=g)
    ids = torch.where(r < 0.3, V // 3, ids)
    return torch.where(r > 0.95, torch.where(r > 0.97, V + 5, -3), ids).to(torch.int32)


def _gradient(ids, dx, scale, V, old=None):
    """In 64 bits, with the bound on what 32-bit sums may be off."""
    there = (ids >= 0) & (ids < V)
    i = ids[there].long()
    want = torch.zeros(V, dx.shape[1], dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    want.index_add_(0, i, dx[there].double())
    size.index_add_(0, i, dx[there].double().abs())
    count = torch.bincount(i, minlength=V)[:, None].double()
    want, size = want * scale, size * abs(scale)
    bound = (count + 3) * 2.0 ** -24 * size
    if old is not None:
        want = want + old.double()
        bound = bound + 2.0 ** -24 * (want.abs() + old.double().abs())
    return want, bound


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind,rows,V,d", [
    ("mixed", 1, 5, 8), ("mixed", 2, 1, 8), ("mixed", 33, 100, 24), ("mixed", 576, 16384, 1280), ("one", 8192, 40, 64),
    ("one", 8193, 600, 16), ("none", 70, 30, 8), ("distinct", 3000, 3001, 512), ("last", 100, 65, 520),
    ("mixed", 8191, 513, 1032), ("mixed", 20011, 70001, 72), ("mixed", 70000, 300000, 8), ("mixed", 12000, 511, 136),
    ("mixed", 0, 130, 16), ("one", 100000, 3, 24), ("distinct", 65, 64 * 3 + 1, 4104)])
def test_gradient(kind, rows, V, d, accumulate, dtype):
    if kind == "distinct":
        rows = min(rows, V)
    g = _gen(rows * 7 + V)
    ids = _tokens(kind, rows, V, g)
    dx = torch.randn(rows, d, device="cuda", generator=g).to(torch.bfloat16)
    out = (ids < 0) | (ids >= V)
    dx[out] = math.nan                                   # rows that do not count may hold anything
    scale = 1.7
    old = torch.randn(V, d, device="cuda", generator=g).to(dtype)
    guard = torch.full((V + 2, d), 7.0, dtype=dtype, device="cuda")
    dW = guard[1:V + 1]
    dW.copy_(old)
    s = _ctx(V, d)
    ws = s.embed_backward_workspace(rows).fill_(0xA5)
    s.embed_backward(ids, dx, scale, dW, ws, accumulate)
    want, bound = _gradient(ids, dx.nan_to_num(0.0), scale, V, old if accumulate else None)
    assert ((dW.double() - want).abs() <= bound + HALF[dtype] * (want.abs() + bound)).all()
    assert (guard[0] == 7).all() and (guard[-1] == 7).all()
    if accumulate:
        untouched = torch.bincount(ids[~out].long(), minlength=V) == 0
        assert torch.equal(dW[untouched], old[untouched])


def test_gradient_is_the_lookup_s_transpose():
    """<embed(W), dx> = <W, embed_backward(dx)> for every W: here for one entry of W at a time, by differences."""
    V, d, rows, scale = 9, 16, 40, 0.5
    g = _gen(3)
    ids = _tokens("mixed", rows, V, g)
    dx = torch.randint(-4, 5, (rows, d), device="cuda", generator=g).to(torch.bfloat16)
    s = _ctx(V, d)
    dW = torch.empty(V, d, device="cuda")
    s.embed_backward(ids, dx, scale, dW, s.embed_backward_workspace(rows))
    x0, x1 = (torch.empty(rows, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    W = torch.zeros(V, d, device="cuda", dtype=torch.bfloat16)
    s.embed(ids, W, scale, x0)
    for v in range(V):
        for k in (0, 7, 15):
            W.zero_()
            W[v, k] = 2.0
            s.embed(ids, W, scale, x1)
            diff = ((x1.double() - x0.double()) * dx.double()).sum() / 2.0
            assert diff == dW[v, k].double()              # small whole numbers: exact


def test_gradient_is_run_to_run_identical_and_graphs_replay():
    V, d, rows = 5000, 264, 30000
    g = _gen(11)
    ids = _tokens("mixed", rows, V, g)
    dx = torch.randn(rows, d, device="cuda", generator=g).to(torch.bfloat16)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        s = B.Scd(B.make_config(B=1, L=1, N=1, V=V, d=d), stream=st)
    dW, first = torch.empty(V, d, device="cuda"), torch.empty(V, d, device="cuda")
    ws = s.embed_backward_workspace(rows)
    torch.cuda.synchronize()
    s.embed_backward(ids, dx, 1.0, first, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        s.embed_backward(ids, dx, 1.0, dW, ws)
    for turn in range(4):
        if turn == 2:                                      # new ids in the recorded call's buffers
            ids.copy_(_tokens("mixed", rows, V, g))
            torch.cuda.synchronize()
            s.embed_backward(ids, dx, 1.0, first, ws)
            torch.cuda.synchronize()
        dW.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dW, first)
        assert torch.randn(1000, device="cuda").sum().isfinite()      # work of the program's own between the replays


@pytest.mark.parametrize("kw", [dict(B=3, L=20, N=47, V=500, v_lo=9, v_hi=410, cfg_lambda=2.0),
                                dict(B=1, L=32, N=20, V=64), dict(B=2, L=1, N=5, V=300, v_lo=250)])
def test_window_reads_the_drafts_of_the_state(kw):
    d, scale = 72, 3.0
    s = _ctx(kw["V"], d, **{k: v for k, v in kw.items() if k != "V"})
    c, n, C = s.cfg, s.n, s.C
    g = _gen(5)
    W = torch.randn(c.V, d, device="cuda", generator=g).to(torch.bfloat16)
    st = s.alloc_state()
    s.reset(st)
    x = torch.full((c.B, C, c.L, d), 7.0, device="cuda", dtype=torch.bfloat16)
    ref = torch.empty_like(x)
    for _ in range(6):
        s.embed_window(st, W, scale, x)
        pos = s.state_field(st, B.F_POS).tolist()
        X = s.state_field(st, B.F_X).view(c.B, c.L).tolist()
        ids = torch.tensor([[[c.v_lo + X[b][(pos[b] + k) % c.L] if pos[b] + k < c.N else -1 for k in range(c.L)]
                             for _ in range(C)] for b in range(c.B)], dtype=torch.int32, device="cuda")
        s.embed(ids, W, scale, ref)
        assert torch.equal(x, ref)
        s.step_logits(torch.randn(c.B, c.L, n, device="cuda", generator=g), st)
    assert s.status(st)[0] == B.SCD_OK
