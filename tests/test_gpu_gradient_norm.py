"""The norm of many gradients and their clipping against 64 bits.

Squares are added up in 64 bits and the root is rounded to fp32 once: u of the norm (and 2^-40 for the sums).  The factor is one
division more, the product one more: 3 u, then half a step of the output's type, or half of its smallest step."""
import math

import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: U}
STEP = {BF: 2.0 ** -134, F32: 2.0 ** -150}


def _ctx(**kw):
    return B.Scd(B.make_config(B=1, L=1, N=1, V=1), **kw)


def _norm(s, grads):
    ts = B.TensorList(grads)
    out, ws = torch.full((1,), math.nan, device="cuda"), s.gradient_norm_workspace(ts)
    s.gradient_norm(ts, out, ws)
    return ts, out, ws


def _views(sizes, dtypes, seed, scale=1.0):
    """Neighbouring pieces of one buffer per type: beginnings at every alignment that elements have."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    made = []
    flat = {t: (scale * torch.randn(sum(sizes) + 8, device="cuda", generator=g)).to(t) for t in set(dtypes)}
    at = 1
    for n, t in zip(sizes, dtypes):
        made.append(flat[t][at:at + n])
        at += n
    return made


SETS = [([1], [BF]), ([7, 1, 9], [BF, F32, BF]), ([8191, 8192, 8193, 3], [F32, BF, BF, F32]), ([0, 5, 0, 100000, 0], [BF, F32, F32, BF, BF]),
        ([1288 * 77, 1288, 3, 40001], [F32] * 4), ([11 + i for i in range(333)], [BF if i % 3 else F32 for i in range(333)]),
        ([16411 * 1288, 1288], [BF, BF]), ([0, 0], [F32, BF]), ([], [])]


@pytest.mark.parametrize("k", range(len(SETS)))
def test_norm_and_clipping(k):
    sizes, types = SETS[k]
    s = _ctx()
    grads = _views(sizes, types, seed=k)
    ts, norm, ws = _norm(s, grads)
    want = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
    assert abs(norm.item() - want) <= (U + 2.0 ** -40) * want
    for most in (0.37 * want, want * 2 + 1, 0.0):
        by = min(1.0, most / want) if want else 1.0
        for types_out in (types, [F32] * len(types), [BF] * len(types)):
            out = _views(sizes, types_out, seed=100)
            ends = [torch.as_strided(t, (1,), (1,), t.storage_offset() + t.numel()).clone() for t in out]
            os_ = B.TensorList(out)
            s.clip_gradients(ts, os_, most, norm)
            for g, o in zip(grads, out):
                w = g.double() * by
                assert ((o.double() - w).abs() <= (HALF[o.dtype] + 4 * U) * w.abs() + STEP[o.dtype]).all()
            if out:                                        # what lies behind the last tensor of the largest buffer
                assert torch.equal(torch.as_strided(out[-1], (1,), (1,), out[-1].storage_offset() + out[-1].numel()), ends[-1])
        place = [g.clone() for g in grads]
        ps = B.TensorList(place)
        s.clip_gradients(ps, ps, most, norm)
        out = [torch.empty_like(g) for g in grads]
        s.clip_gradients(ts, B.TensorList(out), most, norm)
        assert all(torch.equal(p, o) for p, o in zip(place, out))
    again = torch.empty(1, device="cuda")
    s.gradient_norm(ts, again, ws)
    assert torch.equal(again, norm)


def test_squares_beyond_the_range_of_32_bits():
    s = _ctx()
    for size in (1e30, 1e-30):
        g = [torch.full((9000,), size, device="cuda"), torch.full((5,), -size, device="cuda", dtype=BF)]
        _, norm, _ = _norm(s, g)
        want = math.sqrt(sum(float(t.double().square().sum()) for t in g))
        assert abs(norm.item() - want) <= 2 * U * want


def test_what_is_not_finite():
    s = _ctx()
    g = [torch.ones(10, device="cuda"), torch.tensor([math.inf, 2.0], device="cuda", dtype=BF)]
    ts, norm, _ = _norm(s, g)
    assert norm.item() == math.inf
    out = [torch.full_like(t, 9.0) for t in g]
    s.clip_gradients(ts, B.TensorList(out), 1.0, norm)
    assert (out[0] == 0).all() and out[1][0].isnan() and out[1][1] == 0
    g[0][4] = math.nan
    ts, norm, _ = _norm(s, g)
    assert norm.isnan().all()
    s.clip_gradients(ts, B.TensorList(out), 1.0, norm)
    assert out[0].isnan().all() and out[1].isnan().all()
    # any norm that the caller has: of several machines' gradients
    norm.fill_(4.0)
    s.clip_gradients(B.TensorList([torch.ones(3, device="cuda")]), B.TensorList([o := torch.empty(3, device="cuda")]), 1.0, norm)
    assert (o == 0.25).all()


def test_captured_with_a_workspace_each():
    st = torch.cuda.Stream()
    s = _ctx(stream=st)
    sets = [_views(*SETS[i], seed=i) for i in (2, 5)]
    lists = [B.TensorList(x) for x in sets]
    outs = [[torch.empty_like(t) for t in x] for x in sets]
    onto = [B.TensorList(x) for x in outs]
    spaces, norms = [s.gradient_norm_workspace(x) for x in lists], torch.empty(2, device="cuda")
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            s.gradient_norm(lists[i], norms[i:], spaces[i])
            s.clip_gradients(lists[i], onto[i], 1.0, norms[i:])
        graphs.append(graph)
    for turn in range(3):
        for t in sum(sets, []):
            t.mul_(2.0)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for i in range(2):
            want = math.sqrt(sum(float(t.double().square().sum()) for t in sets[i]))
            assert abs(norms[i].item() - want) <= 2 * U * want
            for g, o in zip(sets[i], outs[i]):
                w = g.double() / want
                assert ((o.double() - w).abs() <= (HALF[o.dtype] + 4 * U) * w.abs() + STEP[o.dtype]).all()
        assert torch.randn(1000, device="cuda").sum().isfinite()
