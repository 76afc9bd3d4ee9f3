"""The norm of hidden rows, its 8-bit output and its gradient against 64 bits.

Tolerances, u = 2^-24.  s is one fp32 addition (u of it).  A sum over a row is a chain of at most `chain` additions per thread and a tree of
13, of squares with one rounding each: 1 / sqrt of its mean is off by (chain + 16) / 2 u + 3 u, y = s inv gain by (chain / 2 + 14) u, each
relative.  bf16 adds half a step, 2^-8; a scale (two roundings more) and codes that are v / scale to 3 u, half a step of e4m3: 2^-4, or 2^-10
below its normal numbers.  The gradient's sums are taken as independent roundings with a margin of 4: 4 u sqrt(terms) of the terms' sizes."""
import math

import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: U}
EPS = 1e-5


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ctx(d, **kw):
    return B.Scd(B.make_config(B=1, L=1, N=1, V=1, d=d), **kw)


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _inputs(rows, d, res, gain, seed):
    g = _gen(seed)
    size = torch.exp(_randn(g, d)) * torch.exp(2 * _randn(g, rows, 1))
    size[rows // 2] = 0.0                                           # a row of zeros
    x = (0.3 * _randn(g, rows, d) * size).to(BF)
    r = (_randn(g, rows, d) * size).to(res) if res is not None else None
    return x, r, (1 + 0.5 * _randn(g, d)).to(gain)


def _chain(d):
    return max(4, d // 8 // 1024 + 1)


def _want(x, r, gain):
    s = x.double() + (r.double() if r is not None else 0.0)
    inv = 1 / torch.sqrt(s.square().mean(1) + EPS)
    return s, inv, s * inv[:, None] * gain.double()


def _guarded(rows, width, dtype, fill):
    """rows of an array between two rows that have to stay as they are."""
    whole = torch.full((rows + 2, width), fill, device="cuda", dtype=torch.float32).to(dtype)
    start = whole[1:1 + rows]
    return whole, start


# rows of every kernel's lengths and their borders; d = 24 has a ragged block of 128, 16392 and more are read twice
SHAPES = [(1, 8), (3, 24), (5, 128), (6, 136), (2, 504), (4, 512), (9, 520), (3, 1024), (5, 1032), (2, 1288), (2, 2048), (3, 2056), (2, 4096), (2, 4104),
          (3, 8192), (2, 8200), (2, 16392), (1, 70000), (1030, 64), (515, 1288)]
TYPES = [(None, BF), (BF, BF), (F32, BF), (BF, F32), (F32, F32), (None, F32)]


@pytest.mark.parametrize("rows,d", SHAPES)
def test_norm(rows, d):
    for k, (res, gain) in enumerate(TYPES):
        x, r, g = _inputs(rows, d, res, gain, seed=rows + d + k)
        s = _ctx(d)
        whole, y = _guarded(rows + 0, d, BF, 7.0)
        total = torch.full_like(r, math.nan) if r is not None else None
        inv = torch.full((rows,), math.nan, device="cuda")
        s.norm(x, g, y, EPS, residual=r, sum=total, inv=inv)
        ws, winv, wy = _want(x, r, g)
        off = _chain(d) / 2 + 14
        assert ((inv.double() - winv).abs() <= off * U * winv).all()
        assert ((y.double() - wy).abs() <= (2.0 ** -8 + off * U) * wy.abs()).all()
        if r is not None:
            assert ((total.double() - ws).abs() <= HALF[res] * 1.001 * ws.abs()).all()
            # in place, without what is not wanted
            again, stream = x.clone(), r.clone()
            s.norm(again, g, again, EPS, residual=stream, sum=stream)
            assert torch.equal(stream, total)
            s.norm(x, g, r2 := torch.empty_like(x), EPS, residual=r)
            assert torch.equal(r2, y)
        else:
            s.norm(x, g, again := x.clone(), EPS)
        assert torch.equal(again, y)
        assert (whole[0] == 7).all() and (whole[-1] == 7).all()


@pytest.mark.parametrize("rows,d", SHAPES)
def test_norm_fp8(rows, d):
    G = -(-d // 128)
    for k, (res, gain) in enumerate(TYPES):
        x, r, g = _inputs(rows, d, res, gain, seed=rows + d + k)
        s = _ctx(d)
        whole = torch.full((rows * d + 64,), 3.0, device="cuda").to(torch.float8_e4m3fn)
        codes = whole[32 - 32 % 16:][:rows * d].view(rows, d)
        guard, scales = _guarded(rows, G, F32, 7.0)
        total = torch.full_like(r, math.nan) if r is not None else None
        inv = torch.full((rows,), math.nan, device="cuda")
        s.norm_fp8(x, g, codes, scales, EPS, residual=r, sum=total, inv=inv)
        ws, winv, wy = _want(x, r, g)
        off = _chain(d) / 2 + 14
        pad = torch.nn.functional.pad(wy, (0, G * 128 - d)).view(rows, G, 128)
        most = pad.abs().amax(2)
        assert ((scales.double() - most / 448).abs() <= (off + 2) * U * most / 448).all()
        v = (pad / (most / 448).clamp(min=1e-300)[..., None]).view(rows, -1)[:, :d]
        err = (codes.double() - v).abs()
        assert (err <= (2.0 ** -4 + 2 * (off + 5) * U) * v.abs() + 2.0 ** -10 * (1 + 1e-5)).all(), err.max().item()
        assert ((inv.double() - winv).abs() <= off * U * winv).all()
        if r is not None:
            plain = torch.empty_like(r)
            s.norm(x, g, torch.empty_like(x), EPS, residual=r, sum=plain)
            assert torch.equal(plain, total)
        assert (guard[0] == 7).all() and (guard[-1] == 7).all()
        assert (whole[:32].float() == 3).all() and (whole[32 + rows * d:].float() == 3).all()


def test_codes_are_the_nearest():
    """gain 1 and rows whose norm is 1 by construction: codes of a block are its values over the scale, to the nearest and to even."""
    d = 128
    x = torch.linspace(-1, 1, d, device="cuda").repeat(4, 1)
    x[1] *= torch.linspace(0, 1, d, device="cuda") ** 4               # into the subnormal codes
    x = x.to(BF)
    s = _ctx(d)
    codes, scales = torch.empty(4, d, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(4, 1, device="cuda")
    inv = torch.empty(4, device="cuda")
    s.norm_fp8(x, torch.ones(d, device="cuda"), codes, scales, 1e-30, inv=inv)
    y = x.float() * inv[:, None]
    inverse = (1.0 / scales.double()).float()
    assert torch.equal(codes.float(), (y * inverse).to(torch.float8_e4m3fn).float())


@pytest.mark.parametrize("d", [64, 1032, 2304, 16392])
def test_rows_that_are_not_finite_stay_by_themselves(d):
    g = _gen(d)
    x = _randn(g, 6, d).to(BF)
    clean = x.clone()
    x[1, 3], x[3, d - 1], x[4, 0] = math.nan, math.inf, 3e38
    gain = torch.ones(d, device="cuda", dtype=BF)
    s = _ctx(d)
    y, z = torch.empty_like(x), torch.empty_like(x)
    s.norm(x, gain, y, EPS)
    s.norm(clean, gain, z, EPS)
    keep = [0, 2, 5]
    assert torch.equal(y[keep], z[keep])
    assert y[1].isnan().all() and y[3, d - 1].isnan() and (y[3, :d - 1] == 0).all()
    codes, scales = torch.empty(6, d, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(6, -(-d // 128), device="cuda")
    s.norm_fp8(x, gain, codes, scales, EPS)
    assert codes.float()[1].isnan().all() and scales[1].isnan().all()
    assert codes.float()[keep].isfinite().all() and scales[keep].isfinite().all()
    # a gain that is not finite: its block alone; one too small for a scale counts as zero
    big = gain.float()
    big[0] = math.inf
    s.norm_fp8(clean, big, codes, scales, EPS)
    assert scales[:, 0].isinf().all() and codes.float()[:, 0].isnan().all() and (codes.float()[:, 1:min(d, 128)] == 0).all()
    assert scales[:, 1:].isfinite().all() and codes.float()[:, 128:].isfinite().all()
    s.norm_fp8(clean, gain.float() * 1e-37, codes, scales, EPS)
    assert (scales == 0).all() and (codes.float() == 0).all()


def _grad_want(s, gain, inv, dy, ds):
    s, dy, inv, gain = s.double(), dy.double(), inv.double()[:, None], gain.double()
    a = gain * dy
    mean = (a * s).mean(1, keepdim=True)
    dx = inv * (a - s * inv * inv * mean) + (ds.double() if ds is not None else 0.0)
    d = s.shape[1]
    size = inv * (6 * U * a.abs() + s.abs() * inv * inv * (4 * U * math.sqrt(d + 40) * (a * s).abs().mean(1, keepdim=True) + 8 * U * mean.abs()))
    if ds is not None:
        size = size + 2 * U * ds.double().abs()
    terms = dy * s * inv
    return dx, size, terms.sum(0), 4 * U * math.sqrt(s.shape[0] + 40) * terms.abs().sum(0)


GRADS = [(BF, BF, BF, BF, True), (F32, BF, BF, F32, True), (F32, F32, F32, F32, False), (BF, F32, F32, BF, False), (BF, BF, BF, F32, False)]


@pytest.mark.parametrize("rows,d", SHAPES + [(4000, 72), (3100, 1032), (1700, 4096), (1600, 8200)])
def test_gradient(rows, d):
    for k, (stream, gain, grad, gain_grad, has_ds) in enumerate(GRADS):
        x, r, g = _inputs(rows, d, stream, gain, seed=rows + d + k)
        s = _ctx(d)
        total, inv = torch.empty_like(r), torch.empty(rows, device="cuda")
        s.norm(x, g, torch.empty_like(x), EPS, residual=r, sum=total, inv=inv)
        q = _gen(k)
        dy = _randn(q, rows, d).to(BF)
        ds = _randn(q, rows, d).to(grad) if has_ds else None
        whole, dx = _guarded(rows, d, grad, 7.0)
        dgain = torch.full((d,), math.nan, device="cuda").to(gain_grad)
        ws = s.norm_backward_workspace(rows)
        s.norm_backward(total, g, inv, dy, dx, dgain, ws, dsum=ds)
        wdx, off, wdg, goff = _grad_want(total, g, inv, dy, ds)
        assert ((dx.double() - wdx).abs() <= off + HALF[grad] * (wdx.abs() + off)).all(), ((dx.double() - wdx).abs() / (off + HALF[grad] * wdx.abs())).max()
        assert ((dgain.double() - wdg).abs() <= goff + HALF[gain_grad] * (wdg.abs() + goff)).all()
        assert (whole[0] == 7).all() and (whole[-1] == 7).all()
        # the same bits again, in place, added to what is there, and without the gains
        again = torch.full((d,), 2.0, device="cuda")
        place = ds.clone() if ds is not None else torch.empty_like(dx)
        s.norm_backward(total, g, inv, dy, place, again, ws, dsum=place if ds is not None else None, accumulate=True)
        assert torch.equal(place, dx)
        assert ((again.double() - 2 - wdg).abs() <= goff + U * (2 + wdg.abs() + goff)).all()
        if grad == BF:
            over = dy.clone()
            s.norm_backward(total, g, inv, over, over, None, ws, dsum=ds)
            assert torch.equal(over, dx)


def test_gradient_against_differences():
    """Along random directions, of the loss sum(y dy) with y in 64 bits: central differences, step 1e-4 of rows of size 1 (error about 1e-8),
    against fp32 gradients."""
    rows, d = 5, 200
    g = _gen(3)
    x = _randn(g, rows, d).to(BF)
    gain = (1 + 0.3 * _randn(g, d))
    dy = _randn(g, rows, d).to(BF)
    s = _ctx(d)
    inv = torch.empty(rows, device="cuda")
    s.norm(x, gain, torch.empty_like(x), EPS, inv=inv)
    dx, dgain = torch.empty(rows, d, device="cuda"), torch.empty(d, device="cuda")
    s.norm_backward(x, gain, inv, dy, dx, dgain, s.norm_backward_workspace(rows))

    def loss(x, gain):
        return (x / torch.sqrt(x.square().mean(1, keepdim=True) + EPS) * gain * dy.double()).sum()

    for _ in range(4):
        v, w, h = _randn(g, rows, d).double(), _randn(g, d).double(), 1e-4
        slope = (loss(x.double() + h * v, gain.double()) - loss(x.double() - h * v, gain.double())) / (2 * h)
        assert abs(slope - (dx.double() * v).sum()) <= 1e-5 * (dx.double() * v).abs().sum()
        slope = (loss(x.double(), gain.double() + h * w) - loss(x.double(), gain.double() - h * w)) / (2 * h)
        assert abs(slope - (dgain.double() * w).sum()) <= 1e-5 * (dgain.double() * w).abs().sum()


def test_no_rows():
    s = _ctx(64)
    none, gain = torch.empty(0, 64, device="cuda", dtype=BF), torch.ones(64, device="cuda", dtype=BF)
    s.norm(none, gain, none, EPS)
    s.norm_fp8(none, gain, torch.empty(0, 64, device="cuda", dtype=torch.uint8), torch.empty(0, 1, device="cuda"), EPS)
    ws, dgain = s.norm_backward_workspace(0), torch.full((64,), 5.0, device="cuda")
    s.norm_backward(none, gain, torch.empty(0, device="cuda"), none, none, dgain, ws, accumulate=True)
    assert (dgain == 5).all()
    s.norm_backward(none, gain, torch.empty(0, device="cuda"), none, none, dgain, ws)
    assert (dgain == 0).all()


def test_captured_on_another_stream_replays():
    rows, d = 700, 1288
    x, r, gain = _inputs(rows, d, F32, BF, seed=1)
    dy = _randn(_gen(2), rows, d).to(BF)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    s = _ctx(d, stream=st)
    G = -(-d // 128)
    codes, scales = torch.empty(rows, d, device="cuda", dtype=torch.uint8), torch.empty(rows, G, device="cuda")
    total, inv = torch.empty_like(r), torch.empty(rows, device="cuda")
    dx, dgain, ws = torch.empty(rows, d, device="cuda", dtype=BF), torch.empty(d, device="cuda"), s.norm_backward_workspace(rows)
    outs = (codes, scales, total, inv, dx, dgain)

    def both():
        s.norm_fp8(x, gain, codes, scales, EPS, residual=r, sum=total, inv=inv)
        s.norm_backward(total, gain, inv, dy, dx, dgain, ws)

    torch.cuda.synchronize()
    both()
    torch.cuda.synchronize()
    first = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        both()
    for turn in range(4):
        if turn == 2:                                      # other rows in the recorded calls' buffers
            x.copy_(x.flip(0))
            torch.cuda.synchronize()
            both()
            torch.cuda.synchronize()
            first = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, want in zip(outs, first):
            assert torch.equal(t, want)
        assert torch.randn(1000, device="cuda").sum().isfinite()
