"""The LM head over 4-bit weights against 64 bits, its layout, its quantisation, and steps over it.

Tolerance of a logit, u = 2^-24.  Products of bf16 numbers are exact in fp32.  Within a group of up to 256 weights the sums of
h (16 + q) and of h are chains of additions; then two fused multiply-adds per group, and one addition per part of k.  Taken as
independent roundings with a margin of 4: 4 u sqrt(d) times sum |h| s (16 + q + 16 + o), and 4 u sqrt(groups) of sum |h| s |q - o|.
The guidance mix multiplies by 1 + 2 lambda and rounds three times, tau once more."""
import math

import numpy as np
import pytest
import torch

from oracle import scd as oscd
from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _weights(V, d, group, zeros, seed, wide=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    G = -(-d // group)
    codes = torch.randint(0, 256, (V, d // 2), device="cuda", generator=g, dtype=torch.uint8)
    scales = (0.01 * torch.exp(torch.randn(V, G, device="cuda", generator=g))).to(torch.bfloat16)
    zp = torch.randint(0, 16, (V, G), device="cuda", generator=g, dtype=torch.uint8) if zeros else None
    return codes, scales, zp


def _unpacked(codes, scales, zp, group, lo, hi):
    """q, s, o of rows lo..hi, one per weight, in 64 bits."""
    codes = codes[lo:hi].long()
    q = torch.stack([codes & 15, codes >> 4], 2).reshape(hi - lo, -1).double()
    d = q.shape[1]
    at = torch.arange(d, device="cuda") // group
    s = scales[lo:hi].double()[:, at]
    o = zp[lo:hi].double()[:, at] if zp is not None else torch.full_like(q, 8.0)
    return q, s, o


def _want(h, q, s, o, lam, tau, groups):
    """h [B, C, L, d] -> z [B, L, n] and its bound."""
    h = h.double()
    a = h @ (s * (q - o)).t()
    size = h.abs() @ (s * (32 + q + o)).t() * (4 * U * math.sqrt(h.shape[-1])) + h.abs() @ (s * (q - o).abs()).t() * (4 * U * math.sqrt(groups))
    if lam:
        z = (1 + lam) * a[:, 0] - lam * a[:, 1]
        b = (1 + lam) * (size[:, 0] + 2 * U * a[:, 0].abs()) + lam * (size[:, 1] + 2 * U * a[:, 1].abs())
    else:
        z, b = a[:, 0], size[:, 0]
    return z / tau, b / tau + 3 * U * z.abs() / tau


CASES = [  # B, L, lam, V, v_lo, n, d, group, zeros, tau
    (1, 1, 0.0, 1, 0, 1, 32, 32, False, 1.0), (1, 1, 0.0, 40, 3, 33, 8, 32, True, 1.0), (1, 1, 3.0, 100, 0, 100, 64, 64, False, 1.0),
    (1, 5, 0.0, 300, 7, 257, 200, 32, True, 0.5), (1, 8, 2.0, 70, 1, 64, 136, 96, True, 1.0), (2, 20, 3.0, 515, 5, 510, 264, 128, False, 0.9),
    (1, 33, 0.0, 200, 0, 199, 1288, 64, True, 1.0), (3, 32, 3.0, 1000, 40, 900, 520, 32, False, 1.0), (1, 64, 0.0, 31, 0, 31, 4096, 256, True, 1.0),
    (5, 26, 0.0, 1285, 0, 1285, 1304, 1280, False, 1.0), (1, 32, 3.0, 33000, 3, 32900, 192, 64, True, 1.0),
    (1, 9, 0.0, 66000, 100, 65800, 72, 32, False, 1.0), (4, 40, 1.5, 34000, 0, 33333, 96, 96, True, 2.0), (1, 32, 3.0, 66000, 0, 66000, 1024, 32, True, 1.0),
    (1, 2, 0.0, 70000, 0, 70000, 2048, 32, True, 1.0), (2, 17, 3.0, 260, 0, 256, 8192, 32, True, 1.0), (1, 60, 0.0, 65600, 9, 65555, 256, 160, False, 1.0),
    # many rows: tiles of 256 rows of h, by groups of whole and of half blocks, the last row tile ragged, and with scales that do not fit
    (4, 33, 3.0, 700, 2, 645, 328, 64, True, 1.0), (9, 31, 3.0, 300, 0, 300, 136, 128, False, 0.8), (3, 64, 0.0, 515, 0, 500, 712, 192, True, 1.0),
    (2, 150, 0.0, 200, 10, 130, 200, 32, False, 1.0), (1, 129, 0.0, 64, 0, 64, 64, 64, True, 1.0), (5, 30, 2.0, 260, 0, 259, 7000, 32, True, 1.0)]


@pytest.mark.parametrize("Bn,L,lam,V,v_lo,n,d,group,zeros,tau", CASES)
def test_logits(Bn, L, lam, V, v_lo, n, d, group, zeros, tau):
    C = 2 if lam else 1
    s = B.Scd(B.make_config(B=Bn, L=L, N=L, V=V, d=d, v_lo=v_lo, v_hi=v_lo + n, cfg_lambda=lam, temperature=tau))
    codes, scales, zp = _weights(V, d, group, zeros, seed=n + d)
    h = torch.randn(Bn, C, L, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
    packed = s.pack_quantized(codes, scales, zp, group)
    guard = torch.full((Bn * L + 2, n), 7.0, device="cuda")
    z = guard[1:-1].view(Bn, L, n)
    s.lm_head_quantized(h, packed, z)
    want, bound = _want(h, *_unpacked(codes, scales, zp, group, v_lo, v_lo + n), lam, tau, -(-d // group))
    err = (z.double() - want).abs()
    assert (err <= bound).all(), (err / bound).max().item()
    assert (guard[0] == 7).all() and (guard[-1] == 7).all()
    again = torch.empty_like(z)
    s.lm_head_quantized(h, packed, again)
    assert torch.equal(z, again)


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False)])
def test_one_position_at_a_time_places_every_weight(group, zeros):
    """h with a single one: a logit is one weight, exactly."""
    V, d = 70, 200
    s = B.Scd(B.make_config(B=1, L=d, N=d, V=V, d=d))
    codes, scales, zp = _weights(V, d, group, zeros, seed=9)
    z = torch.empty(1, d, V, device="cuda")
    s.lm_head_quantized(torch.eye(d, device="cuda").to(torch.bfloat16), s.pack_quantized(codes, scales, zp, group), z)
    q, sc, o = _unpacked(codes, scales, zp, group, 0, V)
    assert torch.equal(z[0].double(), (sc * (q - o)).t())


def test_rows_that_are_not_finite_stay_by_themselves():
    V, d, L = 300, 136, 40
    s = B.Scd(B.make_config(B=1, L=L, N=L, V=V, d=d))
    codes, scales, zp = _weights(V, d, 64, True, seed=2)
    packed = s.pack_quantized(codes, scales, zp, 64)
    h = torch.randn(1, 1, L, d, device="cuda").to(torch.bfloat16)
    z, clean = torch.empty(L, V, device="cuda"), torch.empty(L, V, device="cuda")
    s.lm_head_quantized(h, packed, clean)
    h[0, 0, 3, 135], h[0, 0, 33, 0] = math.nan, math.inf
    s.lm_head_quantized(h, packed, z)
    keep = torch.tensor([r not in (3, 33) for r in range(L)], device="cuda")
    assert torch.equal(z[keep], clean[keep]) and not z[~keep].isfinite().any()


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("V,d,group", [(5, 8, 32), (40, 200, 64), (33, 1288, 96), (100, 512, 128)])
def test_quantize(V, d, group, zeros):
    """Codes are the nearest under the rounded scale; a weight inside the range is off by half a step, and one outside it by
    what rounding the scale cuts off: 2^-8 of 8 (or 15) steps."""
    g = torch.Generator(device="cuda").manual_seed(V)
    W = torch.randn(V, d, device="cuda", generator=g).to(torch.bfloat16)
    W[0] = 0
    W[1, :d // 2] = W[1, :d // 2].abs()
    G = -(-d // group)
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=V, d=d))
    codes = torch.empty(V, d // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(V, G, dtype=torch.bfloat16, device="cuda")
    zp = torch.empty(V, G, dtype=torch.uint8, device="cuda") if zeros else None
    s.quantize(W, group, codes, scales, zp)
    q, sc, o = _unpacked(codes, scales, zp, group, 0, V)
    pad = G * group - d
    grouped = torch.nn.functional.pad(W.double(), (0, pad)).view(V, G, group)
    lo, hi = grouped.amin(2).clamp(max=0), grouped.amax(2).clamp(min=0)
    step = (hi - lo) / 15 if zeros else torch.maximum(hi / 7, -lo / 8)
    assert ((scales.double() - step).abs() <= step * (2.0 ** -8 + 2.0 ** -22)).all()
    if zeros:
        assert ((zp.double() * scales.double() + lo).abs() <= scales.double() * (0.5 + 15 * 2.0 ** -7)).all()
    err = (sc * (q - o) - W.double()).abs()
    assert (err <= sc * (0.5 + 15 * 2.0 ** -7 + (0.5 if zeros else 0.0))).all()
    # the nearest of the sixteen
    levels = sc[..., None] * (torch.arange(16, device="cuda").double() - o[..., None])
    best = (levels - W.double()[..., None]).abs().amin(2)
    assert (err <= best + sc * 1e-6).all()
    assert (q[0] == o[0]).all()


@pytest.mark.parametrize("kw,group,zeros", [
    (dict(B=1, L=32, N=150, V=1100, v_lo=4, v_hi=1028, d=256, top_k=200, cfg_lambda=3.0), 64, True),      # short rows
    (dict(B=2, L=16, N=60, V=20000, d=128, top_k=500, temperature=0.9), 32, False),                        # lists of long rows
    (dict(B=3, L=20, N=47, V=6000, v_lo=7, v_hi=5900, d=192, top_k=300, top_p=0.9), 96, True)])
def test_steps_decode_as_over_supplied_logits(kw, group, zeros):
    """A decode over 4-bit weights against the oracle, which is given the kernel's own logits of every step."""
    s = B.Scd(B.make_config(seed=5, **kw))
    c, n = s.cfg, s.n
    W = s.pack_quantized(*_weights(c.V, c.d, group, zeros, seed=4), group)
    o = oscd.ScdOracle(oscd.ScdConfig(B=c.B, L=c.L, N=c.N, V=c.V, v_lo=c.v_lo, v_hi=c.v_hi, top_k=c.top_k, temperature=1.0,
                                      cfg_lambda=0.0, seed=5, top_p=kw.get("top_p", 0.0)))
    g = torch.Generator(device="cuda").manual_seed(8)
    st = s.alloc_state()
    s.reset(st)
    z = torch.empty(c.B, c.L, n, device="cuda")
    base = torch.randn(c.B, s.C, c.N + c.L, c.d, device="cuda", generator=g) * 2
    for _ in range(12):
        pos = s.state_field(st, B.F_POS).tolist()
        h = torch.stack([base[b, :, p:p + c.L] for b, p in enumerate(pos)]).contiguous()
        h = (h + 0.2 * torch.randn(h.shape, device="cuda", generator=g)).to(torch.bfloat16)
        s.lm_head_quantized(h, W, z)
        t = int(s.state_field(st, B.F_ITER).max())
        s.step_quantized(h, W, st)
        # the same logits as the stage's, in the ring slots of the live positions
        ring = s.state_field(st, B.F_Z).view(2, c.B, c.L, n)[t & 1]
        for b, p in enumerate(pos):
            for k in range(min(c.L, c.N - p)):
                assert torch.equal(ring[b, (p + k) % c.L], z[b, k]), (b, k)
        zs = z.cpu().numpy()
        o.step([zs[b, :o.window(b)[1]] if o.window(b)[1] else None for b in range(c.B)])
        assert s.status(st)[0] == B.SCD_OK
        assert np.array_equal(s.state_field(st, B.F_POS).cpu().numpy(), np.asarray([o.window(b)[0] for b in range(c.B)]))
        assert np.array_equal(s.state_field(st, B.F_OUT).cpu().numpy().reshape(c.B, c.N), o.out)


def test_captured_step_replays():
    kw = dict(B=1, L=32, N=200, V=3000, d=320, top_k=100)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        s = B.Scd(B.make_config(seed=3, **kw), stream=st)
    W = s.pack_quantized(*_weights(3000, 320, 64, True, seed=1), 64)
    h = torch.randn(1, 1, 32, 320, device="cuda").to(torch.bfloat16)
    eager, state = s.alloc_state().zero_(), s.alloc_state().zero_()      # (halves that no step has written yet)
    s.reset(eager)
    s.reset(state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        s.step_quantized(h, W, state)
    for _ in range(4):
        h.copy_(torch.randn(1, 1, 32, 320, device="cuda"))
        torch.cuda.synchronize()
        s.step_quantized(h, W, eager)
        graph.replay()
        torch.cuda.synchronize()
        for f in (B.F_OUT, B.F_POS, B.F_X, B.F_LSE, B.F_ITER):
            assert torch.equal(s.state_field(eager, f), s.state_field(state, f)), f
