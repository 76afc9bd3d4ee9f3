"""The LM head over 8-bit rows and weights against 64 bits, the table's quantisation, steps over it, and a run from the norm on.

Tolerance of a logit, u = 2^-24.  Products of e4m3 numbers are exact in fp32.  Within a block of 128 their sum is a chain of additions; then
the block's scale (one rounding) and a fused multiply-add.  Taken as independent roundings with a margin of 4: 4 u (sqrt(128) + sqrt(blocks) + 2)
of sum |h| |W| with their scales.  The guidance mix multiplies by 1 + 2 lambda and rounds three times, tau once more."""
import math

import numpy as np
import pytest
import torch

from fp8_shapes import CASES, MORE
from oracle import scd as oscd
from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _codes(g, *shape):
    return (100 * torch.randn(*shape, device="cuda", generator=g)).clamp(-448, 448).to(E4M3)


def _scales(g, *shape):
    return 0.01 * torch.exp(torch.randn(*shape, device="cuda", generator=g))


def _table(V, d, seed):
    g = _gen(seed)
    return _codes(g, V, d), _scales(g, -(-V // 128), -(-d // 128))


def _rows(c, C, seed):
    g = _gen(seed)
    return _codes(g, c.B, C, c.L, c.d), _scales(g, c.B, C, c.L, -(-c.d // 128))


def _wide(codes, scales):
    return codes.double() * scales.double().repeat_interleave(128, -1)[..., :codes.shape[-1]]


def _want(h, hs, W, Ws, c):
    """z [B, L, n] in 64 bits and its bound."""
    v = torch.arange(c.v_lo, c.v_hi, device="cuda")
    w = _wide(W[c.v_lo:c.v_hi], Ws[v // 128])
    h = _wide(h, hs)
    a = h @ w.t()
    size = h.abs() @ w.abs().t() * (4 * U * (math.sqrt(128) + math.sqrt(hs.shape[-1]) + 2))
    lam, tau = c.cfg_lambda, c.temperature
    if lam:
        z = (1 + lam) * a[:, 0] - lam * a[:, 1]
        b = (1 + lam) * (size[:, 0] + 2 * U * a[:, 0].abs()) + lam * (size[:, 1] + 2 * U * a[:, 1].abs())
    else:
        z, b = a[:, 0], size[:, 0]
    return z / tau, b / tau + 3 * U * z.abs() / tau


@pytest.mark.parametrize("Bn,L,lam,V,v_lo,n,d,tau", CASES + MORE)
def test_logits(Bn, L, lam, V, v_lo, n, d, tau):
    s = B.Scd(B.make_config(B=Bn, L=L, N=L, V=V, d=d, v_lo=v_lo, v_hi=v_lo + n, cfg_lambda=lam, temperature=tau))
    W, Ws = _table(V, d, seed=n + d)
    h, hs = _rows(s.cfg, s.C, seed=1)
    guard = torch.full((Bn * L + 2, n), 7.0, device="cuda")
    z = guard[1:-1].view(Bn, L, n)
    s.lm_head_fp8(h, hs, W, Ws, z)
    want, bound = _want(h, hs, W, Ws, s.cfg)
    err = (z.double() - want).abs()
    assert (err <= bound).all(), (err / bound).max().item()
    assert (guard[0] == 7).all() and (guard[-1] == 7).all()
    again = torch.empty_like(z)
    s.lm_head_fp8(h, hs, W, Ws, again)
    assert torch.equal(again, z)


@pytest.mark.parametrize("L,lam,d", [(1, 0.0, 400), (40, 2.0, 272), (256, 0.0, 144)])
def test_one_position_at_a_time_places_every_weight(L, lam, d):
    """Rows that are 1 at one k and 0 elsewhere read a column of the table back, scales and all."""
    n, lo = 300, 100
    s = B.Scd(B.make_config(B=1, L=L, N=L, V=lo + n, d=d, v_lo=lo, cfg_lambda=lam))
    W, Ws = _table(lo + n, d, seed=2)
    wide = (W.float() * Ws.repeat_interleave(128, 0)[:lo + n].repeat_interleave(128, 1)[:, :d])[lo:]
    hs = torch.ones(1, s.C, L, -(-d // 128), device="cuda")
    z = torch.empty(1, L, n, device="cuda")
    for first in range(0, d, L):
        h = torch.zeros(1, s.C, L, d, device="cuda")
        for k in range(min(L, d - first)):
            h[0, 0, k, first + k] = 1.0
        s.lm_head_fp8(h.to(E4M3), hs, W, Ws, z)
        for k in range(min(L, d - first)):
            assert torch.equal(z[0, k], (1 + lam) * wide[:, first + k] if lam else wide[:, first + k]), first + k


@pytest.mark.parametrize("Bn,L,lam", [(1, 6, 0.0), (4, 40, 2.0)])
def test_rows_that_are_not_finite_stay_by_themselves(Bn, L, lam):
    V, d = 400, 272
    s = B.Scd(B.make_config(B=Bn, L=L, N=L, V=V, d=d, cfg_lambda=lam))
    W, Ws = _table(V, d, seed=3)
    h, hs = _rows(s.cfg, s.C, seed=4)
    z, w = torch.empty(Bn, L, V, device="cuda"), torch.empty(Bn, L, V, device="cuda")
    s.lm_head_fp8(h, hs, W, Ws, z)
    bad, bad_s = h.clone().float(), hs.clone()
    bad[0, 0, 1, 270], bad_s[0, 0, 3, 1] = math.nan, math.nan
    bad_s[-1, 0, 5] = 0.0                                           # padding
    s.lm_head_fp8(bad.to(E4M3), bad_s, W, Ws, w)
    assert w[0, 1].isnan().all() and w[0, 3].isnan().all()
    same = torch.ones(Bn, L, dtype=torch.bool, device="cuda")
    same[0, 1] = same[0, 3] = same[-1, 5] = False
    assert torch.equal(w[same], z[same]) and (lam != 0 or (w[-1, 5] == 0).all())
    # an id whose weights are not finite: its column alone
    spoilt = W.float()
    spoilt[130, 0] = math.nan
    s.lm_head_fp8(h, hs, spoilt.to(E4M3), Ws, w)
    keep = torch.arange(V, device="cuda") != 130
    assert w[..., 130].isnan().all() and torch.equal(w[..., keep], z[..., keep])


@pytest.mark.parametrize("V,d", [(1, 16), (130, 144), (300, 1296), (129, 4096)])
def test_quantize(V, d):
    g = _gen(V)
    W = (torch.randn(V, d, device="cuda", generator=g) * torch.exp(torch.randn(V, 1, device="cuda", generator=g))).to(BF)
    W[0] = 0.0
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=V, d=d))
    R, G = -(-V // 128), -(-d // 128)
    codes, scales = torch.empty(V, d, device="cuda", dtype=E4M3), torch.empty(R, G, device="cuda")
    s.quantize_fp8(W, codes, scales)
    pad = torch.nn.functional.pad(W.double(), (0, G * 128 - d, 0, R * 128 - V)).view(R, 128, G, 128)
    most = pad.abs().amax((1, 3))
    assert ((scales.double() - most / 448).abs() <= U * most / 448).all()
    v = (pad / (most / 448).clamp(min=1e-300)[:, None, :, None]).reshape(R * 128, G * 128)[:V, :d]
    assert ((codes.double() - v).abs() <= (2.0 ** -4 + 6 * U) * v.abs() + 2.0 ** -10 * (1 + 1e-6)).all()


@pytest.mark.parametrize("kw", [dict(B=1, L=16, N=40, V=1000, v_lo=130, v_hi=935, d=272, top_k=100), dict(B=3, L=8, N=20, V=700, d=144),
                                dict(B=2, L=20, N=47, V=20000, d=128, top_k=500)])
def test_steps_decode_as_over_supplied_logits(kw):
    """A decode over 8-bit weights against the oracle, which is given the kernel's own logits of every step."""
    s = B.Scd(B.make_config(seed=5, **kw))
    c, n = s.cfg, s.n
    W, Ws = _table(c.V, c.d, seed=4)
    Ws *= 0.002 / 0.01
    o = oscd.ScdOracle(oscd.ScdConfig(B=c.B, L=c.L, N=c.N, V=c.V, v_lo=c.v_lo, v_hi=c.v_hi, top_k=c.top_k, temperature=1.0, cfg_lambda=0.0, seed=5))
    g = _gen(8)
    st = s.alloc_state()
    s.reset(st)
    z = torch.empty(c.B, c.L, n, device="cuda")
    base = torch.randn(c.B, s.C, c.N + c.L, c.d, device="cuda", generator=g) * 2
    gain = torch.ones(c.d, device="cuda", dtype=BF)
    h = torch.empty(c.B, s.C, c.L, c.d, device="cuda", dtype=E4M3)
    hs = torch.empty(c.B, s.C, c.L, -(-c.d // 128), device="cuda")
    for _ in range(10):
        pos = s.state_field(st, B.F_POS).tolist()
        x = torch.stack([base[b, :, p:p + c.L] for b, p in enumerate(pos)]).contiguous()
        s.norm_fp8((x + 0.2 * torch.randn(x.shape, device="cuda", generator=g)).to(BF), gain, h, hs, 1e-6)
        s.lm_head_fp8(h, hs, W, Ws, z)
        t = int(s.state_field(st, B.F_ITER).max())
        s.step_fp8(h, hs, W, Ws, st)
        ring = s.state_field(st, B.F_Z).view(2, c.B, c.L, n)[t & 1]
        for b, p in enumerate(pos):
            for k in range(min(c.L, c.N - p)):
                assert torch.equal(ring[b, (p + k) % c.L], z[b, k]), (b, k)
        zs = z.cpu().numpy()
        o.step([zs[b, :o.window(b)[1]] if o.window(b)[1] else None for b in range(c.B)])
        assert s.status(st)[0] == B.SCD_OK
        assert np.array_equal(s.state_field(st, B.F_POS).cpu().numpy(), np.asarray([o.window(b)[0] for b in range(c.B)]))
        assert np.array_equal(s.state_field(st, B.F_OUT).cpu().numpy().reshape(c.B, c.N), o.out)


def test_captured_norm_and_step_replay():
    """The norm into 8 bits and the step behind it, recorded once on a stream of their own, against the same calls made eagerly."""
    cfg = dict(B=2, L=8, N=60, V=900, v_lo=5, d=272, top_k=50, cfg_lambda=2.0, seed=3)
    st = torch.cuda.Stream()
    s = B.Scd(B.make_config(**cfg), stream=st)
    W, Ws = _table(900, 272, seed=6)
    Ws *= 0.1
    g = _gen(7)
    x, gain = torch.empty(2, 2, 8, 272, device="cuda", dtype=BF), torch.ones(272, device="cuda")
    h, hs = torch.empty(2, 2, 8, 272, device="cuda", dtype=E4M3), torch.empty(2, 2, 8, 3, device="cuda")
    state, other = s.alloc_state(), s.alloc_state()
    torch.cuda.synchronize()
    s.reset(state)
    s.reset(other)
    graph = torch.cuda.CUDAGraph()

    def both(to):
        s.norm_fp8(x, gain, h, hs, 1e-6)
        s.step_fp8(h, hs, W, Ws, to)

    with torch.cuda.graph(graph, stream=st):
        both(state)
    for _ in range(5):
        x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        both(other)
        torch.cuda.synchronize()
        for f in (B.F_POS, B.F_OUT, B.F_X, B.F_Z):
            assert torch.equal(s.state_field(state, f), s.state_field(other, f))
    assert s.status(state)[0] == B.SCD_OK


def test_a_training_step_through_the_norm():
    """Rows -> norm -> cross entropy, and back to the table, the gains and the rows; the norm of all gradients; clipped copies.  Against
    64 bits, by autograd.  Steps between the calls are rounded to bf16, each to half a step of 2^-8: the gradients are within a few of
    those of their size (2-norm): at most 2^-8 for each of y, dy, dx and the tables' own rounding, together 4 * 2^-8."""
    rows, V, d = 150, 700, 264
    g = _gen(9)
    x = torch.randn(rows, d, device="cuda", generator=g).to(BF)
    gain = (1 + 0.2 * torch.randn(d, device="cuda", generator=g)).to(BF)
    W = (0.05 * torch.randn(V, d, device="cuda", generator=g)).to(BF)
    targets = torch.randint(0, V, (rows,), device="cuda", generator=g, dtype=torch.int32)
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=V, d=d))
    y, inv = torch.empty_like(x), torch.empty(rows, device="cuda")
    s.norm(x, gain, y, 1e-6, inv=inv)
    loss, lse, weight = (torch.empty(rows, device="cuda") for _ in range(3))
    weight.fill_(1.0 / rows)
    s.cross_entropy(y, W, targets, loss, lse, s.cross_entropy_workspace(rows))
    dy, dW = torch.empty_like(x), torch.empty(V, d, device="cuda")
    s.cross_entropy_backward(y, W, targets, lse, weight, dy, dW, s.cross_entropy_backward_workspace(rows, torch.float32))
    dx, dgain = torch.empty_like(x), torch.empty(d, device="cuda")
    s.norm_backward(x, gain, inv, dy, dx, dgain, s.norm_backward_workspace(rows))
    grads = B.TensorList([dW, dgain])
    norm, out = torch.empty(1, device="cuda"), [torch.empty_like(dW, dtype=BF), torch.empty_like(dgain)]
    s.gradient_norm(grads, norm, s.gradient_norm_workspace(grads))
    s.clip_gradients(grads, B.TensorList(out), 1e-3, norm)
    x64, g64, W64 = (t.detach().cpu().double().requires_grad_() for t in (x, gain, W))
    y64 = x64 / torch.sqrt(x64.square().mean(1, keepdim=True) + 1e-6) * g64
    torch.nn.functional.cross_entropy(y64 @ W64.t(), targets.cpu().long()).backward()
    near = lambda a, b: float((a.cpu().double() - b).norm() / b.norm()) <= 4 * 2.0 ** -8  # noqa: E731
    assert near(dx, x64.grad) and near(dgain, g64.grad) and near(dW, W64.grad)
    want = math.sqrt(float(W64.grad.square().sum() + g64.grad.square().sum()))
    assert abs(norm.item() - want) <= 4 * 2.0 ** -8 * want
    assert near(out[0], W64.grad * (1e-3 / want)) and near(out[1], g64.grad * (1e-3 / want))
