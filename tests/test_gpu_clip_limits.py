"""Clipping under an infinite norm with any max_norm, and where max_norm / norm is below the normal numbers of fp32.

Tolerance as of the other clipping: factor and product one rounding of 2^-24 each, a step of the output's type, half of its smallest one."""
import math

import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: U}
STEP = {BF: 2.0 ** -134, F32: 2.0 ** -150}


def _ctx():
    return B.Scd(B.make_config(B=1, L=1, N=1, V=1))


@pytest.mark.parametrize("most", [math.inf, 1.0, 0.0])
@pytest.mark.parametrize("place", [False, True])
def test_an_infinite_norm_leaves_zeros(most, place):
    s = _ctx()
    g = [torch.ones(20000, device="cuda"), torch.full((9,), -2.0, device="cuda", dtype=BF)]
    g[0][7], g[1][3] = math.inf, -math.inf
    ts = B.TensorList(g)
    norm = torch.empty(1, device="cuda")
    s.gradient_norm(ts, norm, s.gradient_norm_workspace(ts))
    assert norm.item() == math.inf
    out = g if place else [torch.full_like(t, 9.0) for t in g]
    s.clip_gradients(ts, B.TensorList(out), most, norm)
    for t, at in zip(out, (7, 3)):
        rest = torch.cat([t[:at], t[at + 1:]])
        assert t[at].isnan() and (rest == 0).all()


@pytest.mark.parametrize("place", [False, True])
def test_no_limit_on_a_finite_norm_leaves_gradients_as_they_are(place):
    s = _ctx()
    g = [torch.randn(20000, device="cuda"), torch.randn(9, device="cuda").to(BF)]
    ts = B.TensorList(g)
    norm = torch.empty(1, device="cuda")
    s.gradient_norm(ts, norm, s.gradient_norm_workspace(ts))
    was = [t.clone() for t in g]
    out = g if place else [torch.full_like(t, 9.0) for t in g]
    s.clip_gradients(ts, B.TensorList(out), math.inf, norm)
    assert all(torch.equal(a, b) for a, b in zip(out, was))
    norm.fill_(math.nan)
    s.clip_gradients(ts, B.TensorList(out), math.inf, norm)
    assert all(t.isnan().all() for t in out)


# factors below 2^-126, of 2^-149 and less, and of a max_norm that is itself below the normal numbers
@pytest.mark.parametrize("most,norm", [(1e-3, 1e37), (1e-5, 3e38), (2.0 ** -20, 2.0 ** 110), (2.0 ** -140, 3.0), (2.0 ** -149, 1e-30), (3 * 2.0 ** -149, 1e-35),
                                       (1e-12, 3e38), (1.0, 2.0 ** 97), (0.0, 2.0 ** -149), (1.0, 1e20)])
@pytest.mark.parametrize("types", [(F32, F32), (F32, BF), (BF, BF), (BF, F32)])
def test_factors_below_the_normal_numbers(most, norm, types):
    s = _ctx()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(17003, device="cuda", generator=g) * torch.exp2(torch.randint(-140, 126, (17003,), device="cuda", generator=g).float())
    x = x.to(types[0])
    have = torch.full((1,), norm, device="cuda")
    out = torch.full((17003,), 9.0, device="cuda").to(types[1])
    s.clip_gradients(B.TensorList([x]), B.TensorList([out]), most, have)
    most = torch.tensor(most, dtype=F32).double().item()
    want = x.double() * (most / have.double().item())
    assert ((out.double() - want).abs() <= (HALF[types[1]] + 4 * U) * want.abs() + STEP[types[1]]).all()
