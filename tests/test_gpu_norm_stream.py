"""Norm and gradient together, from x and the residual on, through a bf16 stream, against 64 bits."""
import pytest
import torch

from test_gpu_norm import BF, EPS, F32, HALF, U, _chain, _ctx, _gen, _grad_want, _inputs, _randn, _want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d", [(64, 136), (515, 1288), (40, 4096), (20, 8200)])
@pytest.mark.parametrize("grad", [BF, F32])
def test_gradient_behind_a_bf16_stream(rows, d, grad):
    """Norm and gradient as they are used together, from x and the residual on: the gradient reads the stream, s rounded by at most half a step, e = 2^-8 of
    it, while inv is the unrounded sum's.  dx = inv (a - s inv^2 mean(a s)) + ds is then off by inv^3 e |s| (|mean(a s)| + (1 + e) mean |a s|)
    at most, a term dy s inv of the gains by e of its size, besides what the arithmetic does (with s and its errors larger by 1 + e)."""
    e = 2.0 ** -8
    x, r, g = _inputs(rows, d, BF, BF, seed=rows + d)
    s = _ctx(d)
    total, inv = torch.empty_like(r), torch.empty(rows, device="cuda")
    s.norm(x, g, torch.empty_like(x), EPS, residual=r, sum=total, inv=inv)
    q = _gen(5)
    dy, ds = _randn(q, rows, d).to(BF), _randn(q, rows, d).to(grad)
    dx, dgain = torch.empty(rows, d, device="cuda", dtype=grad), torch.empty(d, device="cuda")
    s.norm_backward(total, g, inv, dy, dx, dgain, s.norm_backward_workspace(rows), dsum=ds)
    s64, inv64, _ = _want(x, r, g)
    wdx, off, wdg, goff = _grad_want(s64, g, inv64, dy, ds)
    a, i = g.double() * dy.double(), inv64[:, None]
    mean, size = (a * s64).mean(1, keepdim=True), (a * s64).abs().mean(1, keepdim=True)
    # inv itself is off by (chain / 2 + 14) u, which dx has to the third power
    off = (1 + e) ** 2 * (off + 3 * (_chain(d) / 2 + 14) * U * i * (a.abs() + s64.abs() * i * i * size))
    off = off + i ** 3 * e * s64.abs() * (mean.abs() + (1 + e) * size)
    assert ((dx.double() - wdx).abs() <= off + HALF[grad] * (wdx.abs() + off)).all()
    goff = (1 + e) * goff + (e + (_chain(d) / 2 + 16) * U) * (dy.double() * s64 * i).abs().sum(0)
    assert ((dgain.double() - wdg).abs() <= goff + U * (wdg.abs() + goff)).all()
