"""Quantisation at the ends of bf16's range.

A scale is off by half a step of bf16, 2^-8 of it, and the two divisions by 2^-24 each; a weight then by half a step, half of one for the zero
point, and by what the rounding of the scale moves 15 steps."""
import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
LARGEST = torch.finfo(torch.bfloat16).max


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("size", [LARGEST, 1.0, 2.0 ** -100])
def test_quantize_over_the_whole_range(size, zeros):
    V, d, group = 6, 64, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    W = ((torch.rand(V, d, device="cuda", generator=g) * 2 - 1).to(torch.bfloat16).double() * size).to(torch.bfloat16)
    W[0, 0], W[0, 1] = size, -size                           # a range of twice the largest number
    W[1, :32], W[2, 32:] = size, -size
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=V, d=d))
    codes = torch.empty(V, d // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(V, 2, dtype=torch.bfloat16, device="cuda")
    zp = torch.empty(V, 2, dtype=torch.uint8, device="cuda") if zeros else None
    s.quantize(W, group, codes, scales, zp)
    q = torch.stack([codes & 15, codes >> 4], 2).reshape(V, d).double()
    sc = scales.double().repeat_interleave(group, 1)
    o = zp.double().repeat_interleave(group, 1) if zeros else 8.0
    w = W.double().view(V, 2, group)
    lo, hi = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
    step = (hi - lo) / 15 if zeros else torch.maximum(hi / 7, -lo / 8)
    assert ((scales.double() - step).abs() <= step * (2.0 ** -8 + 2.0 ** -22)).all()
    err = (sc * (q - o) - W.double()).abs()
    assert (err <= sc * (0.5 + 15 * 2.0 ** -7 + (0.5 if zeros else 0.0))).all()
