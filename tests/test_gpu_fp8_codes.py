"""e4m3 codes are the quotients value / scale in fp32, to the nearest and, at a border of two codes, to the even one.

No tolerance: the scale is one division, the quotient one more, and a product that leaves the value is repeated here in the same fp32 steps.
Quotients are formed in 64 bits and rounded to 32: two roundings of a quotient of 24-bit numbers, the first to 53 >= 2 * 24 + 2 bits, are as one."""
import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
BF, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def _codes(v, scale):
    q = (v.double() / scale.double()).float()
    return torch.where(scale == 0, 0.0, q).to(E4M3).float()


def _scale(most):
    return torch.where(most < 448 * 2.0 ** -126, 0.0, (most.double() / 448).float())


def _pairs(exponent):
    """[128, 128, 128]: block g has the largest value (1 + g / 128) 2^exponent, and every other bf16 value of 64 binades below it, of both signs:
    all pairs of digits that a quotient of bf16 numbers can have."""
    j = torch.arange(128, device="cuda", dtype=torch.float64)
    most = (1 + j / 128)[:, None] * 2.0 ** exponent
    b = torch.arange(64, device="cuda", dtype=torch.float64)
    v = ((1 + j / 128)[None, :] * 2.0 ** (exponent - b)[:, None]).reshape(1, -1)
    v = torch.where(v > most, most, v)
    v = torch.cat([v, -v], 1)
    v[:, 127] = most[:, 0]
    return v.view(128, 128, 128).to(BF)


@pytest.mark.parametrize("exponent", [0, -4, 100, 127, -80, -110, -117, -118, -126])
def test_every_quotient_of_weights(exponent):
    W = _pairs(exponent).view(128 * 128, 128)
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=len(W), d=128))
    codes, scales = torch.empty(len(W), 128, device="cuda", dtype=E4M3), torch.empty(128, 1, device="cuda")
    s.quantize_fp8(W, codes, scales)
    want = _scale(W.float().abs().view(128, -1).amax(1))
    assert torch.equal(scales[:, 0], want)
    want = _codes(W.float(), want.repeat_interleave(128)[:, None])
    assert torch.equal(codes.float(), want), (codes.float() != want).sum().item()


@pytest.mark.parametrize("V,d", [(2560, 2560), (130, 144)])
def test_random_weights(V, d):
    W = (0.02 * torch.randn(V, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(V))).to(BF)
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=V, d=d))
    codes, scales = torch.empty(V, d, device="cuda", dtype=E4M3), torch.empty(-(-V // 128), -(-d // 128), device="cuda")
    s.quantize_fp8(W, codes, scales)
    wide = scales.repeat_interleave(128, 0)[:V].repeat_interleave(128, 1)[:, :d]
    assert torch.equal(codes.float(), _codes(W.float(), wide))


@pytest.mark.parametrize("d", [512, 1024, 2048, 4096, 8192, 128 * 128 * 128])
@pytest.mark.parametrize("exponent", [0, -60, -117])
def test_every_quotient_of_normed_rows(exponent, d):
    """Rows of ones have a norm of 1 exactly (eps is lost beside it), so the gains are what is stored in 8 bits."""
    pairs = _pairs(exponent)
    blocks = pairs.reshape(-1, 128).clone()
    blocks[:, 0] = pairs.float().amax((1, 2)).to(BF).repeat_interleave(128)             # each 128 of a row with the block's largest
    gain = blocks.reshape(-1)
    if d < gain.numel():                                                                # some of all pairs for every length of rows
        start = torch.randperm(len(blocks), generator=torch.Generator().manual_seed(d))[:d // 128]
        gain = blocks[start.to("cuda")].reshape(-1)
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=1, d=d))
    x, inv = torch.ones(3, d, device="cuda", dtype=BF), torch.empty(3, device="cuda")
    codes, scales = torch.empty(3, d, device="cuda", dtype=E4M3), torch.empty(3, d // 128, device="cuda")
    s.norm_fp8(x, gain, codes, scales, 1e-30, inv=inv)
    assert (inv == 1).all()
    want = _scale(gain.float().view(-1, 128).abs().amax(1))
    assert torch.equal(scales, want.expand(3, -1))
    want = _codes(gain.float(), want.repeat_interleave(128))
    assert torch.equal(codes.float(), want.expand(3, -1)), (codes.float() != want).sum().item()


@pytest.mark.parametrize("rows,d", [(300, 136), (300, 1288), (100, 4096), (20, 9000)])
def test_random_rows(rows, d):
    g = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(rows, d, device="cuda", generator=g).to(BF)
    r, gain = torch.randn(rows, d, device="cuda", generator=g), 1 + 0.3 * torch.randn(d, device="cuda", generator=g)
    G = -(-d // 128)
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=1, d=d))
    codes, scales, inv = torch.empty(rows, d, device="cuda", dtype=E4M3), torch.empty(rows, G, device="cuda"), torch.empty(rows, device="cuda")
    s.norm_fp8(x, gain, codes, scales, 1e-6, residual=r, inv=inv)
    y = (x.float() + r) * inv[:, None] * gain
    most = torch.nn.functional.pad(y, (0, G * 128 - d)).view(rows, G, 128).abs().amax(2)
    assert torch.equal(scales, _scale(most))
    assert torch.equal(codes.float(), _codes(y, scales.repeat_interleave(128, 1)[:, :d]))
