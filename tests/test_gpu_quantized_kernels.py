"""Every instance of the LM head over 4-bit weights against 64 bits; the tolerance is the one derived in test_gpu_quantized."""
import pytest
import torch

from paper_2510_24211_amd import binding as B
from quantized_shapes import SHAPES, config, name
from test_gpu_quantized import _unpacked, _want, _weights

pytestmark = pytest.mark.gpu


def _check(shape, s):
    _, _, zeros, sequences, window, n, d, group = shape
    c = s.cfg
    codes, scales, zp = _weights(c.V, d, group, zeros, seed=n + d)
    h = torch.randn(sequences, s.C, window, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(d)).to(torch.bfloat16)
    guard = torch.full((sequences * window + 2, n), 7.0, device="cuda")
    z = guard[1:-1].view(sequences, window, n)
    packed = s.pack_quantized(codes, scales, zp, group)
    s.lm_head_quantized(h, packed, z)
    want, bound = _want(h, *_unpacked(codes, scales, zp, group, c.v_lo, c.v_hi), c.cfg_lambda, c.temperature, -(-d // group))
    err = (z.double() - want).abs()
    assert (err <= bound).all(), (err / bound).max().item()
    assert (guard[0] == 7).all() and (guard[-1] == 7).all()
    for _ in range(2):
        again = torch.empty_like(z)
        s.lm_head_quantized(h, packed, again)
        assert torch.equal(z, again)


@pytest.mark.parametrize("shape", SHAPES, ids=name)
def test_logits_of_the_instance(shape):
    s = B.Scd(config(B.make_config, shape))
    assert s.lm_head_quantized_kernel_name(shape[-1], shape[2]) == name(shape)
    _check(shape, s)


# (one wavefront per tile on groups of whole blocks: only where long rows' scales leave no room for two tiles)
@pytest.mark.parametrize("shape", [s for s in SHAPES if not (s[0].endswith("1, 8, 1, 160, 1") and s[1] == 4)], ids=name)
def test_short_rows_of_the_instance(shape):
    """One step of k to more than the stages hold, with parts of k of one length and with a block less in some; where the instance serves them."""
    share_k, ran = int(shape[0].split(", ")[5]), 0
    for steps in range(1, 10):
        for d in {64 * share_k * steps - 40, 64 * (share_k * (steps - 1) + 1), 64 * share_k * steps - 72}:
            short = (*shape[:6], d, shape[7])
            s = B.Scd(config(B.make_config, short)) if d > 0 else None
            if s and s.lm_head_quantized_kernel_name(shape[-1], shape[2]) == name(shape):
                _check(short, s)
                ran += 1
    assert ran >= 20, ran
