"""The largest numbers of ids that the operators on the vocabulary table take.

A loss of rows that all ids share alike is log(n): exact but for the sum of n equal terms, the logarithm and the result's rounding."""
import math

import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("rows", [1, 130])
def test_cross_entropy_over_2_30_ids(rows):
    """W is zero but for its last row, 20.75 e_0, and h = e_0: the last id is about as likely as all others together, and dh is
    (p_last - [t = last]) W_last."""
    n, d = 1 << 30, 8
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=n, d=d))
    W = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    W[-1, 0] = 20.75                                        # log(2^30) = 20.794
    h = torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda")
    h[:, 0] = 1
    t = torch.full((rows,), n - 1, dtype=torch.int32, device="cuda")
    t[0] = 5
    loss, lse = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    s.cross_entropy(h, W, t, loss, lse, s.cross_entropy_workspace(rows))
    want = math.log(n - 1 + math.exp(20.75))
    assert ((lse.double() - want).abs() <= 64 * U * want).all()
    expected = torch.full((rows,), want - 20.75, dtype=torch.float64, device="cuda")
    expected[0] = want
    assert ((loss.double() - expected).abs() <= 64 * U * want).all()
    dh = torch.full_like(h, 7.0)
    s.cross_entropy_backward(h, W, t, lse, None, dh, None, s.cross_entropy_backward_workspace(rows))
    last = math.exp(20.75 - want)
    wanted = torch.full((rows,), (last - 1) * 20.75, dtype=torch.float64, device="cuda")
    wanted[0] = last * 20.75
    # p to 64 u (1 + z) of itself, 2^-11 of dz, 2^-8 of the result; zero columns stay zero
    assert ((dh[:, 0].double() - wanted).abs() <= wanted.abs() * (2.0 ** -8 + 2.0 ** -10)).all()
    assert not dh[:, 1:].any()


def test_a_packed_table_of_64_gib():
    """2^37 codes: those of the first and the last rows are where they belong (logits of whole numbers, exact)."""
    n, d = 1 << 30, 128
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 150 GiB")
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=n, d=d))
    codes = torch.full((n, d // 2), 0x88, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for at in (0, n // 2, n - 40):
        codes[at:at + 40] = torch.randint(0, 256, (40, d // 2), device="cuda", generator=g, dtype=torch.uint8)
    W = s.pack_quantized(codes, torch.ones(n, 1, dtype=torch.bfloat16, device="cuda"), None, 128)
    h = torch.randint(-8, 9, (1, 1, 1, d), device="cuda", generator=g).to(torch.bfloat16)
    z = torch.full((1, 1, n), 7.0, device="cuda")
    s.lm_head_quantized(h, W, z)
    q = lambda at: torch.stack([codes[at:at + 40] & 15, codes[at:at + 40] >> 4], 2).reshape(40, d).double() - 8  # noqa: E731
    for at in (0, n // 2, n - 40):
        assert torch.equal(z[0, 0, at:at + 40].double(), q(at) @ h[0, 0, 0].double()), at
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    for at in (0, n // 2, n - 40):
        rest[at:at + 40] = False
    assert not z[0, 0, rest].any()
    del codes, W, z, rest
    torch.cuda.empty_cache()
