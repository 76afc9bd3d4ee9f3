"""The fp32 gradient of the table where the gradients of the logits span many binary orders: rows of little weight, ids of little
probability.

Tolerance of dW[v, k] = sum_r dz[r, v] h[r, k], u = 2^-24, dz = c_r (p - [v = t]), c = weight / tau.  E: the largest error of a row's logits, d
products in one chain, independent roundings with a margin of 4.  p errs by p (2 E + 32 u (1 + |z|max)): its exponent by the
logit's and the normaliser's errors and by roundings of |z| log2(e).  The two fp16 terms of dz leave 2^-22 of it, or half a step of the
second, 2^-25 / 2^11 in the place of 2^14 of the power of two at or below the largest weight: 2^-50 c_max.  h in fp16 under a power of two errs
by 2^-39 of its largest element.  The sum over the rows is a chain of fp32 additions (4 sqrt(rows) u of the magnitudes, twice: one for each of the
terms), the result is rounded once.  The one subtraction: p - 1 of a target rounds once more, u of 1 before the weight."""
import math

import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("rows,n,d,light,accumulate", [(64, 3000, 64, 2.0 ** -20, False), (200, 900, 136, 2.0 ** -27, False),
                                                      (300, 17000, 264, 2.0 ** -16, True), (33, 500, 72, 1.0, False)])
def test_light_rows_and_unlikely_ids_keep_their_digits(rows, n, d, light, accumulate):
    g = torch.Generator(device="cuda").manual_seed(rows)
    W = torch.randn(n, d, device="cuda", generator=g).to(torch.bfloat16)
    # logits with a deviation of 6: probabilities from nearly 1 down to some 2^-60
    h = (torch.randn(rows, d, device="cuda", generator=g) * 6 / math.sqrt(d)).to(torch.bfloat16)
    t = torch.randint(0, n, (rows,), device="cuda", generator=g, dtype=torch.int32)
    w = torch.where(torch.arange(rows, device="cuda") == 0, 1.0, light)
    # the heavy row has no part in the second half of the columns of h: there the light rows are alone
    h[0, d // 2:] = 0
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=n, d=d))
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    s.cross_entropy(h, W, t, loss, lse, s.cross_entropy_workspace(rows))
    dW = torch.zeros(n, d, device="cuda")
    s.cross_entropy_backward(h, W, t, lse, w, None, dW, s.cross_entropy_backward_workspace(rows, torch.float32), accumulate)

    h, W, c = h.double(), W.double(), w.double()[:, None]
    z = h @ W.t()
    E = (h.abs() @ W.abs().t() * (4 * math.sqrt(d) * U) + 2 * U * z.abs()).amax(1, keepdim=True)
    zmax = z.abs().amax(1, keepdim=True)
    p = torch.softmax(z, 1)
    hot = torch.nn.functional.one_hot(t.long(), n).double()
    dz = c * (p - hot)
    want = dz.t() @ h
    e_dz = c * (p * (2 * E + 32 * U * (1 + zmax)) + hot * U) + dz.abs() * 2.0 ** -22 + 2.0 ** -50
    bound = e_dz.t() @ h.abs() + dz.abs().t() @ torch.full_like(h, 2.0 ** -39 * h.abs().max().item()) + \
        dz.abs().t() @ h.abs() * (8 * math.sqrt(rows) + 4) * U
    err, allowed = (dW.double() - want).abs(), bound + U * want.abs() + 2.0 ** -126
    assert (err <= allowed).all(), (err / allowed).max().item()
