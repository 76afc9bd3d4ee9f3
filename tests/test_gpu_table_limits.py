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


def _whole(g, *shape):
    """Small whole numbers: sums of them are exact in fp32, whatever the order."""
    return torch.randint(-3, 4, shape, device="cuda", generator=g).to(torch.bfloat16)


@pytest.mark.parametrize("rows,V,d", [(3, 5, 1 << 24), (1 << 25, 40, 8), (1000, (1 << 31) - 1, 8)])
def test_embedding_and_gradient_at_the_largest_sizes(rows, V, d):
    """Whole numbers: the looked-up rows times 2 and the gradient of as many rows of one id as there are (up to 2^24) are exact; bf16 rounds once."""
    g = torch.Generator(device="cuda").manual_seed(7)
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=V, d=d))
    ids = torch.randint(max(0, V - 700), V, (rows,), device="cuda", generator=g, dtype=torch.int32)
    ids[:3] = torch.tensor([0, V - 1, -1], dtype=torch.int32)
    low = max(0, V - 700)
    W = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    W[0], W[low:] = 3.0, _whole(g, V - low, d)
    x = torch.full((rows, d), 7.0, dtype=torch.bfloat16, device="cuda")
    s.embed(ids, W, 2.0, x)
    there = ids >= 0
    for a in range(0, rows, 1 << 22):
        b = min(a + (1 << 22), rows)
        want = torch.where(there[a:b, None], W[ids[a:b].clamp(min=0).long()] * 2, 0)
        assert torch.equal(x[a:b], want)
    dx = x.copy_(_whole(g, rows, d))
    dW = W.fill_(7.0)
    s.embed_backward(ids, dx, 1.0, dW, s.embed_backward_workspace(rows))
    want = torch.zeros(V - low, d, device="cuda")
    far = there & (ids >= low)
    want.index_add_(0, (ids[far] - low).long(), dx[far].float())
    assert torch.equal(dW[low:], want.to(torch.bfloat16))
    if low > 0:
        assert torch.equal(dW[0].float(), dx[0].float())
        for a in range(1, low, 1 << 28):
            assert not dW[a:min(a + (1 << 28), low)].any()
    del W, x, dx, dW
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,n,d", [(3, 40, 1 << 21), (130, 300, 1 << 21), (1 << 20, 70, 8), (1 << 20, 300, 72)])
def test_cross_entropy_at_the_largest_sizes(rows, n, d):
    """Rows that hold one number each: h_r = a_r e_(k_r), so that a logit is one product, W has whole numbers / 2, and
    the gradients are dh_r = (p - hot) W and dW = (p - hot)^T h.  dz errs by p times twice the logits' and lse's errors (64 u (1 + |z|)) and by
    2^-11 of itself or 2^-39 of 1; sums in one chain of `rows` or n terms with a margin of 4; the result by half a step."""
    g = torch.Generator(device="cuda").manual_seed(rows + d)
    s = B.Scd(B.make_config(B=1, L=1, N=1, V=n, d=d))
    W = (_whole(g, n, d).float() / 2).to(torch.bfloat16)
    k = torch.randint(0, d, (rows,), device="cuda", generator=g)
    k[0], k[-1] = d - 1, 0
    h = torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda")
    r = torch.arange(rows, device="cuda")
    h[r, k] = _whole(g, rows)
    a = h[r, k].double()
    t = torch.randint(-1, n, (rows,), device="cuda", generator=g, dtype=torch.int32)
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    s.cross_entropy(h, W, t, loss, lse, s.cross_entropy_workspace(rows))
    dh, dW = torch.empty_like(h), torch.empty_like(W)
    s.cross_entropy_backward(h, W, t, lse, None, dh, dW, s.cross_entropy_backward_workspace(rows))
    z = a[:, None] * W[:, k].t().double()
    want = torch.logsumexp(z, 1)
    assert ((lse.double() - want).abs() <= 64 * U * (1 + z.abs().amax(1))).all()
    dz = torch.softmax(z, 1)
    there = (t >= 0).nonzero()[:, 0]
    dz[there, t[there].long()] -= 1
    dz[t < 0] = 0
    e = (128 * U * (1 + z.abs().amax(1, keepdim=True)) + 2.0 ** -11) * dz.abs() + 64 * U * (dz < 0) + 2.0 ** -39
    # dW by its columns: the rows that hold a number there
    cols = k.unique()[:2000]
    at = torch.searchsorted(cols, k).clamp(max=len(cols) - 1)
    mine = cols[at] == k
    wanted, bound = (torch.zeros(len(cols), n, dtype=torch.float64, device="cuda") for _ in range(2))
    wanted.index_add_(0, at[mine], a[mine, None] * dz[mine])
    bound.index_add_(0, at[mine], a[mine, None].abs() * (e[mine] + 4 * math.sqrt(rows) * U * dz[mine].abs()))
    got = dW[:, cols].t().double()
    assert ((got - wanted).abs() <= bound + 2.0 ** -8 * (wanted.abs() + bound)).all()
    rest = torch.ones(d, dtype=torch.bool, device="cuda")
    rest[k] = False
    assert not dW[:, rest].any()
    for lo in range(0, d, 1 << 15):
        w = W[:, lo:lo + (1 << 15)].double()
        wanted, bound = dz @ w, (e + 4 * math.sqrt(n) * U * dz.abs()) @ w.abs()
        got = dh[:, lo:lo + (1 << 15)].double()
        assert ((got - wanted).abs() <= bound + 2.0 ** -8 * (wanted.abs() + bound)).all(), lo


@pytest.mark.parametrize("lam,L,n", [(0.0, 256, 70), (3.0, 130, 40)])
def test_quantized_head_over_the_longest_rows(lam, L, n):
    """2^20 weights a row, 256 groups: whole numbers times powers of two, exact."""
    d, group = 1 << 20, 4096
    g = torch.Generator(device="cuda").manual_seed(5)
    s = B.Scd(B.make_config(B=2, L=L, N=L, V=n, d=d, cfg_lambda=lam))
    codes = torch.randint(0, 256, (n, d // 2), device="cuda", generator=g, dtype=torch.uint8)
    scales = torch.where(torch.rand(n, 256, device="cuda", generator=g) < 0.5, 0.5, 1.0).to(torch.bfloat16)
    zp = torch.randint(0, 16, (n, 256), device="cuda", generator=g, dtype=torch.uint8)
    h = torch.zeros(2, s.C, L, d, dtype=torch.bfloat16, device="cuda")
    h[..., :64] = _whole(g, 2, s.C, L, 64)
    h[..., -4100:-4000] = _whole(g, 2, s.C, L, 100)
    h[..., d // 2] = 2
    z = torch.empty(2, L, n, device="cuda")
    s.lm_head_quantized(h, s.pack_quantized(codes, scales, zp, group), z)
    q = torch.stack([codes & 15, codes >> 4], 2).reshape(n, 256, group).float()
    W = (scales.float()[:, :, None] * (q - zp.float()[:, :, None])).reshape(n, d)
    used = torch.cat([torch.arange(64), torch.arange(d - 4100, d - 4000), torch.tensor([d // 2])]).cuda()
    a = h[..., used].double() @ W[:, used].double().t()
    want = (1 + lam) * a[:, 0] - lam * a[:, -1]
    assert torch.equal(z.double(), want)
