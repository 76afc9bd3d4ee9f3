"""Cross entropy of hidden rows and its gradient against 64 bits.

Tolerances, u = 2^-24.  A logit is a sum of d products in fp32: at most d roundings of u of the products' magnitudes; the
errors of one chain are independent, so sqrt(d) of them with a margin of 4 is taken (and the operand sums of 16 that the
matrix unit makes at once count as one).  With E the largest error of a row's logits, lse errs by at most E and by its own
arithmetic: exponentials and logarithms of 2 to 1 ulp of arguments up to |z| log2(e), a sum of n positive terms added up in a
tree: 16 u (1 + |z|max).  loss = lse - z_t errs by twice that.
dz errs by the relative error of p, e_p = 2 E + 16 u (1 + |z|max), and by its rounding to fp16, 2^-11 (2^-22 in two terms) of
itself and 2^-25 units in the place of 2^-14 (2^-39) of the largest weight; h and W may err by 2^-39 of their largest element,
to which that of dz, at most 1, adds nothing that its own 2^-39 does not cover; the products add the same kind of chain; the result is rounded to its type.  The roundings of dz's terms are taken at their
full size and of one sign: sum |dz| |W|.
Underflow: fp32 and bf16 hold nothing between 0 and 2^-126 but denormal numbers, which the units may take for 0.  p is off by up
to 2^-126 more for that, and so is each of dz's terms (a rest that its first term leaves may be that small where dz itself is
not): 3 * 2^-126 (coefficients of up to 2 among them) per term of the products, 3 * 2^-126 * sum |h|, and 2^-126 of the result."""
import math

import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _ctx(n, d, V=None, v_lo=0, tau=1.0, **kw):
    V = n + v_lo if V is None else V
    return B.Scd(B.make_config(B=1, L=1, N=1, V=V, d=d, v_lo=v_lo, v_hi=v_lo + n, temperature=tau, **kw))


def _inputs(rows, n, d, V, v_lo, seed, sharp=4.0, out=0.1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    W = (torch.randn(V, d, device="cuda", generator=g) / math.sqrt(d)).to(torch.bfloat16)
    t = torch.randint(0, n, (rows,), device="cuda", generator=g)
    h = torch.randn(rows, d, device="cuda", generator=g) + sharp * W[v_lo + t].float()
    t = torch.where(torch.rand(rows, device="cuda", generator=g) < out, -1, t).to(torch.int32)
    w = torch.rand(rows, device="cuda", generator=g) - 0.3
    return h.to(torch.bfloat16), W, t, w


def _oracle(h, W, t, w, tau, two_terms=False):
    """64 bits: values and bounds."""
    h, W = h.double(), W.double()
    d, n = h.shape[1], W.shape[0]
    chain = 4 * math.sqrt(d) * U
    z = h @ W.t() / tau
    E = (h.abs() @ W.abs().t() / tau * chain + 2 * U * z.abs()).amax(1)
    zmax = z.abs().amax(1)
    e_lse = E + 16 * U * (1 + zmax)
    lse = torch.logsumexp(z, 1)
    there, inside = t >= 0, (t >= 0) & (t < n)
    ti = t.clamp(0, n - 1).long()
    zt = torch.gather(z, 1, ti[:, None])[:, 0]
    loss = torch.where(there, torch.where(inside, lse - zt, math.inf), 0.0)
    p = torch.exp(z - lse[:, None])
    hot = torch.zeros_like(p)
    hot[inside.nonzero()[:, 0], t[inside].long()] = 1.0
    coef = torch.where(there, w.double() / tau, 0.0)[:, None]
    dz = coef * (p - hot)
    e_dz = coef.abs() * p * (2 * E + 32 * U * (1 + zmax))[:, None]
    bf, tab = 2.0 ** -11, (2.0 ** -22 if two_terms else 2.0 ** -11)
    w_max = w[there].abs().max().double() if there.any() else 1.0
    floor = 2.0 ** -38 * w_max / tau
    r = dict(loss=loss, lse=lse, dh=dz @ W, dW=dz.t() @ h)
    tiny = 3 * 2.0 ** -126
    chain_n, chain_m = 4 * math.sqrt(n) * U, 4 * math.sqrt(max(h.shape[0], 1)) * U
    b = dict(loss=2 * e_lse + 4 * U * (lse.abs() + zt.abs()), lse=e_lse + 4 * U * lse.abs(),
             dh=(e_dz + dz.abs() * (bf + chain_n + 4 * U) + tiny + coef.abs() * 2.0 ** -38) @ W.abs() + tiny,
             dW=(e_dz + dz.abs() * (tab + chain_m + 4 * U) + tiny + floor).t() @ h.abs() + tiny)
    return r, b


def _run(s, h, W, t, w, dtype, accumulate=False, dW=None, want_dh=True):
    rows, d = h.shape
    loss, lse = (torch.full((rows + 2,), 7.0, device="cuda") for _ in range(2))
    dh = torch.full((rows + 2, d), 7.0, dtype=torch.bfloat16, device="cuda")
    dW = torch.full((s.cfg.V, d), 7.0, dtype=dtype, device="cuda") if dW is None else dW
    s.cross_entropy(h, W, t, loss[1:rows + 1], lse[1:rows + 1], s.cross_entropy_workspace(rows).fill_(0xFF))
    s.cross_entropy_backward(h, W, t, lse[1:rows + 1], w, dh[1:rows + 1] if want_dh else None, dW,
                             s.cross_entropy_backward_workspace(rows, dtype).fill_(0xFF), accumulate)
    for x in (loss, lse, dh):
        assert (x[0] == 7).all() and (x[-1] == 7).all()
    return dict(loss=loss[1:rows + 1], lse=lse[1:rows + 1], dh=dh[1:rows + 1], dW=dW)


def _near(got, want, bound, dtype, what):
    half = 2.0 ** -8 if dtype == torch.bfloat16 else U
    err, allowed = (got.double() - want).abs(), bound + half * (want.abs() + bound)
    assert (err <= allowed).all(), (what, (err - allowed).max().item(), (err / allowed).max().item())


SHAPES = [  # rows, n, d, V, v_lo, tau
    (1, 1, 8, 1, 0, 1.0), (1, 2, 16, 5, 2, 0.5), (3, 100, 64, 130, 7, 1.0), (33, 257, 72, 257, 0, 0.8), (128, 128, 128, 128, 0, 1.0),
    (129, 1000, 200, 1031, 5, 1.0), (257, 513, 136, 600, 40, 2.0), (64, 4099, 320, 4200, 3, 1.0), (300, 20000, 64, 20003, 1, 1.0),
    (700, 3001, 1288, 3001, 0, 0.9), (2, 40000, 128, 40000, 0, 1.0), (1100, 129, 520, 300, 100, 1.0), (520, 8192, 192, 8200, 4, 1.0)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,n,d,V,v_lo,tau", SHAPES)
def test_loss_and_gradients(rows, n, d, V, v_lo, tau, dtype):
    h, W, t, w = _inputs(rows, n, d, V, v_lo, seed=rows + n)
    got = _run(_ctx(n, d, V, v_lo, tau), h, W, t, w, dtype)
    want, bound = _oracle(h, W[v_lo:v_lo + n], t, w, tau, dtype == torch.float32)
    for key in ("loss", "lse"):
        _near(got[key], want[key], bound[key], torch.float32, key)
    _near(got["dh"], want["dh"], bound["dh"], torch.bfloat16, "dh")
    _near(got["dW"][v_lo:v_lo + n], want["dW"], bound["dW"], dtype, "dW")
    assert (got["dh"][t < 0] == 0).all() and (got["loss"][t < 0] == 0).all()
    assert (got["dW"][:v_lo] == 7).all() and (got["dW"][v_lo + n:] == 7).all()      # rows of other ids are left alone


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_accumulate_adds_in_32_bits(dtype):
    rows, n, d, V, v_lo = 150, 700, 136, 720, 11
    h, W, t, w = _inputs(rows, n, d, V, v_lo, seed=5)
    old = torch.randn(V, d, device="cuda").to(dtype)
    got = _run(_ctx(n, d, V, v_lo), h, W, t, w, dtype, True, old.clone())["dW"]
    want, bound = _oracle(h, W[v_lo:v_lo + n], t, w, 1.0, dtype == torch.float32)
    total = want["dW"] + old[v_lo:v_lo + n].double()
    _near(got[v_lo:v_lo + n], total, bound["dW"] + U * total.abs(), dtype, "dW")
    assert torch.equal(got[:v_lo], old[:v_lo]) and torch.equal(got[v_lo + n:], old[v_lo + n:])


def test_one_gradient_alone_and_unit_weights():
    rows, n, d = 90, 600, 64
    h, W, t, _ = _inputs(rows, n, d, n, 0, seed=8)
    s = _ctx(n, d)
    both = _run(s, h, W, t, torch.ones(rows, device="cuda"), torch.bfloat16)
    ws = s.cross_entropy_backward_workspace(rows)
    dh, dW = torch.empty_like(both["dh"]), torch.empty_like(both["dW"])
    s.cross_entropy_backward(h, W, t, both["lse"], None, dh, None, ws)
    s.cross_entropy_backward(h, W, t, both["lse"], None, None, dW, ws)
    assert torch.equal(dh, both["dh"]) and torch.equal(dW, both["dW"])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_rows_and_rows_left_out(dtype):
    """No rows: a gradient of zeros, or nothing added.  All rows left out, whatever they hold: the same."""
    n, d, V, v_lo = 300, 72, 310, 4
    W = torch.randn(V, d, device="cuda").to(torch.bfloat16)
    s = _ctx(n, d, V, v_lo)
    for rows in (0, 70):
        h = torch.full((rows, d), math.nan, device="cuda", dtype=torch.bfloat16)
        t = torch.full((rows,), -100, device="cuda", dtype=torch.int32)
        got = _run(s, h, W, t, torch.full((rows,), math.inf, device="cuda"), dtype)
        assert (got["loss"] == 0).all() and (got["dh"] == 0).all()
        assert (got["dW"][v_lo:v_lo + n] == 0).all() and (got["dW"][:v_lo] == 7).all() and (got["dW"][v_lo + n:] == 7).all()
        kept = torch.randn(V, d, device="cuda").to(dtype)
        assert torch.equal(_run(s, h, W, t, None, dtype, True, kept.clone())["dW"], kept)


def test_rows_left_out_do_not_reach_the_others():
    rows, n, d = 200, 900, 72
    h, W, t, w = _inputs(rows, n, d, n, 0, seed=21)
    s = _ctx(n, d)
    clean = _run(s, torch.where((t < 0)[:, None], 0.0, h.float()).to(torch.bfloat16), W, t, w, torch.float32)
    h[t < 0] = math.nan
    h[(t < 0).nonzero()[0, 0]] = math.inf
    w[t < 0] = math.nan
    got = _run(s, h, W, t, w, torch.float32)
    for key in ("loss", "dh", "dW"):
        assert torch.equal(got[key], clean[key]), key


def test_targets_outside_the_allowed_ids():
    rows, n, d = 40, 130, 64
    h, W, t, w = _inputs(rows, n, d, n, 0, seed=2, out=0.0)
    t[3], t[17], t[39] = n, n + 1000000, 2 ** 31 - 1
    got = _run(_ctx(n, d), h, W, t, w, torch.float32)
    want, bound = _oracle(h, W, t, w, 1.0, True)
    bad = t >= n
    assert torch.isposinf(got["loss"][bad]).all() and got["loss"][~bad].isfinite().all()
    _near(got["dh"], want["dh"], bound["dh"], torch.bfloat16, "dh")
    _near(got["dW"], want["dW"], bound["dW"], torch.float32, "dW")


def test_peaked_and_flat_rows():
    """Logits of several hundred, a row of equal ones, and a row of zeros."""
    rows, n, d = 64, 1000, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    W = torch.randn(n, d, device="cuda", generator=g).to(torch.bfloat16)
    h = (torch.randn(rows, d, device="cuda", generator=g) * 30).to(torch.bfloat16)
    h[0] = 0
    t = torch.randint(0, n, (rows,), device="cuda", generator=g, dtype=torch.int32)
    w = torch.ones(rows, device="cuda")
    got = _run(_ctx(n, d), h, W, t, w, torch.float32)
    want, bound = _oracle(h, W, t, w, 1.0, True)
    for key, kind in (("loss", torch.float32), ("lse", torch.float32), ("dh", torch.bfloat16), ("dW", torch.float32)):
        _near(got[key], want[key], bound[key], kind, key)
    assert abs(got["loss"][0].item() - math.log(n)) < 1e-5


def test_small_losses_keep_their_digits():
    """Rows that are all but sure of their target: the loss is log(1 + r), r = sum of exp(z - z_t), and errs by r times the
    errors of logits' differences (2 E each) and a few roundings of 1 + r, not by roundings of the logits' size (300 here)."""
    rows, n, d = 40, 500, 64
    g = torch.Generator(device="cuda").manual_seed(9)
    W = torch.randn(n, d, device="cuda", generator=g).to(torch.bfloat16)
    t = torch.randint(0, n, (rows,), device="cuda", generator=g, dtype=torch.int32)
    h = (W[t.long()].float() * torch.linspace(0.2, 6.0, rows, device="cuda")[:, None]).to(torch.bfloat16)
    got = _run(_ctx(n, d), h, W, t, None, torch.bfloat16)["loss"].double()
    z = h.double() @ W.double().t()
    E = (h.double().abs() @ W.double().abs().t() * (4 * math.sqrt(d) * U) + 2 * U * z.abs()).amax(1)
    zt = torch.gather(z, 1, t.long()[:, None])
    r = torch.exp(z - zt).sum(1) - 1
    want = torch.log1p(r)
    # the sum holds 1 and r in 32 bits, tree by tree: 16 roundings of it; its logarithm one more
    bound = 2 * E * r / (1 + r) + 16 * U * (1 + z.abs().amax(1) * r / (1 + r)) + 2 * U * want
    assert ((got - want).abs() <= bound).all(), ((got - want).abs() / bound).max().item()
    assert (want < 1e-4).sum() > 5 and (got >= 0).all()


def test_rows_that_are_not_finite_stay_by_themselves():
    rows, n, d = 50, 300, 64
    h, W, t, w = _inputs(rows, n, d, n, 0, seed=6, out=0.0)
    s = _ctx(n, d)
    clean = _run(s, h, W, t, w, torch.bfloat16)
    h[7, 3], h[30, 0] = math.nan, math.inf
    got = _run(s, h, W, t, w, torch.bfloat16)
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[7] = bad[30] = True
    assert got["loss"][bad].isnan().all() and got["dh"][bad].isnan().any(1).all()
    for key in ("loss", "lse", "dh"):
        assert torch.equal(got[key][~bad], clean[key][~bad]), key


def test_gradient_by_differences():
    """d(sum w loss) along random directions of h and W, by central differences in 64 bits of the forward pass's definition,
    against the kernel's gradients (which hold about 2^-8 of the terms' size)."""
    rows, n, d = 12, 50, 16
    h, W, t, w = _inputs(rows, n, d, n, 0, seed=12)
    got = _run(_ctx(n, d, tau=0.7), h, W, t, w, torch.float32)
    _, bound = _oracle(h, W, t, w, 0.7, True)

    def total(h64, W64):
        z = h64 @ W64.t() / 0.7
        there = t >= 0
        zt = torch.gather(z, 1, t.clamp(min=0).long()[:, None])[:, 0]
        return (torch.where(there, torch.logsumexp(z, 1) - zt, 0.0) * w.double()).sum()

    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for key, at in (("dh", 0), ("dW", 1)):
            args = [h.double(), W.double()]
            u = torch.randn(args[at].shape, device="cuda", generator=g, dtype=torch.float64)
            eps, side = 1e-5, []
            for sign in (1, -1):
                moved = list(args)
                moved[at] = args[at] + sign * eps * u
                side.append(total(*moved))
            slope = (side[0] - side[1]) / (2 * eps)
            value = got[key].double()
            half = 2.0 ** -8 if key == "dh" else U
            allowed = ((bound[key] + half * value.abs()) * u.abs()).sum() + 1e-7
            assert ((value * u).sum() - slope).abs() <= allowed, key


def test_same_bits_again_on_another_stream_and_in_a_graph():
    rows, n, d = 260, 5000, 264
    h, W, t, w = _inputs(rows, n, d, n, 0, seed=31)
    first = _run(_ctx(n, d), h, W, t, w, torch.bfloat16)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        s = _ctx(n, d)
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dh, dW = torch.empty_like(h), torch.empty_like(W)
    ws, wb = s.cross_entropy_workspace(rows), s.cross_entropy_backward_workspace(rows)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        s.cross_entropy(h, W, t, loss, lse, ws)
        s.cross_entropy_backward(h, W, t, lse, w, dh, dW, wb)
    for turn in range(4):
        if turn == 2:
            t.copy_(t.flip(0))
            first = _run(_ctx(n, d), h, W, t, w, torch.bfloat16)
        for x in (loss, lse, dh, dW):
            x.fill_(math.nan)
        ws.fill_(turn)
        wb.fill_(turn)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for key, x in (("loss", loss), ("lse", lse), ("dh", dh), ("dW", dW)):
            assert torch.equal(x, first[key]), (turn, key)


def test_tied_table_learns_from_both_ends():
    """One table: embedded, scored, and its gradient gathered from both uses."""
    V, d, rows, scale = 700, 64, 130, 8.0
    g = torch.Generator(device="cuda").manual_seed(17)
    W = (torch.randn(V, d, device="cuda", generator=g) / 8).to(torch.bfloat16)
    ids = torch.randint(0, V, (rows,), device="cuda", generator=g, dtype=torch.int32)
    t = torch.roll(ids, -1)
    t[-1] = -1
    s = _ctx(V, d)
    x = torch.empty(rows, d, device="cuda", dtype=torch.bfloat16)
    s.embed(ids, W, scale, x)
    w = torch.full((rows,), 1.0 / rows, device="cuda")
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dx, dW = torch.empty_like(x), torch.empty(V, d, device="cuda")
    s.cross_entropy(x, W, t, loss, lse, s.cross_entropy_workspace(rows))
    wb = s.cross_entropy_backward_workspace(rows, torch.float32)
    eb = s.embed_backward_workspace(rows)
    s.cross_entropy_backward(x, W, t, lse, w, dx, dW, wb)
    s.embed_backward(ids, dx, scale, dW, eb, accumulate=True)
    other = torch.empty_like(dW)                            # the other way round
    s.embed_backward(ids, dx, scale, other, eb)
    s.cross_entropy_backward(x, W, t, lse, w, None, other, wb, accumulate=True)
    want, bound = _oracle(x, W, t, w, 1.0, True)
    total = want["dW"].clone()
    total.index_add_(0, ids.long(), dx.double() * scale)
    most = bound["dW"].clone()
    most.index_add_(0, ids.long(), dx.double().abs() * scale * 40 * U)
    for got in (dW, other):
        _near(got, total, most + 2 * U * (total.abs() + want["dW"].abs()), torch.float32, "dW")
    _near(dx, want["dh"], bound["dh"], torch.bfloat16, "dx")


def test_wide_rows_of_many_ids():
    """Offsets past 4 GiB: a table of 70000 rows of 32768 bf16 values, the gradient of its last ids."""
    V, d, rows = 70000, 32768, 40
    v_lo = V - 300
    g = torch.Generator(device="cuda").manual_seed(3)
    W = torch.zeros(V, d, device="cuda", dtype=torch.bfloat16)
    W[v_lo:] = (torch.randn(300, d, device="cuda", generator=g) / 180).to(torch.bfloat16)
    h = torch.randn(rows, d, device="cuda", generator=g).to(torch.bfloat16)
    t = torch.randint(0, 300, (rows,), device="cuda", generator=g, dtype=torch.int32)
    w = torch.ones(rows, device="cuda")
    got = _run(_ctx(300, d, V, v_lo), h, W, t, w, torch.bfloat16, False, torch.zeros_like(W))
    want, bound = _oracle(h, W[v_lo:], t, w, 1.0)
    _near(got["lse"], want["lse"], bound["lse"], torch.float32, "lse")
    _near(got["dh"], want["dh"], bound["dh"], torch.bfloat16, "dh")
    _near(got["dW"][v_lo:], want["dW"], bound["dW"], torch.bfloat16, "dW")
    assert not got["dW"][:v_lo].any()
