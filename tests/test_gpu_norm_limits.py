"""The operators around the last norm at sizes whose offsets pass 32 bits, and with more rows than a launch has workgroups for."""
import math

import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, E4M3 = torch.bfloat16, torch.float8_e4m3fn


def _ctx(d, V=1, **kw):
    return B.Scd(B.make_config(B=1, L=1, N=1, V=V, d=d, **kw))


@pytest.mark.parametrize("rows,d", [((1 << 21) + 3, 1032), ((1 << 23) + 5, 8), (270000, 8200)])
def test_rows_beyond_4_gib_and_beyond_a_launch(rows, d):
    """Every row is one of 64 kinds: its results are those of a call on the kinds alone, the gains' gradient the kinds' times their number."""
    g = torch.Generator(device="cuda").manual_seed(d)
    kinds = torch.randn(64, d, device="cuda", generator=g).to(BF)
    gain = (1 + 0.3 * torch.randn(d, device="cuda", generator=g)).to(BF)
    s = _ctx(d)
    y0, inv0, dx0 = torch.empty_like(kinds), torch.empty(64, device="cuda"), torch.empty_like(kinds)
    s.norm(kinds, gain, y0, 1e-6, inv=inv0)
    s.norm_backward(kinds, gain, inv0, y0, dx0, None, s.norm_backward_workspace(64))
    kind = torch.arange(rows, device="cuda") % 64
    x = kinds[kind]
    y, inv = torch.empty_like(x), torch.empty(rows, device="cuda")
    s.norm(x, gain, y, 1e-6, inv=inv)
    assert torch.equal(inv, inv0[kind])
    for part in (slice(0, 1000), slice(rows // 2, rows // 2 + 1000), slice(rows - 1000, rows)):
        assert torch.equal(y[part], y0[kind[part]])
    dgain = torch.empty(d, device="cuda")
    s.norm_backward(x, gain, inv, y, x, dgain, s.norm_backward_workspace(rows), dsum=None)
    for part in (slice(0, 1000), slice(rows // 2, rows // 2 + 1000), slice(rows - 1000, rows)):
        assert torch.equal(x[part], dx0[kind[part]])
    terms = y0.double() * kinds.double() * inv0.double()[:, None] * torch.bincount(kind, minlength=64).double()[:, None]
    # (chains of rows / 512 additions at most, taken as independent roundings with a margin of 4, of sums that are all positive here or nearly)
    assert ((dgain.double() - terms.sum(0)).abs() <= 4 * U * math.sqrt(rows / 512 + 100) * terms.abs().sum(0)).all()


def test_a_gradient_beyond_4_gib():
    n = (1 << 31) + 12345
    big = torch.ones(n, device="cuda", dtype=BF)
    big[-3:] = 1000.0
    s = _ctx(0)
    grads = B.TensorList([big, torch.full((7,), 2.0, device="cuda")])
    norm = torch.empty(1, device="cuda")
    s.gradient_norm(grads, norm, s.gradient_norm_workspace(grads))
    want = math.sqrt(n - 3 + 3e6 + 28)
    assert abs(norm.item() - want) <= 2 * U * want
    s.clip_gradients(grads, grads, want / 4, norm)
    assert (big[:1000] == 0.25).all() and (big[n // 2:n // 2 + 1000] == 0.25).all() and (big[-1000:-3] == 0.25).all() and (big[-3:] == 250).all()


def test_a_table_beyond_4_gib():
    """The last ids of such a table, against 64 bits (4 u (sqrt(128) + sqrt(blocks) + 2) of the terms' sizes, as in the other tests)."""
    V, d, last = 1100000, 4096, 300
    g = torch.Generator(device="cuda").manual_seed(1)
    W = torch.randint(0, 120, (V, d), device="cuda", generator=g, dtype=torch.uint8)
    Ws = 0.01 * torch.exp(torch.randn(-(-V // 128), d // 128, device="cuda", generator=g))
    h = torch.randint(0, 120, (1, 1, 1, d), device="cuda", generator=g, dtype=torch.uint8)
    hs = 0.01 * torch.exp(torch.randn(1, 1, 1, d // 128, device="cuda", generator=g))
    s = _ctx(d, V=V)
    z = torch.empty(1, 1, V, device="cuda")
    s.lm_head_fp8(h, hs, W, Ws, z)
    v = torch.arange(V - last, V, device="cuda")
    w = W[-last:].view(E4M3).double() * Ws.double()[v // 128].repeat_interleave(128, 1)
    a = h.view(E4M3).double().view(-1) * hs.double().view(-1).repeat_interleave(128)
    want, size = w @ a, w.abs() @ a.abs()
    assert ((z[0, 0, -last:].double() - want).abs() <= 4 * U * (math.sqrt(128) + math.sqrt(d / 128) + 2) * size).all()
    codes, scales = torch.empty(V, d, device="cuda", dtype=torch.uint8), torch.empty_like(Ws)
    table = torch.ones(V, d, device="cuda", dtype=BF)
    s.quantize_fp8(table, codes, scales)
    assert (codes[-200:].view(E4M3).float() == 448).all() and ((scales - 1 / 448).abs() <= U / 448).all()


def test_step_events_and_streams():
    """Events of set_lm_head_events take the kernel's times, and what the binding allocates is its stream's."""
    st = torch.cuda.Stream()
    s = B.Scd(B.make_config(B=1, L=8, N=20, V=500, d=128), stream=st)
    state = s.alloc_state()
    s.reset(state)
    h, hs = torch.zeros(1, 1, 8, 128, device="cuda", dtype=torch.uint8), torch.ones(1, 1, 8, 1, device="cuda")
    W, Ws = torch.zeros(500, 128, device="cuda", dtype=torch.uint8), torch.ones(4, 1, device="cuda")
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    a.record(st)
    big = torch.ones(4096, 4096, device="cuda")
    with torch.cuda.stream(st):
        for _ in range(20):
            big = big @ big * 0.0
    b.record(st)
    torch.cuda.synchronize()
    before = a.elapsed_time(b)                             # (what no step takes)
    s.set_lm_head_events(a.cuda_event, b.cuda_event)
    s.step_fp8(h, hs, W, Ws, state)
    s.set_lm_head_events(None, None)
    torch.cuda.synchronize()
    assert 0 < a.elapsed_time(b) < before / 4
    ts = B.TensorList([torch.ones(10, device="cuda")])
    for t in (s.norm_backward_workspace(5000), s.gradient_norm_workspace(ts)):
        segments = torch.cuda.memory_snapshot()
        assert [x["stream"] for x in segments if x["address"] <= t.data_ptr() < x["address"] + x["total_size"]] == [st.cuda_stream]
