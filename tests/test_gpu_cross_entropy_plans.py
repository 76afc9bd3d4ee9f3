"""Every instance of the cross entropy's products, and the gradient of vocabularies in several pieces, against 64 bits; the tolerances are
those derived in test_gpu_cross_entropy."""
import pytest
import torch

from cross_entropy_shapes import SHAPES, names
from test_gpu_cross_entropy import U, _ctx, _inputs, _near, _oracle, _run

pytestmark = pytest.mark.gpu


def _id(shape):
    return "{}-{}-{}-{}".format(*shape[:3], "f32" if shape[3] else "bf16")


@pytest.mark.parametrize("shape", SHAPES, ids=_id)
def test_loss_and_gradients_of_the_plan(shape):
    rows, n, d, f32 = shape[:4]
    dtype, V, v_lo, tau = torch.float32 if f32 else torch.bfloat16, n + 9, 5, 0.9
    s = _ctx(n, d, V, v_lo, tau)
    assert s.cross_entropy_kernel_names(rows, dtype) == names(shape)
    h, W, t, w = _inputs(rows, n, d, V, v_lo, seed=rows + n)
    if rows > 3:                                            # the first and the last of every piece are targets
        ends = torch.tensor([v for p in range(0, n, shape[5]) for v in (p, min(p + shape[5], n) - 1)], dtype=torch.int32, device="cuda")
        t[-min(len(ends), rows):] = ends[:rows]
    got = _run(s, h, W, t, w, dtype)
    want, bound = _oracle(h, W[v_lo:v_lo + n], t, w, tau, f32)
    for key in ("loss", "lse"):
        _near(got[key], want[key], bound[key], torch.float32, key)
    _near(got["dh"], want["dh"], bound["dh"], torch.bfloat16, "dh")
    _near(got["dW"][v_lo:v_lo + n], want["dW"], bound["dW"], dtype, "dW")
    assert (got["dh"][t < 0] == 0).all() and (got["loss"][t < 0] == 0).all()
    assert (got["dW"][:v_lo] == 7).all() and (got["dW"][v_lo + n:] == 7).all()
    del want, bound
    again = _run(s, h, W, t, w, dtype)
    for key in got:
        assert torch.equal(got[key], again[key]), key


@pytest.mark.parametrize("shape", [s for s in SHAPES if s[5] < s[1] and s[1] < 100000 and s[0] < 1000], ids=_id)
def test_pieces_accumulate_and_replay(shape):
    """Added to what is there, in a graph whose workspace holds something else at every replay."""
    rows, n, d, f32 = shape[:4]
    dtype = torch.float32 if f32 else torch.bfloat16
    h, W, t, w = _inputs(rows, n, d, n, 0, seed=3)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        s = _ctx(n, d)
    lse, loss = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ws, wb = s.cross_entropy_workspace(rows), s.cross_entropy_backward_workspace(rows, dtype)
    old = torch.randn(n, d, device="cuda").to(dtype)
    dW, dh = old.clone(), torch.empty_like(h)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        s.cross_entropy(h, W, t, loss, lse, ws)
        s.cross_entropy_backward(h, W, t, lse, w, dh, dW, wb, True)
    want, bound = _oracle(h, W, t, w, 1.0, f32)
    total = want["dW"] + old.double()
    for turn in range(3):
        dW.copy_(old)
        dh.fill_(7.0)
        wb.fill_(0xFF - turn)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _near(dW, total, bound["dW"] + U * total.abs(), dtype, "dW")
        _near(dh, want["dh"], bound["dh"], torch.bfloat16, "dh")
    assert len(range(0, n, shape[5])) > 1
