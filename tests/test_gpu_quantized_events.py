"""Events around the LM head of a step over 4-bit weights."""
import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw,group", [(dict(B=1, L=2, N=40, V=9000, d=136, top_k=50), 64),
                                      (dict(B=2, L=32, N=200, V=4000, d=512, top_k=50, cfg_lambda=3.0), 32)])
def test_events_take_the_kernels_time(kw, group):
    s = B.Scd(B.make_config(seed=1, **kw))
    c = s.cfg
    codes = torch.full((c.V, c.d // 2), 0x79, dtype=torch.uint8, device="cuda")
    W = s.pack_quantized(codes, torch.full((c.V, -(-c.d // group)), 0.01, dtype=torch.bfloat16, device="cuda"), None, group)
    h = torch.randn(c.B, s.C, c.L, c.d, device="cuda").to(torch.bfloat16)
    st = s.alloc_state()
    s.reset(st)
    before, start, stop, after = (torch.cuda.Event(enable_timing=True) for _ in range(4))
    big = torch.ones(4096, 4096, device="cuda")
    start.record()                                          # (makes the handles; a time that no step takes)
    for _ in range(20):
        big = big @ big * 0.0
    stop.record()
    s.step_quantized(h, W, st)
    s.set_lm_head_events(start.cuda_event, stop.cuda_event)
    for _ in range(3):
        torch.cuda.synchronize()
        before.record()
        s.step_quantized(h, W, st)
        after.record()
        torch.cuda.synchronize()
        head = start.elapsed_time(stop)
        assert 0 < head < before.elapsed_time(after)
    s.set_lm_head_events(None, None)
    s.step_quantized(h, W, st)
    torch.cuda.synchronize()
    assert start.elapsed_time(stop) == head
