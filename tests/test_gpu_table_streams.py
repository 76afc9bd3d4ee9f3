"""Memory that the binding allocates belongs to the stream that its kernels run on."""
import pytest
import torch

from paper_2510_24211_amd import binding as B

pytestmark = pytest.mark.gpu


def _stream_of(t):
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= t.data_ptr() < segment["address"] + segment["total_size"]:
            return segment["stream"]
    raise AssertionError("not the allocator's")


@pytest.mark.parametrize("size", [8, 40000])         # small blocks and large ones come from different pools
def test_what_a_context_allocates_is_its_streams(size):
    st = torch.cuda.Stream()
    s = B.Scd(B.make_config(B=1, L=2, N=2, V=size, d=64), stream=st)
    codes = torch.zeros(size, 32, dtype=torch.uint8, device="cuda")
    scales = torch.ones(size, 2, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    packed = s.pack_quantized(codes, scales, None, 32)
    torch.cuda.synchronize()
    for t in (s.workspace, s.alloc_state(), packed.data, s.embed_backward_workspace(size), s.cross_entropy_workspace(size),
              s.cross_entropy_backward_workspace(size)):
        assert _stream_of(t) == st.cuda_stream
