"""Host-only checks of the binding's methods on the vocabulary table: what it refuses before the library is called."""
import ctypes

import pytest
import torch

from paper_2510_24211_amd import binding as B

WORKSPACE = 1 << 20          # never touched: every call here is refused


class OnGpu(torch.Tensor):
    """A tensor without memory that says it is a GPU's."""
    is_cuda = True

    def data_ptr(self):
        return 256


def _gpu(dtype, *shape):
    return torch.empty(*shape, dtype=dtype, device="meta").as_subclass(OnGpu)


def _scd(**kw):
    s = object.__new__(B.Scd)
    s.lib, s.cfg = B.load(), B.make_config(**dict(dict(B=1, L=1, N=1, V=100, d=64), **kw))
    s.n, s.C, s.device, s.ctx = s.cfg.v_hi - s.cfg.v_lo, 2 if s.cfg.cfg_lambda else 1, torch.device("cuda:0"), ctypes.c_void_p()
    need = B.workspace_bytes(s.cfg)
    assert s.lib.scd_create(ctypes.byref(s.ctx), ctypes.byref(s.cfg), ctypes.c_void_p(WORKSPACE), need, None) == B.SCD_OK
    return s


@pytest.mark.parametrize("group", [(1 << 32) + 32, -(1 << 32) + 32, 1 << 31])
def test_groups_that_32_bits_do_not_hold_are_refused(group):
    """Cut off to 32 bits such a group is another, valid one, with more scales than the arrays were checked for."""
    s, u8, bf = _scd(), torch.uint8, torch.bfloat16
    codes, scales = _gpu(u8, 100, 32), _gpu(bf, 100, 1)
    with pytest.raises(ValueError):
        s.quantize(_gpu(bf, 100, 64), group, codes, scales)
    with pytest.raises(ValueError):
        s.pack_quantized(codes, scales, None, group)
    W = B.QuantizedWeights(_gpu(u8, 1 << 20), group, False)
    with pytest.raises(ValueError):
        s.lm_head_quantized(_gpu(bf, 64), W, _gpu(torch.float32, 100))
    with pytest.raises(ValueError):
        s.step_quantized(_gpu(bf, 64), W, _gpu(u8, B.state_bytes(s.cfg)))


@pytest.mark.parametrize("rows", [(1 << 32) + 5, 1 << 31])
def test_rows_that_32_bits_do_not_hold_are_refused(rows):
    """Cut off to 32 bits such a number of rows is another, and the rest of them would be left out in silence."""
    s, bf, f32 = _scd(d=8), torch.bfloat16, torch.float32
    ids, wide, one, W = _gpu(torch.int32, rows), _gpu(bf, rows, 8), _gpu(f32, rows), _gpu(bf, 100, 8)
    ws = _gpu(torch.uint8, 1 << 40)
    calls = [lambda: s.embed(ids, W, 1.0, wide), lambda: s.embed_backward_workspace(rows),
             lambda: s.embed_backward(ids, wide, 1.0, W, ws), lambda: s.cross_entropy_workspace(rows),
             lambda: s.cross_entropy(wide, W, ids, one, one, ws), lambda: s.cross_entropy_backward_workspace(rows),
             lambda: s.cross_entropy_backward(wide, W, ids, one, None, wide, W, ws)]
    for call in calls:
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("other", [dict(V=100, v_lo=10, v_hi=42, d=64), dict(V=100, v_lo=0, v_hi=32, d=40)])
def test_weights_laid_out_for_other_ids_are_refused(other):
    """Rows 10 .. 41 of a table take the bytes of rows 0 .. 31, and so do rows of 40 weights those of 64."""
    s = _scd(V=100, v_lo=0, v_hi=32)
    c = B.make_config(B=1, L=1, N=1, **other)
    need = s.lib.scd_quantized_bytes(ctypes.byref(c), 64, 0)
    assert need == s.lib.scd_quantized_bytes(ctypes.byref(s.cfg), 64, 0)
    h, z, st = _gpu(torch.bfloat16, 64), _gpu(torch.float32, 32), _gpu(torch.uint8, B.state_bytes(s.cfg))
    W = B.QuantizedWeights(_gpu(torch.uint8, need), 64, False, c)
    for call in (lambda: s.lm_head_quantized(h, W, z), lambda: s.step_quantized(h, W, st)):
        with pytest.raises(ValueError, match="laid out for"):
            call()
