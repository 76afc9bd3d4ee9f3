"""Host-only checks of the operators around the last norm: refusals before anything is launched, workspace sizes, the binding's own checks."""
import ctypes

import pytest
import torch

from paper_2510_24211_amd import binding as B
from test_table_binding import _gpu, _scd
from test_table_host import Ctx, _refused

ALIGNED = 1 << 20          # device addresses are never touched by a refused call
INF, NAN = float("inf"), float("nan")
BF, F32 = torch.bfloat16, torch.float32


def test_norm_refuses():
    c, p = Ctx(), ALIGNED
    good = [c.ptr, p, p, 1, p, 0, 1e-6, 5, p, p, p]
    alike = [(0, None), (1, None), (3, 2), (3, -1), (4, None), (5, 2), (6, 0.0), (6, -1.0), (6, INF), (6, NAN), (7, -1), (7, (1 << 25) + 1),
             (8, None), (1, p + 8), (2, p + 8), (4, p + 2), (8, p + 8)]
    _refused(c.lib.scd_norm, good, alike + [(2, None), (9, p + 4), (10, p + 2)])       # (2: a sum without a residual)
    good = [c.ptr, p, p, 1, p, 0, 1e-6, 5, p, p, p, p]
    _refused(c.lib.scd_norm_fp8, good, alike + [(2, None), (9, None), (9, p + 2), (10, p + 4), (11, p + 2)])
    for kw in (dict(d=0), dict(d=(1 << 24) + 8)):
        other = Ctx(**kw)
        assert c.lib.scd_norm_fp8(other.ptr, *good[1:]) == B.SCD_EINVAL


def test_norm_backward_refuses():
    c, p = Ctx(), ALIGNED
    need = c.lib.scd_norm_backward_workspace_bytes(ctypes.byref(c.cfg), 5)
    assert need > 0
    good = [c.ptr, p, 0, p, 0, p, p, p, 0, 5, p, p, 0, 0, p, need]
    _refused(c.lib.scd_norm_backward, good, [(0, None), (1, None), (2, 2), (3, None), (4, 2), (5, None), (6, None), (8, -1), (9, -1),
                                             (9, (1 << 25) + 1), (10, None), (12, 2), (13, 2), (13, -1), (1, p + 8), (3, p + 8), (5, p + 2),
                                             (6, p + 8), (7, p + 8), (10, p + 8), (11, p + 8)])
    _refused(c.lib.scd_norm_backward, good, [(14, None), (14, p + 16), (15, need - 1)], B.SCD_EWORKSPACE)
    for cfg, rows in ((c.cfg, -1), (c.cfg, (1 << 25) + 1), (B.make_config(B=1, L=1, N=1, V=10, d=0), 4), (B.make_config(B=0, L=1, N=1, V=10, d=8), 4)):
        assert c.lib.scd_norm_backward_workspace_bytes(ctypes.byref(cfg), rows) == 0


@pytest.mark.parametrize("d", [8, 4096, 8192, 8200, 1 << 24])
def test_norm_backward_workspace_has_room_for_what_workgroups_leave(d):
    lib = B.load()
    for rows in (0, 1, 700, 1 << 25):
        need = lib.scd_norm_backward_workspace_bytes(ctypes.byref(B.make_config(B=1, L=1, N=1, V=1, d=d)), rows)
        assert 256 <= need <= 768 * 8 * max(d, 8192) + 4 * rows + 1024
        assert rows == 0 or need >= 4 * d


def test_fp8_head_refuses():
    c, p = Ctx(d=64), ALIGNED
    name = ctypes.create_string_buffer(128)
    for call in (c.lib.scd_lm_head_fp8, c.lib.scd_step_fp8):
        _refused(call, [c.ptr, p, p, p, p, p], [(0, None), (1, None), (2, None), (3, None), (4, None), (5, None), (1, p + 8), (2, p + 2), (3, p + 8),
                                                (4, p + 1), (5, p + 2)])
        for kw in (dict(d=72), dict(d=(1 << 20) + 16), dict(L=1, V=(1 << 30) + 1, d=64)):
            other = Ctx(**kw)
            assert call(other.ptr, p, p, p, p, p) == B.SCD_EUNSUPPORTED
            assert c.lib.scd_lm_head_fp8_kernel_name(other.ptr, name, 128) == B.SCD_EUNSUPPORTED
        assert call(Ctx(d=0).ptr, p, p, p, p, p) == B.SCD_EINVAL
    _refused(c.lib.scd_quantize_fp8, [c.ptr, p, p, p], [(0, None), (1, None), (2, None), (3, None), (1, p + 8), (2, p + 8), (3, p + 2)])
    assert c.lib.scd_quantize_fp8(Ctx(d=72).ptr, p, p, p) == B.SCD_EUNSUPPORTED
    _refused(c.lib.scd_lm_head_fp8_kernel_name, [c.ptr, name, 128], [(0, None), (1, None), (2, 0), (2, 5)])


def _list(*tensors):
    return (B.ScdTensor * max(1, len(tensors)))(*[B.ScdTensor(*t) for t in tensors])


def test_gradient_norm_and_clipping_refuse():
    c, p = Ctx(d=0), ALIGNED
    ok = _list((p, 10, 0), (p + 2, 3, 0), (None, 0, 1), (p + 4, 1 << 40, 1))
    bad = [_list((p, -1, 0)), _list((p, (1 << 40) + 1, 0)), _list((None, 1, 0)), _list((p + 1, 1, 0)), _list((p + 2, 1, 1)), _list((p, 1, 2)), _list((p, 1, -1))]
    need = c.lib.scd_gradient_norm_workspace_bytes(ok, 4)
    assert need > 0 and c.lib.scd_gradient_norm_workspace_bytes(ok, 0) > 0
    good = [c.ptr, ok, 4, p, p, need]
    _refused(c.lib.scd_gradient_norm, good, [(0, None), (1, None), (2, -1), (3, None), (3, p + 2)])
    _refused(c.lib.scd_gradient_norm, good, [(4, None), (4, p + 16), (5, need - 1)], B.SCD_EWORKSPACE)
    for t in bad:
        assert c.lib.scd_gradient_norm_workspace_bytes(t, 1) == 0
        assert c.lib.scd_gradient_norm(c.ptr, t, 1, p, p, 1 << 20) == B.SCD_EINVAL
        assert c.lib.scd_clip_gradients(c.ptr, t, _list((p + 64, 1, 0)), 1, 1.0, p) == B.SCD_EINVAL
        assert c.lib.scd_clip_gradients(c.ptr, _list((p + 64, 1, 0)), t, 1, 1.0, p) == B.SCD_EINVAL
    one, same = _list((p, 10, 0)), _list((p, 10, 1))
    assert c.lib.scd_clip_gradients(c.ptr, one, same, 1, 1.0, p) == B.SCD_EINVAL            # in place, in another type
    good = [c.ptr, one, _list((p + 64, 10, 1)), 1, 1.0, p]
    _refused(c.lib.scd_clip_gradients, good, [(0, None), (1, None), (2, None), (2, _list((p + 64, 9, 1))), (3, -1), (4, -1.0), (4, NAN), (5, None), (5, p + 1)])


def test_binding_refuses():
    s, x, gain, one = _scd(d=64), _gpu(BF, 5, 64), _gpu(BF, 64), _gpu(F32, 5)
    codes, scales, ws = _gpu(torch.float8_e4m3fn, 5, 64), _gpu(F32, 5, 1), _gpu(torch.uint8, 1 << 30)
    calls = [lambda: s.norm(_gpu(BF, 5, 63), gain, x, 1e-6),                        # no whole rows
             lambda: s.norm(x, gain, _gpu(BF, 4, 64), 1e-6), lambda: s.norm(x, _gpu(BF, 63), x, 1e-6),
             lambda: s.norm(x, gain, x, 1e-6, residual=_gpu(BF, 4, 64)), lambda: s.norm(x, gain, x, 1e-6, inv=_gpu(F32, 4)),
             lambda: s.norm(_gpu(BF, 10, 64)[::2], gain, x, 1e-6),                  # strided
             lambda: s.norm_fp8(x, gain, codes, _gpu(F32, 4, 1), 1e-6), lambda: s.norm_fp8(x, gain, _gpu(torch.uint8, 4, 64), scales, 1e-6),
             lambda: s.norm(_gpu(BF, 1 << 31, 64), gain, x, 1e-6), lambda: s.norm_backward_workspace(1 << 32),
             lambda: s.norm_backward(x, gain, one, _gpu(BF, 4, 64), x, None, ws), lambda: s.norm_backward(x, gain, _gpu(F32, 4), x, x, None, ws),
             lambda: s.norm_backward(x, gain, one, x, x, _gpu(F32, 63), ws),
             lambda: s.lm_head_fp8(_gpu(torch.uint8, 63), _gpu(F32, 1), _gpu(torch.uint8, 100, 64), _gpu(F32, 1), _gpu(F32, 100)),
             lambda: s.lm_head_fp8(_gpu(torch.uint8, 64), _gpu(F32, 1), _gpu(torch.uint8, 99, 64), _gpu(F32, 1), _gpu(F32, 100)),
             lambda: s.lm_head_fp8(_gpu(torch.uint8, 64), _gpu(F32, 1), _gpu(torch.uint8, 100, 64), _gpu(F32, 0), _gpu(F32, 100)),
             lambda: s.clip_gradients(B.TensorList([x]), B.TensorList([]), 1.0, one)]
    for call in calls:
        with pytest.raises(ValueError):
            call()
    calls = [lambda: s.norm(x.to(F32), gain, x, 1e-6), lambda: s.norm(x, gain.to(torch.float16), x, 1e-6),
             lambda: s.norm(x, gain, x, 1e-6, residual=x, sum=_gpu(F32, 5, 64)),
             lambda: s.norm_backward(x, gain, one, x, x, None, ws, dsum=_gpu(F32, 5, 64)), lambda: s.norm_backward(x, gain, one, x, _gpu(torch.float16, 5, 64), None, ws),
             lambda: s.quantize_fp8(_gpu(BF, 100, 64), _gpu(torch.int8, 100, 64), scales), lambda: B.TensorList([None]), lambda: B.TensorList([torch.ones(3)]),
             lambda: B.TensorList([_gpu(torch.float16, 3)])]
    for call in calls:
        with pytest.raises(TypeError):
            call()
    with pytest.raises(B.ScdError):
        s.norm(x, None, x, 1e-6)
