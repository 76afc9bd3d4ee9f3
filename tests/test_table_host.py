"""Host-only checks of the operators on the vocabulary table: refusals before anything is launched, workspace sizes."""
import ctypes

import pytest

from paper_2510_24211_amd import binding as B

ALIGNED = 1 << 20          # device addresses are never touched by a refused call
INF = float("inf")


class Ctx:
    def __init__(self, **kw):
        self.lib = B.load()
        self.cfg = B.make_config(**dict(dict(B=2, L=4, N=8, V=100, d=64), **kw))
        self.need = B.workspace_bytes(self.cfg)
        self.ptr = ctypes.c_void_p()
        rc = self.lib.scd_create(ctypes.byref(self.ptr), ctypes.byref(self.cfg), ctypes.c_void_p(ALIGNED), self.need, None)
        assert rc == B.SCD_OK

    def __del__(self):
        self.lib.scd_destroy(self.ptr)


def _refused(call, good, bad, code=B.SCD_EINVAL):
    for at, value in bad:
        args = list(good)
        args[at] = value
        assert call(*args) == code, (at, value)


def test_embed_refuses():
    c, p = Ctx(), ALIGNED
    good = [c.ptr, p, 5, p, 1.0, p]
    _refused(c.lib.scd_embed, good, [(0, None), (1, None), (2, -1), (3, None), (5, None), (1, p + 2), (3, p + 8), (5, p + 2)])
    bare = Ctx(d=0)
    assert c.lib.scd_embed(bare.ptr, *good[1:]) == B.SCD_EINVAL
    good = [c.ptr, p, p, 1.0, p]
    _refused(c.lib.scd_embed_window, good, [(0, None), (1, None), (2, None), (4, None), (1, p + 16), (2, p + 8), (4, p + 2)])
    assert c.lib.scd_embed_window(bare.ptr, *good[1:]) == B.SCD_EINVAL


def test_embed_backward_refuses():
    c, p = Ctx(), ALIGNED
    need = c.lib.scd_embed_backward_workspace_bytes(ctypes.byref(c.cfg), 5)
    assert need > 0
    good = [c.ptr, p, 5, p, 1.0, p, 0, 0, p, need]
    _refused(c.lib.scd_embed_backward, good, [(0, None), (1, None), (2, -1), (3, None), (5, None), (1, p + 1), (3, p + 4), (5, p + 8),
                                              (6, 2), (6, -1), (7, 2), (7, -1)])
    _refused(c.lib.scd_embed_backward, good, [(8, None), (8, p + 16), (9, need - 1)], B.SCD_EWORKSPACE)
    for cfg, rows in ((c.cfg, -1), (B.make_config(B=1, L=1, N=1, V=10, d=0), 4), (B.make_config(B=0, L=1, N=1, V=10, d=8), 4)):
        assert c.lib.scd_embed_backward_workspace_bytes(ctypes.byref(cfg), rows) == 0


def test_cross_entropy_refuses():
    c, p = Ctx(), ALIGNED
    need = c.lib.scd_cross_entropy_workspace_bytes(ctypes.byref(c.cfg), 5)
    assert need > 0
    good = [c.ptr, p, p, p, 5, p, p, p, need]
    _refused(c.lib.scd_cross_entropy, good, [(0, None), (1, None), (2, None), (3, None), (4, -1), (4, (1 << 20) + 1), (5, None), (6, None),
                                             (1, p + 8), (2, p + 2), (3, p + 2), (5, p + 1), (6, p + 2)])
    _refused(c.lib.scd_cross_entropy, good, [(7, None), (7, p + 128), (8, need - 1)], B.SCD_EWORKSPACE)
    guided = Ctx(cfg_lambda=3.0)
    assert c.lib.scd_cross_entropy(guided.ptr, *good[1:]) == B.SCD_EUNSUPPORTED
    bare = Ctx(d=0)
    assert c.lib.scd_cross_entropy(bare.ptr, *good[1:]) == B.SCD_EINVAL


def test_cross_entropy_backward_refuses():
    c, p = Ctx(), ALIGNED
    size = c.lib.scd_cross_entropy_backward_workspace_bytes
    need = size(ctypes.byref(c.cfg), 5, B.GRAD_F32)
    assert need > 0
    good = [c.ptr, p, p, p, 5, p, p, p, p, B.GRAD_F32, 0, p, need]
    _refused(c.lib.scd_cross_entropy_backward, good,
             [(0, None), (1, None), (2, None), (3, None), (4, -1), (4, (1 << 20) + 1), (5, None), (1, p + 8), (2, p + 2), (3, p + 1),
              (5, p + 2), (6, p + 2), (7, p + 8), (8, p + 4), (9, 2), (9, -1), (10, 2)])
    _refused(c.lib.scd_cross_entropy_backward, good, [(11, None), (11, p + 64), (12, need - 1)], B.SCD_EWORKSPACE)
    guided = Ctx(cfg_lambda=1.0)
    assert c.lib.scd_cross_entropy_backward(guided.ptr, *good[1:]) == B.SCD_EUNSUPPORTED
    for rows, kind in ((-1, 0), (5, 2), ((1 << 20) + 1, 0)):
        assert size(ctypes.byref(c.cfg), rows, kind) == 0


@pytest.mark.parametrize("rows,V,d", [(1, 10, 8), (4096, 65536, 4096), (1 << 20, 128000, 1024)])
def test_backward_workspace_does_not_hold_the_logits(rows, V, d):
    cfg = B.make_config(B=1, L=1, N=1, V=V, d=d)
    for kind in (B.GRAD_BF16, B.GRAD_F32):
        need = B.load().scd_cross_entropy_backward_workspace_bytes(ctypes.byref(cfg), rows, kind)
        # a piece of 400 MiB or of 256 columns, the rows turned and their gradient's sums
        piece = max(400 << 20, 256 * 2 * (rows * 4 + d + 512))
        assert need <= piece * 1.1 + rows * d * 2 * 1.1 + 16 * 4 * rows * d + (1 << 20)


def test_quantize_refuses():
    c, p = Ctx(), ALIGNED
    good = [c.ptr, p, 32, p, p, p]
    _refused(c.lib.scd_quantize, good, [(0, None), (1, None), (2, 0), (2, -32), (2, 48), (3, None), (4, None), (1, p + 8), (3, p + 2),
                                        (4, p + 1)])
    good = [c.ptr, p, p, p, 32, p]
    _refused(c.lib.scd_pack_quantized, good, [(0, None), (1, None), (2, None), (4, 0), (4, 40), (5, None), (1, p + 1), (2, p + 1), (5, p + 128)])
    many = Ctx(d=32 * 257)                                  # 257 groups of 32, 129 of 64
    assert c.lib.scd_quantize(many.ptr, p, 32, p, p, None) == B.SCD_EINVAL
    bare = Ctx(d=0)
    assert c.lib.scd_quantize(bare.ptr, p, 32, p, p, None) == B.SCD_EINVAL


def test_quantized_bytes():
    size = B.load().scd_quantized_bytes
    bad = [(dict(d=64), 0, 0), (dict(d=64), 33, 0), (dict(d=64), 32, 2), (dict(d=64), 32, -1), (dict(d=0), 32, 0), (dict(d=32 * 257), 32, 0),
           (dict(d=12), 32, 0)]
    for kw, group, zeros in bad:
        cfg = B.make_config(**dict(dict(B=1, L=1, N=1, V=100), **kw))
        assert size(ctypes.byref(cfg), group, zeros) == 0, (kw, group, zeros)
    # 4 bits a weight, padded to 256 columns and 64 weights, two or four bytes a group
    cfg = B.make_config(B=1, L=1, N=1, V=5000, d=4096, v_lo=4, v_hi=4100)
    assert 4096 * 2048 <= size(ctypes.byref(cfg), 64, 0) - 4096 * 64 * 2 <= 4096 * 2048 + 2048
    assert 4096 * 2048 <= size(ctypes.byref(cfg), 64, 1) - 4096 * 64 * 4 <= 4096 * 2048 + 2048
    assert size(ctypes.byref(B.make_config(B=1, L=1, N=1, V=5000, d=32 * 257)), 64, 0) > 0


def test_lm_head_quantized_refuses():
    c, p = Ctx(), ALIGNED
    w = lambda at, group, zeros: ctypes.byref(B.ScdQuantized(at, group, zeros))  # noqa: E731
    for call, align in ((c.lib.scd_lm_head_quantized, 4), (c.lib.scd_step_quantized, 256)):
        good = [c.ptr, p, w(p, 32, 0), p]
        _refused(call, good, [(0, None), (1, None), (2, None), (3, None), (1, p + 8), (3, p + align // 2), (2, w(None, 32, 0)), (2, w(p + 16, 32, 0)),
                              (2, w(p, 0, 0)), (2, w(p, 16, 0)), (2, w(p, 32, 2))])
        bare = Ctx(d=0)
        assert call(bare.ptr, *good[1:]) == B.SCD_EINVAL


def test_every_entry_point_of_the_header_is_exported_and_bound():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "scd.h")).read(), flags=re.S)
    lib = B.load()
    for name in re.findall(r"\b(scd_\w+)\s*\(", text):
        assert getattr(lib, name).argtypes is not None or name == "scd_strerror", name
