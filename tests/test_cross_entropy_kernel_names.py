"""Which products the cross entropy and its gradient launch for a shape (host-only)."""
import ctypes

import pytest

from cross_entropy_shapes import SHAPES, names
from paper_2510_24211_amd import binding as B
from test_table_host import ALIGNED, Ctx

TILES = {(128, 64), (128, 128), (256, 128), (256, 192), (256, 256)}


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:4])))
def test_the_shape_reaches_the_plan(shape):
    rows, n, d, f32 = shape[:4]
    lib, cfg, ctx = B.load(), B.make_config(B=1, L=1, N=1, V=n + 9, v_lo=5, v_hi=n + 5, d=d), ctypes.c_void_p()
    assert lib.scd_create(ctypes.byref(ctx), ctypes.byref(cfg), ctypes.c_void_p(ALIGNED), 1 << 40, None) == B.SCD_OK
    want, buf, call = names(shape), ctypes.create_string_buffer(256), lib.scd_cross_entropy_kernel_names
    assert call(ctx, rows, int(f32), buf, 256) == B.SCD_OK and buf.value.decode() == want
    assert call(ctx, rows, int(f32), buf, len(want) + 1) == B.SCD_OK
    assert call(ctx, rows, int(f32), buf, len(want)) == B.SCD_EINVAL
    assert lib.scd_destroy(ctx) == B.SCD_OK


def test_the_shapes_are_all_instances_and_plans():
    for at in (4, 6, 7):
        assert {s[at] for s in SHAPES} == TILES, at
    for f32 in (False, True):
        assert {s[9] for s in SHAPES if s[3] == f32} == TILES, f32
        # one piece or several, k of dh's product whole or dealt out
        assert {(s[5] < s[1], s[8] > 1) for s in SHAPES if s[3] == f32} == {(a, b) for a in (False, True) for b in (False, True)}, f32


def test_the_names_are_refused_for_bad_arguments():
    c, buf = Ctx(), ctypes.create_string_buffer(256)
    call = c.lib.scd_cross_entropy_kernel_names
    good = [c.ptr, 5, 0, buf, 256]
    assert call(*good) == B.SCD_OK
    for at, value in ((0, None), (1, -1), (1, (1 << 20) + 1), (2, 2), (2, -1), (3, None), (4, 0), (4, 50)):
        args = list(good)
        args[at] = value
        assert call(*args) == B.SCD_EINVAL, (at, value)
    bare, guided = Ctx(d=0), Ctx(cfg_lambda=3.0)
    assert call(bare.ptr, *good[1:]) == B.SCD_EINVAL and call(guided.ptr, *good[1:]) == B.SCD_EUNSUPPORTED
