"""Which kernel the LM head over 4-bit weights launches for a shape (host-only)."""
import ctypes

import pytest

from paper_2510_24211_amd import binding as B
from quantized_shapes import SHAPES, config, name
from test_table_host import ALIGNED, Ctx


@pytest.mark.parametrize("shape", SHAPES, ids=name)
def test_the_shape_reaches_the_instance(shape):
    lib, cfg, ctx = B.load(), config(B.make_config, shape), ctypes.c_void_p()
    assert lib.scd_create(ctypes.byref(ctx), ctypes.byref(cfg), ctypes.c_void_p(ALIGNED), 1 << 40, None) == B.SCD_OK
    want, buf = name(shape), ctypes.create_string_buffer(128)
    call = lib.scd_lm_head_quantized_kernel_name
    assert call(ctx, shape[-1], int(shape[2]), buf, 128) == B.SCD_OK and buf.value.decode() == want
    assert call(ctx, shape[-1], int(shape[2]), buf, len(want) + 1) == B.SCD_OK
    assert call(ctx, shape[-1], int(shape[2]), buf, len(want)) == B.SCD_EINVAL
    assert lib.scd_destroy(ctx) == B.SCD_OK


def test_the_shapes_are_all_instances():
    """Four, two or one wavefronts that share k, with groups of whole and of half blocks; two tiles per wavefront and tiles of 256 rows with whole
    ones; two small workgroups per CU for up to 8 rows; each with and without zero points."""
    want = set()
    for c, rb, hrb in ((1, 1, 8), (2, 1, 8), (1, 1, 32), (1, 2, 32), (2, 1, 32)):
        some = [("1, 4, 4, 160, 1", 2), ("1, 8, 2, 160, 1", 2), ("1, 8, 1, 160, 1", 2), ("2, 8, 2, 160, 1", 4)] + \
            ([("1, 4, 4, 80, 1", 2)] if hrb == 8 else [])
        want |= {(f"{c}, {rb}, {hrb}, {rest}", step, zeros) for rest, first in some for step in range(first, 5, 2) for zeros in (False, True)}
    want |= {(f"{c}, {8 // c}, 32, 2, 8, 1, 160, 4", 4, zeros) for c in (1, 2) for zeros in (False, True)}
    assert {s[:3] for s in SHAPES} == want and len(SHAPES) == len(want)


def test_the_name_is_refused_for_bad_arguments():
    c, buf = Ctx(), ctypes.create_string_buffer(128)
    call = c.lib.scd_lm_head_quantized_kernel_name
    good = [c.ptr, 32, 0, buf, 128]
    assert call(*good) == B.SCD_OK
    for at, value in ((0, None), (1, 0), (1, 48), (1, -32), (2, 2), (2, -1), (3, None), (4, 0), (4, 20)):
        args = list(good)
        args[at] = value
        assert call(*args) == B.SCD_EINVAL, (at, value)
    bare = Ctx(d=0)
    assert call(bare.ptr, *good[1:]) == B.SCD_EINVAL
