"""Every instance of the 8-bit LM head is launched by a shape of the tests."""
import ctypes
import os
import re

from fp8_shapes import CASES, MORE
from paper_2510_24211_amd import binding as B

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_24211_amd", "csrc", "lm_head_fp8.hip")


def _name(Bn, L, lam, V, v_lo, n, d, tau):
    lib, cfg, ctx = B.load(), B.make_config(B=Bn, L=L, N=L, V=V, d=d, v_lo=v_lo, v_hi=v_lo + n, cfg_lambda=lam, temperature=tau), ctypes.c_void_p()
    assert lib.scd_create(ctypes.byref(ctx), ctypes.byref(cfg), ctypes.c_void_p(1 << 20), 1 << 40, None) == B.SCD_OK
    buf = ctypes.create_string_buffer(128)
    assert lib.scd_lm_head_fp8_kernel_name(ctx, buf, 128) == B.SCD_OK
    lib.scd_destroy(ctx)
    return buf.value.decode()


def test_every_instance_has_a_shape():
    names = {_name(*c) for c in CASES + MORE}
    text = open(SOURCE).read()
    chosen = text[text.index("void choose_of("):text.index("void choose(const")]
    # the shapes that choose_of names, for one and for two rows per position
    shapes = {re.sub(r"\s", "", s) for s in re.findall(r"Fp8Cfg<([^<>]*)>", chosen)}
    want = set()
    for shape in shapes:
        parts = shape.split(",")
        parts += ["1"] * (7 - len(parts)) + (["false"] if len(parts) < 8 else [])
        for C in ("1", "2") if parts[0] == "C" else (parts[0],):
            rb = parts[1].split("/")
            rb = str(int(rb[0]) // int(C)) if len(rb) == 2 else rb[0]
            for borders in ("true", "false"):
                want.add("lm_head_fp8_kernel<Fp8Cfg<%s>, %s>" % (", ".join([C, rb] + parts[2:]), borders))
    assert names == want, (sorted(want - names), sorted(names - want))
