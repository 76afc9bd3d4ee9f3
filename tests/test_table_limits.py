"""Host-only checks of the limits that the operators on the vocabulary table set to sizes and settings."""
import ctypes

import pytest

from paper_2510_24211_amd import binding as B
from test_table_host import ALIGNED, Ctx


def _cross_entropy(c, rows):
    p, plenty = ALIGNED, 1 << 62
    return (c.lib.scd_cross_entropy(c.ptr, p, p, p, rows, p, p, None, plenty),
            c.lib.scd_cross_entropy_backward(c.ptr, p, p, p, rows, p, p, p, p, B.GRAD_F32, 0, None, plenty),
            c.lib.scd_cross_entropy_workspace_bytes(ctypes.byref(c.cfg), rows),
            c.lib.scd_cross_entropy_backward_workspace_bytes(ctypes.byref(c.cfg), rows, B.GRAD_BF16))


@pytest.mark.parametrize("tau,there", [(1.0, True), (5e-39, True), (3e38, True), (4e-39, False), (1e-45, False)])
def test_cross_entropy_needs_a_temperature_with_a_finite_inverse(tau, there):
    """Otherwise the largest logit's difference from itself, 0, times infinity is no number, and so is every loss.  (A call that is not refused for
    it gets as far as its workspace, which is missing.)"""
    loss, gradient, need, need_back = _cross_entropy(Ctx(B=1, L=1, temperature=tau), 5)
    assert loss == gradient == (B.SCD_EWORKSPACE if there else B.SCD_EUNSUPPORTED)
    assert (need > 0) == (need_back > 0) == there


@pytest.mark.parametrize("grad_type", [B.GRAD_BF16, B.GRAD_F32])
def test_workspaces_of_gradients_that_no_card_holds(grad_type):
    """2^20 rows of 2^21 columns are more tiles than a launch takes, whatever their shape; their sizes have an answer all the same."""
    c = Ctx(B=1, L=1, V=1 << 18, d=1 << 21)
    need = c.lib.scd_cross_entropy_backward_workspace_bytes(ctypes.byref(c.cfg), 1 << 20, grad_type)
    assert need > (1 << 20) * (1 << 21) * 2
    buf = ctypes.create_string_buffer(256)
    assert c.lib.scd_cross_entropy_kernel_names(c.ptr, 1 << 20, grad_type, buf, 256) == B.SCD_OK
    assert b"gemm_kernel<256, 256, kRows>" in buf.value
