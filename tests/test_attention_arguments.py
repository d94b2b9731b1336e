"""Attention's checks of its arguments, on the host (no call reaches the GPU: where nothing else is wrong, the backward pass has no lse)."""
import ctypes

import pytest

pytest.importorskip("torch")
import paper_2103_15940_amd as lib  # noqa: E402

NULL, SHAPE, RANGE, ALIAS = -2, -3, -5, -6
BUF = (ctypes.c_float * (1 << 17))()
BASE = ctypes.addressof(BUF)
SHAPES = dict(batch=2, heads=2, kv_heads=2, q_len=4, k_len=4, dim=8, causal=0, window=0, sinks=0, scale=1.0, k_lens=None, q_pos=None)


def view(at, sb=64, st=16, sh=8):
    return lib._CView(BASE + 4 * at, sb, st, sh)


def bwd(dq=view(5000), dk=view(6000), dv=view(7000), **kw):
    a = lib._CAttention(*(SHAPES | kw).values())
    return lib.raw_library().fmt_attention_bwd(a, view(0), view(1000), view(2000), view(3000), view(4000), None, dq, dk, dv, 0, 0,
                                               lib._CFormat(6, 9, 1), None)


@pytest.mark.parametrize("scale", [2.0 ** 90, -2.0 ** 90, 3e38, -3e38, float("inf"), float("nan")])
def test_scales_that_overflow_are_refused(scale):
    assert bwd(scale=scale) == RANGE


@pytest.mark.parametrize("scale", [0.0, 1e-45, -1e27, 1.2e27])
def test_other_scales_are_taken(scale):
    assert bwd(scale=scale) == NULL
