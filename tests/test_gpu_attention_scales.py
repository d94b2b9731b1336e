"""Scales at the ends of their range, for few rows and for many."""
import numpy as np
import pytest

from test_gpu_attention import check, fmt, inputs  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("f,codes", [((8, 7, True), True), ((8, 7, True), False), ((7, 8, True), True)])
@pytest.mark.parametrize("nq", [1, 40])
@pytest.mark.parametrize("exponent", [-100, -60, 60, 89])
def test_scales_far_from_one(fmt, f, codes, nq, exponent):  # noqa: F811
    rng = np.random.default_rng(nq)
    q, k, v, do = inputs(rng, 1, nq, 70, 1, 1, 40, grad=1.0)
    down = 2.0 ** -exponent / 8
    half = 2.0 ** (-exponent // 2)
    if f[0] == 7 and abs(exponent) > 60:
        pytest.skip("past the format's range")
    check(fmt, (q * half / 8).astype(np.float32), (k * (down * 8 / half)).astype(np.float32), v, do if nq > 1 and abs(exponent) <= 60 else None, f, codes,
          "f32", True, scale=2.0 ** exponent)
