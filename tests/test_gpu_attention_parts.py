"""Attention's gradients where a tile's rows are taken in parts, and some of the parts leave the fp16 operands and others do not: every row
is added up once.  Tolerances as in test_gpu_attention.py."""
import numpy as np
import pytest

from test_gpu_attention import check, fmt, inputs  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SIX, BF16, HALF = (6, 9, True), (8, 7, True), (5, 10, True)


@pytest.mark.parametrize("f,codes,result", [(SIX, False, "f32"), (BF16, True, "code16"), (SIX, True, "code16")])
@pytest.mark.parametrize("b,n,h,hk,d,row", [(1, 2048, 8, 8, 64, 300), (1, 2048, 8, 8, 64, 1000), (1, 1111, 6, 2, 40, 90), (2, 1000, 4, 4, 64, 600),
                                            (1, 1500, 2, 2, 128, 400)])
def test_one_part_out_of_range(fmt, f, codes, result, b, n, h, hk, d, row):  # noqa: F811
    """One element of Q of 300 in one part's rows, in each head."""
    rng = np.random.default_rng(n + row)
    q, k, v, do = inputs(rng, b, n, n, h, hk, d)
    q *= np.float32(0.1)
    q[:, row, :, 5] = 300.0
    check(fmt, q, k, v, do, f, codes, result, True)


@pytest.mark.parametrize("window,sinks", [(20, 5), (60, 130)])
@pytest.mark.parametrize("n,row", [(2000, 300), (2000, 1500), (1300, 900)])
def test_one_part_of_the_sinks_out_of_range(fmt, window, sinks, n, row):  # noqa: F811
    rng = np.random.default_rng(n + row)
    q, k, v, do = inputs(rng, 1, n, n, 2, 2, 64)
    q *= np.float32(0.1)
    q[:, row, :, 5] = 300.0
    check(fmt, q, k, v, do, SIX, False, "f32", True, window, sinks)


@pytest.mark.parametrize("row", [300, 1000])
@pytest.mark.parametrize("result", ["f32", "code16"])
def test_one_part_with_large_ds(fmt, row, result):  # noqa: F811
    """binary16: one row's dS past 65504 (in the units it is held in): half of the row's weight on one key, dO along that key's V."""
    rng = np.random.default_rng(row)
    n, key = 2048, 140
    q, k, v, do = inputs(rng, 1, n, n, 8, 8, 64)
    v *= np.float32(16.0)
    q[0, row] = k[0, key] * np.float32(0.75)
    do[0, row] = np.where(v[0, key] > 0, 1.0, -1.0) * np.float32(4.0)              # the largest of all rows: no other's power of two holds it down
    check(fmt, q, k, v, do, HALF, True, result, True)
