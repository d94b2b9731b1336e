"""Attention rounds what it reads as the format does, its overflow to infinity too: fp32 tensors, formats of at most 5 exponent bits, for a few
rows and for many."""
import numpy as np
import pytest

import layerdef as L
from test_gpu_attention import check, fmt, inputs  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FORMATS = [(4, 3, True), (4, 3, False), (5, 2, True), (5, 2, False), (5, 10, False), (5, 10, True), (3, 4, True), (5, 7, True)]


def largest(f):
    """(largest finite value, the least fp32 value that the format rounds to infinity)."""
    bias = (1 << (f[0] - 1)) - 1
    top = (2.0 - 2.0 ** -f[1]) * 2.0 ** bias
    return np.float32(top), np.float32((2.0 - 2.0 ** -(f[1] + 1)) * 2.0 ** bias)


@pytest.mark.parametrize("f", FORMATS)
@pytest.mark.parametrize("nq", [1, 5, 9, 40, 150])
@pytest.mark.parametrize("d", [40, 128])
@pytest.mark.parametrize("sign", [1, -1])
def test_values_that_round_to_infinity(fmt, f, nq, d, sign):  # noqa: F811
    rng = np.random.default_rng(nq + d)
    q, k, v, _ = (np.clip(t, -1.5, 1.5).astype(np.float32) for t in inputs(rng, 2, nq, 200, 2, 2, d))
    least = largest(f)[1]
    over = [least, np.float32(least * 1.1), np.float32(least * 3), np.float32(2.0 ** 60)]
    assert all(np.isinf(L.rounded(np.float32(x), f)) for x in over) and np.isfinite(L.rounded(np.nextafter(least, np.float32(0)), f))
    t = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    clean, lse = fmt.fmt_attention_fwd(t(q), t(k), t(v), f, result="f32")
    assert bool(torch.isfinite(clean).all())
    for value in over:
        bad = v.copy()
        bad[1, 77, 1, 7] = sign * value
        o, _ = fmt.fmt_attention_fwd(t(q), t(k), t(bad), f, result="f32")
        assert not bool(torch.isfinite(o[1, :, 1, 7]).any()), float(value)          # every row sees the key
        assert torch.equal(o[0], clean[0]) and float((o[1, :, 0] - clean[1, :, 0]).abs().max()) <= 1e-5 * float(clean.abs().max())
        bad = k.copy()
        bad[1, 77, 1, 7] = sign * value
        o, ls = fmt.fmt_attention_fwd(t(np.abs(q) + np.float32(0.25)), t(bad), t(v), f, result="f32")
        if sign > 0:                                                                # a score of +infinity takes its rows with it
            assert not bool(torch.isfinite(o[1, :, 1]).any()) and not bool(torch.isfinite(ls[1, 1]).any()), float(value)
        bad = q.copy()
        bad[1, nq - 1, 1, 7] = sign * value
        o, ls = fmt.fmt_attention_fwd(t(bad), t(k), t(v), f, result="f32")
        assert not bool(torch.isfinite(o[1, nq - 1, 1]).any()) and not bool(torch.isfinite(ls[1, 1, nq - 1])), float(value)
        assert bool(torch.isfinite(o[1, :, 0]).all())


@pytest.mark.parametrize("f", FORMATS)
@pytest.mark.parametrize("nq", [4, 60])
def test_the_largest_values_stay(fmt, f, nq):  # noqa: F811
    """Just below the threshold: the largest finite value."""
    rng = np.random.default_rng(nq)
    q, k, v, do = (np.clip(t, -1.5, 1.5).astype(np.float32) for t in inputs(rng, 1, nq, 100, 1, 1, 64, grad=1.0))
    v[0, 30, 0, 3] = np.nextafter(largest(f)[1], np.float32(0))
    v[0, 31, 0, 9] = -np.nextafter(largest(f)[1], np.float32(0))
    check(fmt, q, k, v, do, f, False, "f32")


@pytest.mark.parametrize("f", FORMATS)
def test_nan_stays(fmt, f):  # noqa: F811
    rng = np.random.default_rng(1)
    q, k, v, _ = (np.clip(t, -1.5, 1.5).astype(np.float32) for t in inputs(rng, 1, 50, 100, 1, 1, 64))
    t = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    for which in range(3):
        x = [q.copy(), k.copy(), v.copy()]
        x[which][0, 20, 0, 5] = np.nan
        o, _ = fmt.fmt_attention_fwd(*(t(a) for a in x), f, result="f32")
        assert bool(torch.isnan(o[0, 20, 0] if which == 0 else o[0, :, 0, 5]).all())
