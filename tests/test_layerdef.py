"""The definitions that the transformer layer's operators are compared with, pinned on their own: known values of the generator,
gradients against differences, masks by hand."""
import numpy as np
import pytest

import layerdef as L


def test_generator_known_values():
    for counter, key, want in (
            ([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
            ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
            ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
             [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])):
        assert [int(v) for v in L.philox(counter, key)] == want


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9, 1.0])
def test_dropped_share_and_mean(p):
    kept, factor = L.drop_mask(331, 1003, p, 0x123456789ABCDEF0, 7, 2)
    n = kept.size
    assert abs(kept.mean() - (1 - p)) <= 5 * np.sqrt(p * (1 - p) / n) + 2.0 ** -16
    assert p == 1.0 or abs(kept.mean() * factor - 1) <= 5 * np.sqrt(p / (1 - p) / n) + 1e-6
    other, _ = L.drop_mask(331, 1003, p, 0x123456789ABCDEF0, 7, 3)
    assert p in (0.0, 1.0) or (kept != other).mean() > 0.5 * 2 * p * (1 - p)


def numeric(f, x, h):
    g = np.zeros_like(x)
    for at in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[at] += h
        b[at] -= h
        g[at] = (f(a) - f(b)) / (2 * h)
    return g


def test_norm_gradients_against_differences():
    rng = np.random.default_rng(1)
    z, gamma, beta, dy = rng.normal(0.5, 2.0, (3, 7)), rng.normal(1, 0.3, 7), rng.normal(0, 0.3, 7), rng.normal(size=(3, 7))
    _, mean, rstd = L.norm_fwd(z, gamma, beta, 1e-5)
    dz, dgamma, dbeta = L.norm_bwd(dy, z, mean, rstd, gamma)
    h = 1e-5                                          # differences: h^2 f''' / 6 + 2^-53 |f| / h, a few 1e-10
    loss = lambda z_, g_, b_: (L.norm_fwd(z_, g_, b_, 1e-5)[0] * dy).sum()  # noqa: E731
    assert np.allclose(dz, numeric(lambda t: loss(t, gamma, beta), z, h), rtol=0, atol=1e-8)
    assert np.allclose(dgamma, numeric(lambda t: loss(z, t, beta), gamma, h), rtol=0, atol=1e-8)
    assert np.allclose(dbeta, numeric(lambda t: loss(z, gamma, t), beta, h), rtol=0, atol=1e-8)


@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 3, 1), (False, 2, 2)])
def test_attention_gradients_against_differences(causal, window, sinks):
    rng = np.random.default_rng(2)
    q, k, v, do = (rng.normal(size=(n, 4)) for n in (5, 6, 6, 5))
    seen = L.visible(5, 6, 5, 0, causal, window, sinks)
    seen[3] = False                                   # a row that sees nothing
    o, lse, dq, dk, dv = L.attention(q, k, v, seen, 0.5, do)
    assert np.all(o[3] == 0) and lse[3] == -np.inf and np.all(dq[3] == 0)
    loss = lambda q_, k_, v_: (L.attention(q_, k_, v_, seen, 0.5)[0] * do).sum()  # noqa: E731
    assert np.allclose(dq, numeric(lambda t: loss(t, k, v), q, 1e-5), rtol=0, atol=1e-8)
    assert np.allclose(dk, numeric(lambda t: loss(q, t, v), k, 1e-5), rtol=0, atol=1e-8)
    assert np.allclose(dv, numeric(lambda t: loss(q, k, t), v, 1e-5), rtol=0, atol=1e-8)


def test_visible_by_hand():
    seen = L.visible(4, 8, 7, 4, True, 2, 1)          # queries 4 to 7, seven keys, the last two and the first
    assert [list(np.flatnonzero(r)) for r in seen] == [[0, 3, 4], [0, 4, 5], [0, 5, 6], [0, 6]]
    seen = L.visible(3, 4, 4, 0, False, 2, 0)
    assert [list(np.flatnonzero(r)) for r in seen] == [[0, 1], [0, 1, 2], [1, 2, 3]]
    assert not L.visible(3, 4, 0, 0, False, 0, 4).any() and not L.visible(2, 4, 4, -3, True, 0, 4).any()
