"""Dropout, layer norm and attention by their definitions, in 64 bits on the CPU (numpy): what the tests of the transformer
layer's operators compare with.  Rounding to a format is the oracle's."""
import math

import numpy as np

import oracle

U = 2.0 ** -24      # half a unit in the last place of fp32, relative


def rounded(x, fmt):
    """R of fp32 values, as fp32."""
    return oracle.quantize(np.ascontiguousarray(x, dtype=np.float32), fmt[0], fmt[1], bool(fmt[2])).reshape(np.shape(x))


def philox(counter, key):
    """Philox-4x32 with ten rounds: arrays of four counter words, two key words; four words."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def drop_mask(rows, cols, p, seed, step, site):
    """(kept, factor) of a dropout."""
    least = int(math.floor(float(np.float32(p)) * 65536 + 0.5))
    blocks = (cols + 7) // 8
    n = np.arange(rows * blocks, dtype=np.uint64)
    full = lambda v: np.full(n.shape, v, dtype=np.uint64)  # noqa: E731
    w = philox([n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), full(step & 0xFFFFFFFF), full(site)],
               [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF])
    bits = np.stack([(w[i // 2] >> np.uint64(16 * (i % 2))) & np.uint64(0xFFFF) for i in range(8)], 1).astype(np.int64)
    kept = bits.reshape(rows, blocks * 8)[:, :cols] >= least
    return kept, np.float32(65536.0 / (65536 - least)) if least < 65536 else np.float32(0)


def norm_input(x, residual, mask, fmt):
    """z, as fp32: the two single-precision operations on the way are rounded as such."""
    h = rounded(x, fmt)
    if mask is not None:
        kept, factor = mask
        with np.errstate(over="ignore", invalid="ignore"):
            h = np.where(kept, h * factor, np.float32(0))
    if residual is not None:
        h = rounded(residual, fmt) + h
    return rounded(h, fmt) if mask is not None or residual is not None else h


def norm_fwd(z, gamma, beta, eps):
    z = z.astype(np.float64)
    mean = z.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((z - mean) ** 2).mean(1, keepdims=True) + eps)
    return (z - mean) * rstd * gamma + beta, mean[:, 0], rstd[:, 0]


def norm_bwd(dy, z, mean, rstd, gamma):
    dy, z, mean, rstd, gamma = (np.asarray(v, dtype=np.float64) for v in (dy, z, mean, rstd, gamma))
    xhat = (z - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dz = rstd[:, None] * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
    return dz, (dy * xhat).sum(0), dy.sum(0)


def visible(q_len, k_len, length, first, causal, window, sinks):
    """Which keys each query sees: [q_len, k_len]."""
    i, j = first + np.arange(q_len)[:, None], np.arange(k_len)[None, :]
    seen = (j < length) & (i == i)
    if causal:
        seen = seen & (j <= i)
    if window:
        seen = seen & ((np.abs(i - j) < window) | (j < sinks))
    return seen


def attention(q, k, v, seen, scale, do=None):
    """One head: q [m, d], k and v [n, d], seen [m, n].  (o, lse), and with do (o, lse, dq, dk, dv).  P is an fp32 number: what lies
    below its smallest normal one is 0."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    used = seen.any(0)
    k, v = np.where(used[:, None], k, 0.0), np.where(used[:, None], v, 0.0)
    s = np.where(seen, q @ k.T * scale, -np.inf)
    top = s.max(1, initial=-np.inf, keepdims=True)
    with np.errstate(divide="ignore"):
        p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
        total = p.sum(1, keepdims=True)
        lse = (np.where(np.isfinite(top), top, -np.inf) + np.log(total))[:, 0]
    p = p / np.where(total == 0, 1.0, total)
    p = np.where(p < 2.0 ** -126, 0.0, p)
    o = p @ v
    if do is None:
        return o, lse
    do = np.asarray(do, dtype=np.float64)
    ds = p * (do @ v.T - (do * o).sum(1, keepdims=True)) * scale
    return o, lse, ds @ k, ds.T @ q, p.T @ do
