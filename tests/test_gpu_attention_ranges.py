"""Attention where its kernels change their way: elements out of the fp16 operands' range, in some tiles only; tiles whose rows are taken in
parts; every way that codes and fp32 are read.  Tolerances as in test_gpu_attention.py."""
import numpy as np
import pytest

import layerdef as L
from test_gpu_attention import check, fmt, inputs, values  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SIX, BF16 = (6, 9, True), (8, 7, True)


@pytest.mark.parametrize("f,codes,result", [(SIX, False, "f32"), (SIX, True, "code16"), (BF16, True, "code16"), ((7, 8, False), True, "round")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where", ["q", "k", "v", "do"])
def test_one_large_element(fmt, f, codes, result, d, where):  # noqa: F811
    """One element of 300 among those around 1: the workgroups that meet it go the other way, the others do not."""
    rng = np.random.default_rng(d)
    q, k, v, do = inputs(rng, 2, 300, 300, 2, 2, d)
    t = {"q": q, "k": k, "v": v, "do": do}[where]
    t[1, 200, 1, 5] = 300.0
    check(fmt, q * np.float32(0.1) if where in "qk" else q, k, v, do, f, codes, result, True, 100, 3)


@pytest.mark.parametrize("limit", [111.0, 112.0, 127.0, 127.75, 127.9, 128.0, 255.0])
def test_around_the_limit(fmt, limit):  # noqa: F811
    rng = np.random.default_rng(1)
    q, k, v, do = inputs(rng, 1, 70, 130, 1, 1, 64)
    v[0, 50, 0, 3] = limit
    k[0, 60, 0, 2] = limit / 4096
    for f, codes, result in ((SIX, False, "f32"), (SIX, True, "f32"), (BF16, False, "f32"), (BF16, True, "code16")):
        check(fmt, q, k, v, do, f, codes, result, True)


@pytest.mark.parametrize("f,codes,result", [(SIX, False, "f32"), (SIX, True, "code16"), (BF16, True, "code16"), ((5, 10, False), False, "round")])
@pytest.mark.parametrize("n,h,hk,window,sinks", [(700, 2, 2, 20, 5), (900, 4, 2, 100, 130), (650, 1, 1, 1, 1), (1000, 3, 1, 33, 300)])
def test_sinks_that_many_rows_see(fmt, f, codes, result, n, h, hk, window, sinks):  # noqa: F811
    rng = np.random.default_rng(n)
    check(fmt, *inputs(rng, 1, n, n, h, hk, 40), f, codes, result, True, window, sinks)


@pytest.mark.parametrize("f,codes,result", [((4, 3, True), True, "round"), ((4, 3, False), False, "f32"), ((7, 8, True), True, "code16"), ((2, 5, True), True, "round"),
                                            ((5, 10, False), True, "code16"), ((6, 5, True), True, "f32"), ((8, 4, False), True, "code16"),
                                            ((8, 10, True), False, "f32"), ((3, 12, True), True, "code16"), ((7, 15, False), False, "round"),
                                            ((5, 10, True), False, "round"), ((8, 7, False), False, "code16")])
@pytest.mark.parametrize("nq,h,hk,d", [(1, 1, 1, 64), (1, 2, 1, 128), (2, 2, 1, 40), (1, 7, 1, 64), (1, 8, 1, 128), (90, 2, 1, 64), (40, 1, 1, 100)])
def test_every_way_of_reading(fmt, f, codes, result, nq, h, hk, d):  # noqa: F811
    """Formats of every kind, with rows for each of the kernels: 1, 2, 4 and 8 rows per head of keys, and tiles."""
    rng = np.random.default_rng(nq + d)
    q, k, v, do = inputs(rng, 2, nq, 700 if nq <= 2 else 150, h, hk, d)
    if f[0] <= 3:
        q, k, v, do = (np.clip(t, -1.5, 1.5) for t in (q, k, v, do * 16))
    check(fmt, q, k, v, do, f, codes, result, True, 600 if nq <= 2 else 0, 2)


@pytest.mark.parametrize("exponent", [-29, -20, 10, 20])
@pytest.mark.parametrize("h", [1, 4])
def test_single_tokens_of_any_magnitude(fmt, exponent, h):  # noqa: F811
    """Values near the format's ends, in codes: their bits are used as fp32's."""
    rng = np.random.default_rng(5)
    q, k, v, _ = inputs(rng, 2, 1, 900, h, 1, 64)
    c = np.float32(2.0 ** exponent)
    check(fmt, q, k, v * c, None, SIX, True, "f32", True)
    check(fmt, q / c if abs(exponent) <= 20 else q, k * c, v, None, SIX, True, "f32", True)


@pytest.mark.parametrize("f", [SIX, BF16, (5, 10, True), (7, 8, True)])
@pytest.mark.parametrize("nq", [1, 50])
@pytest.mark.parametrize("codes", [False, True])
def test_infinities_and_nan(fmt, f, nq, codes):  # noqa: F811
    """A visible NaN or infinity in V makes the rows of its head that see it non-finite, and leaves other heads and sequences as they are; past
    the length it is not looked at, and the gradient of what is not looked at is zero."""
    rng = np.random.default_rng(6)
    q, k, v, do = inputs(rng, 2, nq, 200, 2, 2, 64)
    lens = [150, 200]
    make = lambda t: fmt.fmt_pack16(torch.from_numpy(t).cuda(), f) if codes else torch.from_numpy(t).cuda()  # noqa: E731
    how = dict(k_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), result="f32")
    clean, lse = fmt.fmt_attention_fwd(make(q), make(k), make(v), f, **how)
    bad_v, bad_k = v.copy(), k.copy()
    bad_v[0, 150:], bad_k[0, 150:] = np.nan, np.inf
    same, lse2 = fmt.fmt_attention_fwd(make(q), make(bad_k), make(bad_v), f, **how)
    assert torch.equal(clean, same) and torch.equal(lse, lse2)
    g = torch.from_numpy(do).cuda()
    one, two = (fmt.fmt_attention_bwd(g, make(q), make(a), make(b), clean, lse, f, **how) for a, b in ((k, v), (bad_k, bad_v)))
    for s, t in zip(one, two):
        assert torch.equal(s, t)
    assert bool((one[1][0, 150:] == 0).all()) and bool((one[2][0, 150:] == 0).all())
    for value in (np.inf, np.nan):
        bad_v = v.copy()
        bad_v[1, 20, 1, 7] = value
        out, _ = fmt.fmt_attention_fwd(make(q), make(k), make(bad_v), f, **how)
        assert not bool(torch.isfinite(out[1, :, 1, 7]).any())
        assert torch.equal(out[0], clean[0])
        assert float((out[1, :, 0] - clean[1, :, 0]).abs().max()) <= 1e-5 * float(clean.abs().max())


def test_offsets_past_32_bits_backward(fmt):  # noqa: F811
    """Strides that put sequences 2^31 elements and more apart."""
    f = (8, 7, True)
    big = torch.zeros((1 << 31) + 70 * 128, dtype=torch.bfloat16, device="cuda")
    view = lambda first: torch.as_strided(big, (2, 50, 1, 64), (1 << 31, 128, 64, 1), first)  # noqa: E731
    rng = np.random.default_rng(2)
    q, k, v, do = inputs(rng, 2, 50, 50, 1, 1, 64)
    store = [torch.from_numpy(t).cuda().bfloat16() for t in (q, k, v, do)]
    view(0).copy_(store[1])
    view(64).copy_(store[2])
    o, lse = fmt.fmt_attention_fwd(store[0], view(0), view(64), f, causal=True)
    o2, lse2 = fmt.fmt_attention_fwd(*store[:3], f, causal=True)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for s, t in zip(fmt.fmt_attention_bwd(store[3], store[0], view(0), view(64), o, lse, f, causal=True),
                    fmt.fmt_attention_bwd(store[3], *store[:3], o, lse, f, causal=True)):
        assert torch.equal(s, t)


@pytest.mark.parametrize("f,codes", [(SIX, True), (SIX, False), (BF16, True)])
@pytest.mark.parametrize("h", [4, 16, 32])
def test_no_drift_over_many_keys(fmt, f, codes, h):  # noqa: F811
    """A part's running sums pass over thousands of keys: their error is that of random roundings, not one that grows with every tile.
    A score has an error of a few 2^-24, a weight's is as large, and n additions to a sum of random signs put sqrt(n / 2) 2^-25 beside it,
    n = 8191 / 16 keys to a lane at most: 2^-20 in all."""
    g = torch.Generator(device="cuda").manual_seed(h)
    b, n, hk, d = 48, 8191, 4, 64
    q, k, v = (torch.randn(s, generator=g, device="cuda") for s in ((b, 1, h, d), (b, n, hk, d), (b, n, hk, d)))
    t = [fmt.fmt_quantize(x.reshape(-1, d), f).view(x.shape) for x in (1.5 * q, k, v)]
    o, lse = fmt.fmt_attention_fwd(*(fmt.fmt_pack16(x, f) if codes else x for x in t), f, result="f32")
    wrong, size = 0.0, 0.0
    for i in range(0, b, 12):
        qd, kd, vd = (x[i].double().cpu() for x in t)
        s = torch.matmul(qd.view(hk, h // hk, d), kd.permute(1, 2, 0).contiguous()) * 0.125
        want = torch.matmul(torch.softmax(s, 2), vd.transpose(0, 1).contiguous()).view(h, d)
        wrong += float((o[i, 0].double().cpu() - want).square().sum())
        size += float(want.square().sum())
        # lse: rounded once itself, beside the largest score's error, of 64 products added in 8 steps and 3 and times the scale
        top = torch.matmul(qd.abs().view(hk, h // hk, d), kd.abs().permute(1, 2, 0).contiguous()).amax(2) * 0.125
        want = torch.logsumexp(s, 2)
        assert bool(((lse[i].view(hk, h // hk).double().cpu() - want).abs() <= 2.0 ** -24 * (2 * want.abs() + 14 * top)).all())
    assert wrong ** 0.5 <= 2.0 ** -20 * size ** 0.5


@pytest.mark.parametrize("f,codes,result", [(BF16, True, "code16"), (SIX, False, "f32")])
@pytest.mark.parametrize("batch,h,hk,n,sinks", [(64, 2, 2, 512, 4), (64, 4, 2, 512, 130), (43, 3, 3, 515, 1)])
def test_sinks_in_parts_where_sequences_are_many(fmt, f, codes, result, batch, h, hk, n, sinks):  # noqa: F811
    """Many tiles of keys, of which only those with sinks are seen by rows outside their window."""
    rng = np.random.default_rng(n)
    check(fmt, *inputs(rng, batch, n, n, h, hk, 16), f, codes, result, True, 30, sinks)
