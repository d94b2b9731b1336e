"""Dropout and layer norm on the GPU against their definitions in 64 bits.

Tolerances (u = 2^-24): a thread adds at most 32 values of a row and at most 11 partial sums follow, so a row's mean is within
45 u of the mean magnitude; with that, y is within |gamma| (48 u max|z| rstd + 40 u |xhat|) + 2 u (|y| + |beta|), and dz within
rstd (4 u |g| + 50 u mean|g| + 64 u |xhat| mean|g xhat|) + 2 u |dz|.  Sums over rows pass at most 128 additions one after the
other: 160 u of the sum of magnitudes.  A rounded result has to lie between the roundings of the two ends of that interval."""
import ctypes

import numpy as np
import pytest

import layerdef as L
import oracle

torch = pytest.importorskip("torch")

FORMATS = [(5, 10, True), (5, 10, False), (6, 9, True), (6, 9, False), (8, 7, True), (8, 7, False), (8, 23, True), (4, 23, True)]
U = L.U


@pytest.fixture(scope="module")
def fmt():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2103_15940_amd as lib
    return lib


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def store(fmt, x, f, codes):
    """(tensor as a program holds it, its values)."""
    t = dev(x)
    return (fmt.fmt_pack16(t, f) if codes else t), L.rounded(x, f)


def values(fmt, t, f, result):
    if result == "code16":
        return fmt.fmt_unpack16(t.contiguous(), f).cpu().numpy()
    return t.cpu().numpy()


def close(got, want, tol, f, result, what):
    lo, hi = want - tol, want + tol
    if result != "f32":
        with np.errstate(over="ignore"):
            lo, hi = (L.rounded(np.nextafter(v.astype(np.float32), np.float32(s * np.inf)), f) for v, s in ((lo, -1), (hi, 1)))
    bad = ~((got >= lo) & (got <= hi))
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])


def same_bits(a, b):
    return np.array_equal(a.view(np.uint32)[~np.isnan(b)], b.view(np.uint32)[~np.isnan(b)]) and np.array_equal(np.isnan(a), np.isnan(b))


gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("f", FORMATS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 8), (17, 129), (2, 4097), (300, 1024)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(fmt, f, rows, cols, p):
    rng = np.random.default_rng(rows * 1000 + cols)
    x = (rng.normal(size=(rows, cols)) * np.exp2(rng.normal(size=(rows, cols)) * 6)).astype(np.float32)
    seed, step, site = 0xFEDCBA9876543210, 5 + (3 << 32), 0xFFFFFFFF
    x.reshape(-1)[:: 5][:3] = [np.inf, np.nan, -0.0][: len(x.reshape(-1)[:: 5][:3])]
    kept, factor = L.drop_mask(rows, cols, p, seed, step, site)
    state = fmt.new_rng(seed, step)
    for codes in (False, True):
        if codes and f[0] + f[1] > 15:
            continue
        t, v = store(fmt, x, f, codes)
        with np.errstate(over="ignore", invalid="ignore"):
            want = np.where(kept, v * factor, np.float32(0))
        for result in ("f32", "round", "code16"):
            if result == "code16" and f[0] + f[1] > 15:
                continue
            got = values(fmt, fmt.fmt_dropout(t, p, state, f, site=site, result=result), f, result)
            ref = want if result == "f32" else L.rounded(want, f)
            if result == "code16":
                ref = oracle.unpack16(oracle.pack16(want, f[0], f[1], f[2]), f[0], f[1]).reshape(ref.shape)
            assert same_bits(got, ref), (codes, result)


@gpu
def test_dropout_in_place_strides_and_second_stream(fmt):
    f = (6, 9, True)
    rng = np.random.default_rng(3)
    x = rng.normal(size=(33, 50)).astype(np.float32)
    state = fmt.new_rng(11)
    whole = dev(np.pad(x, ((0, 0), (3, 6)), constant_values=7.0))
    want = fmt.fmt_dropout(dev(x), 0.3, state, f).cpu().numpy()
    part = whole[:, 3:53]
    fmt.fmt_dropout(part, 0.3, state, f, out=part)
    assert same_bits(part.cpu().numpy(), want)
    assert bool((whole[:, :3] == 7).all()) and bool((whole[:, 53:] == 7).all())
    side = torch.cuda.Stream()
    t = dev(x)
    torch.cuda.synchronize()
    got = torch.empty_like(t)
    fmt.fmt_dropout(t, 0.3, state, f, out=got, stream=side)
    side.synchronize()
    assert same_bits(got.cpu().numpy(), want)


@gpu
def test_dropout_in_a_recorded_graph_takes_the_step_at_replay(fmt):
    f = (8, 7, False)
    x = torch.randn(64, 100, device="cuda")
    state = fmt.new_rng(5, 0)
    y = torch.empty_like(x)
    fmt.fmt_dropout(x, 0.5, state, f, out=y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fmt.fmt_dropout(x, 0.5, state, f, out=y)
    seen = []
    for step in (1, 2, 3):
        state.copy_(fmt.new_rng(5, step))
        g.replay()
        torch.cuda.synchronize()
        want = fmt.fmt_dropout(x, 0.5, fmt.new_rng(5, step), f)
        assert torch.equal(y, want)
        seen.append(y.clone())
    assert not torch.equal(seen[0], seen[1])


SHAPES = [(1, 1), (2, 3), (5, 8), (33, 77), (7, 128), (130, 129), (9, 512), (64, 768), (11, 1024), (3, 1025), (5, 2048), (4, 2055),
          (3, 4096), (3, 5000), (2, 8192), (2, 8200), (3, 16384), (2, 16391), (1, 32768)]


def norm_inputs(rows, cols, seed):
    rng = np.random.default_rng(seed)
    return (rng.normal(0.3, 2.0, (rows, cols)).astype(np.float32), rng.normal(1.0, 1.0, (rows, cols)).astype(np.float32),
            rng.normal(1, 0.3, cols).astype(np.float32), rng.normal(0, 0.3, cols).astype(np.float32))


@gpu
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("residual,p", [(False, 0.0), (True, 0.1), (False, 0.5), (True, 0.0)])
def test_norm_forward(fmt, rows, cols, residual, p):
    f = FORMATS[(rows + cols) % 7]
    codes = f[0] + f[1] <= 15 and cols % 2 == 0
    result = ("f32", "round", "code16" if f[0] + f[1] <= 15 else "f32")[(rows + (1 if p else 0)) % 3]
    x, res, gamma, beta = norm_inputs(rows, cols, cols)
    (xt, _), (rt, _) = store(fmt, x, f, codes), store(fmt, res, f, codes)
    state = fmt.new_rng(99, 4)
    y, z, mean, rstd = fmt.fmt_layernorm_fwd(xt, dev(gamma), dev(beta), f, residual=rt if residual else None, p=p, rng=state, site=2,
                                             eps=1e-5, result=result)
    zin = L.norm_input(x, res if residual else None, L.drop_mask(rows, cols, p, 99, 4, 2) if p else None, f)
    if residual or p:
        assert same_bits(values(fmt, z, f, result), zin)
    else:
        assert z is None
    g, b = L.rounded(gamma, f).astype(np.float64), L.rounded(beta, f).astype(np.float64)
    want, m, r = L.norm_fwd(zin, g, b, float(np.float32(1e-5)))
    top = np.abs(zin).max(1).astype(np.float64)
    assert np.all(np.abs(mean.cpu().numpy() - m) <= 45 * U * top)
    assert np.all(np.abs(rstd.cpu().numpy() / r - 1) <= 40 * U + (45 * U * top * r) ** 2)
    xhat = (zin - m[:, None]) * r[:, None]
    tol = np.abs(g) * (48 * U * top[:, None] * r[:, None] + 40 * U * np.abs(xhat)) + 2 * U * (np.abs(want) + np.abs(b))
    close(values(fmt, y, f, result), want, tol, f, result, "y")
    only = fmt.fmt_layernorm_fwd(xt, dev(gamma), dev(beta), f, residual=rt if residual else None, p=p, rng=state, site=2, eps=1e-5,
                                 result=result, keep=False)
    assert torch.equal(only[0].view(torch.int16 if result == "code16" else torch.int32), y.view(torch.int16 if result == "code16" else torch.int32))
    assert only[1:] == (None, None, None)


@gpu
@pytest.mark.parametrize("rows,cols", SHAPES + [(5000, 40), (2049, 1024)])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_norm_backward(fmt, rows, cols, p):
    f = FORMATS[(rows * 3 + cols) % 7]
    codes = f[0] + f[1] <= 15 and (rows + cols) % 2 == 0
    result = ("f32", "round", "code16" if f[0] + f[1] <= 15 else "f32")[(cols + (1 if p else 0)) % 3]
    zin, dy, gamma, _ = norm_inputs(rows, cols, 7 * cols + rows)
    dy = dy * np.float32(0.25)
    (zt, z), (dt, d) = store(fmt, zin, f, codes), store(fmt, dy, f, codes)
    _, m, r = L.norm_fwd(z, 1.0, 0.0, 1e-5)
    m, r = m.astype(np.float32), r.astype(np.float32)
    state = fmt.new_rng(1 << 63, 1)
    dz, dx, dgamma, dbeta = fmt.fmt_layernorm_bwd(dt, zt, dev(m), dev(r), dev(gamma), f, p=p, rng=state, site=9, result=result)
    w = L.rounded(gamma, f).astype(np.float64)
    want, wg, wb = L.norm_bwd(d, z, m, r, w)
    xhat = (z.astype(np.float64) - m[:, None]) * r[:, None]
    g = d * w
    tol = r[:, None] * (4 * U * np.abs(g) + 50 * U * np.abs(g).mean(1, keepdims=True) +
                        64 * U * np.abs(xhat) * np.abs(g * xhat).mean(1, keepdims=True)) + 2 * U * np.abs(want)
    close(values(fmt, dz, f, result), want, tol, f, result, "dz")
    if p:
        kept, factor = L.drop_mask(rows, cols, p, 1 << 63, 1, 9)
        close(values(fmt, dx, f, result), np.where(kept, want * factor, 0.0), np.where(kept, (tol + U * np.abs(want)) * factor, 0.0), f, result, "dx")
    else:
        assert dx is dz
    assert np.all(np.abs(dgamma.cpu().numpy() - wg) <= 160 * U * (np.abs(d) * np.abs(xhat)).sum(0))
    assert np.all(np.abs(dbeta.cpu().numpy() - wb) <= 160 * U * np.abs(d).astype(np.float64).sum(0))
    again = fmt.fmt_layernorm_bwd(dt, zt, dev(m), dev(r), dev(gamma), f, p=p, rng=state, site=9, result=result)
    assert torch.equal(again[2], dgamma) and torch.equal(again[3], dbeta)


@gpu
def test_norm_strides_leading_dimensions_and_no_weights(fmt):
    f = (6, 9, True)
    x, res, _, _ = norm_inputs(37, 100, 5)
    whole, other = dev(np.pad(x, ((0, 0), (1, 10)))), dev(np.pad(res, ((0, 0), (5, 0))))
    a = fmt.fmt_layernorm_fwd(whole[:, 1:101], None, None, f, residual=other[:, 5:])
    one, zero = torch.ones(100, device="cuda"), torch.zeros(100, device="cuda")
    b = fmt.fmt_layernorm_fwd(dev(x), one, zero, f, residual=dev(res))
    for s, t in zip(a, b):
        assert torch.equal(s, t)
    three = fmt.fmt_layernorm_fwd(dev(x).view(37, 1, 100), one, zero, f, residual=dev(res).view(37, 1, 100))
    assert three[0].shape == (37, 1, 100) and three[2].shape == (37, 1) and torch.equal(three[0].view(37, 100), b[0])
    g = fmt.fmt_layernorm_bwd(whole[:, 1:101], other[:, 5:], b[2], b[3], None, f)
    h = fmt.fmt_layernorm_bwd(dev(x), dev(res), b[2], b[3], one, f)
    for s, t in zip(g, h):
        assert torch.equal(s, t)


@gpu
def test_norm_special_values(fmt):
    """A row that is constant, one with an infinity, one with NaN; the others are not touched by them."""
    f = (8, 23, True)
    x, _, gamma, beta = norm_inputs(6, 200, 8)
    clean, m0, r0 = L.norm_fwd(x, gamma.astype(np.float64), beta.astype(np.float64), 1e-5)
    x[1] = 3.0
    x[2, 17] = np.inf
    x[4, 199] = np.nan
    y, _, mean, rstd = fmt.fmt_layernorm_fwd(dev(x), dev(gamma), dev(beta), f)
    y = y.cpu().numpy()
    assert np.allclose(y[1], beta, rtol=0, atol=1e-6) and np.isnan(y[2]).all() and np.isnan(y[4]).all()
    for r in (0, 3, 5):
        assert np.abs(y[r] - clean[r]).max() <= 1e-5
    dropped = fmt.fmt_layernorm_fwd(dev(x), dev(gamma), dev(beta), f, p=1.0, rng=fmt.new_rng(1))
    assert np.array_equal(dropped[0].cpu().numpy(), np.broadcast_to(beta, x.shape)) and bool((dropped[1] == 0).all())


@gpu
def test_empty(fmt):
    f = (6, 9, True)
    none = torch.empty(0, 12, device="cuda")
    w = torch.ones(12, device="cuda")
    y, z, mean, rstd = fmt.fmt_layernorm_fwd(none, w, w, f)
    assert y.shape == (0, 12) and mean.shape == (0,)
    dz, dx, dgamma, dbeta = fmt.fmt_layernorm_bwd(none, none, mean, rstd, w, f)
    assert dz.shape == (0, 12) and bool((dgamma == 0).all()) and bool((dbeta == 0).all())
    assert fmt.fmt_dropout(none, 0.5, fmt.new_rng(1), f).shape == (0, 12)


@gpu
def test_binding_refusals(fmt):
    f = (6, 9, True)
    x, w = torch.randn(4, 6, device="cuda"), torch.ones(6, device="cuda")
    state = fmt.new_rng(1)
    with pytest.raises(TypeError):
        fmt.fmt_dropout(x.double(), 0.1, state, f)
    with pytest.raises(TypeError):
        fmt.fmt_dropout(x.half(), 0.1, state, f)                 # codes of 1/5/10
    with pytest.raises(TypeError):
        fmt.fmt_dropout(x, 0.1, torch.zeros(2, device="cuda"), f)
    with pytest.raises(fmt.FmtError):
        fmt.fmt_dropout(x, 1.5, state, f)
    with pytest.raises(fmt.FmtError):
        fmt.fmt_layernorm_fwd(x, w, w, f, p=0.1)                 # no generator
    with pytest.raises(fmt.FmtError):
        fmt.fmt_layernorm_fwd(x, w, w, f, eps=-1.0)
    with pytest.raises(fmt.FmtError):
        fmt.fmt_layernorm_fwd(x, w, w, (8, 23, True), result="code16")
    with pytest.raises(ValueError):
        fmt.fmt_layernorm_fwd(x, torch.ones(5, device="cuda"), None, f)
    with pytest.raises(ValueError):
        fmt.fmt_layernorm_fwd(x.t(), None, None, f)
    with pytest.raises(TypeError):
        fmt.fmt_layernorm_fwd(x, w, w, f, residual=x.half())
    with pytest.raises(ValueError):
        fmt.fmt_layernorm_fwd(x, w, w, f, result="int8")


def test_arguments_are_checked_before_the_gpu():
    import paper_2103_15940_amd as lib
    c = lib.raw_library()
    f, d0 = lib._CFormat(6, 9, 1), lib._CDropout(0.0, 0, None)
    buf = (ctypes.c_float * 4096)()
    a = ctypes.addressof(buf)
    b, r = a + 8192, a + 12288
    drop = lib._CDropout(0.5, 0, r)
    OK, FORMAT, NULL, SHAPE, ALIGN, RANGE, ALIAS = 0, -1, -2, -3, -4, -5, -6

    def dropout(x=a, ldx=8, y=b, ldy=8, rows=4, cols=8, d=drop, store=0, result=0, f=f):
        return c.fmt_dropout(x, ldx, y, ldy, rows, cols, d, store, result, f, None)
    assert dropout(f=lib._CFormat(9, 9, 1)) == FORMAT and dropout(f=lib._CFormat(8, 23, 1), store=1) == FORMAT
    assert dropout(store=2) == RANGE and dropout(result=3) == RANGE and dropout(d=lib._CDropout(1.5, 0, r)) == RANGE
    assert dropout(d=lib._CDropout(float("nan"), 0, r)) == RANGE and dropout(d=lib._CDropout(0.5, 0, None)) == NULL
    assert dropout(x=None) == NULL and dropout(y=None) == NULL and dropout(d=lib._CDropout(0.5, 0, r + 4)) == ALIGN
    assert dropout(rows=-1) == SHAPE and dropout(ldx=7) == SHAPE and dropout(ldy=7) == SHAPE
    assert dropout(x=a + 2) == ALIGN and dropout(y=a + 4) == ALIAS and dropout(y=a, result=2) == ALIAS and dropout(y=r - 4) == ALIAS
    assert dropout(rows=0) == OK and dropout(cols=0, x=None) == OK

    def fwd(rows=4, cols=8, x=a, ldx=8, res=None, ldres=0, d=d0, gamma=None, beta=None, eps=1e-5, z=None, ldz=0, y=b, ldy=8, mean=None,
            rstd=None, store=0, result=0, f=f):
        return c.fmt_layernorm_fwd(rows, cols, x, ldx, res, ldres, d, gamma, beta, eps, z, ldz, y, ldy, mean, rstd, store, result, f, None)
    assert fwd(cols=32769, ldx=40000, ldy=40000) == SHAPE and fwd(rows=-1) == SHAPE and fwd(ldx=7) == SHAPE
    assert fwd(res=a + 1024, ldres=7) == SHAPE and fwd(z=r, ldz=7) == SHAPE
    assert fwd(x=None) == NULL and fwd(y=None) == NULL and fwd(mean=r) == NULL and fwd(d=lib._CDropout(0.1, 0, None)) == NULL
    assert fwd(eps=-1.0) == RANGE and fwd(eps=float("nan")) == RANGE and fwd(gamma=a + 2) == ALIGN and fwd(mean=r + 1, rstd=r + 64) == ALIGN
    assert fwd(y=a) == ALIAS and fwd(z=b, ldz=8) == ALIAS and fwd(mean=r, rstd=r) == ALIAS and fwd(gamma=b) == ALIAS
    assert fwd(rows=0, x=None, y=None) == OK and fwd(cols=0) == OK and fwd(f=lib._CFormat(1, 9, 1)) == FORMAT

    def bwd(rows=4, cols=8, dy=a, lddy=8, z=a + 512, ldz=8, mean=a + 1024, rstd=a + 1088, gamma=None, d=d0, dz=b, lddz=8, dx=None, lddx=0,
            dgamma=None, dbeta=None, store=0, result=0, f=f):
        return c.fmt_layernorm_bwd(rows, cols, dy, lddy, z, ldz, mean, rstd, gamma, d, dz, lddz, dx, lddx, dgamma, dbeta, store, result, f, None)
    assert bwd(dy=None) == NULL and bwd(mean=None) == NULL and bwd(dz=None) == NULL and bwd(dgamma=r) == NULL
    assert bwd(lddz=7) == SHAPE and bwd(dx=r, lddx=7) == SHAPE and bwd(cols=32769) == SHAPE and bwd(dz=b + 2) == ALIGN
    assert bwd(dz=a) == ALIAS and bwd(dx=b, lddx=8) == ALIAS and bwd(dgamma=r, dbeta=r + 16) == ALIAS
    assert bwd(rows=0, dy=None, z=None, mean=None, rstd=None, dz=None) == OK and bwd(store=5) == RANGE


@gpu
@pytest.mark.parametrize("f", FORMATS + [(7, 8, True), (3, 4, False), (8, 4, False)])
@pytest.mark.parametrize("rows,cols", [(5, 100), (3, 1030), (2, 9000)])
@pytest.mark.parametrize("codes", [False, True])
def test_norm_in_every_format(fmt, f, rows, cols, codes):
    """Every way of rounding, tensors in fp32 and in codes, with values that overflow and underflow the format."""
    if codes and f[0] + f[1] > 15:
        pytest.skip("the format has no 16-bit codes")
    x, res, gamma, beta = norm_inputs(rows, cols, 3)
    if f[0] >= 4:
        x[0, ::7] *= np.float32(2.0 ** -20)
    state = fmt.new_rng(3)
    (xt, _), (rt, _) = store(fmt, x, f, codes), store(fmt, res, f, codes)
    for result in ("f32", "round") + (("code16",) if f[0] + f[1] <= 15 else ()):
        y, z, mean, rstd = fmt.fmt_layernorm_fwd(xt, dev(gamma), dev(beta), f, residual=rt, p=0.25, rng=state, site=1, result=result)
        zin = L.norm_input(x, res, L.drop_mask(rows, cols, 0.25, 3, 0, 1), f)
        assert same_bits(values(fmt, z, f, result), zin)
        g, b = L.rounded(gamma, f).astype(np.float64), L.rounded(beta, f).astype(np.float64)
        want, m, r = L.norm_fwd(zin, g, b, float(np.float32(1e-5)))
        top = np.abs(zin).max(1).astype(np.float64)
        xhat = (zin - m[:, None]) * r[:, None]
        tol = np.abs(g) * (48 * U * top[:, None] * r[:, None] + 40 * U * np.abs(xhat)) + 2 * U * (np.abs(want) + np.abs(b))
        close(values(fmt, y, f, result), want, tol, f, result, "y")
        if result == "code16" and codes:
            dz, dx, dgamma, dbeta = fmt.fmt_layernorm_bwd(rt, z, mean, rstd, dev(gamma), f, p=0.25, rng=state, site=1)
            d = L.rounded(res, f).astype(np.float64)
            want, wg, wb = L.norm_bwd(d, zin, mean.cpu().numpy(), rstd.cpu().numpy(), g)
            gx = d * g
            tol = r[:, None] * (4 * U * np.abs(gx) + 50 * U * np.abs(gx).mean(1, keepdims=True) + 64 * U * np.abs(xhat) *
                                np.abs(gx * xhat).mean(1, keepdims=True)) * (1 + 2.0 ** -10) + 2 * U * np.abs(want)
            close(values(fmt, dz, f, "code16"), want, tol, f, "code16", "dz")


@gpu
def test_dropout_past_32_bits_of_elements(fmt):
    """More than 2^32 elements: the last rows' mask is that of their own blocks, not of blocks 2^32 back."""
    f = (8, 7, False)
    rows, cols = 131080, 32768
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    state = fmt.new_rng(21, 2)
    fmt.fmt_dropout(x, 0.5, state, f, site=4, out=x)
    tail = x[-3:].float().cpu().numpy()
    n0 = (rows - 3) * (cols // 8)
    n = np.arange(n0, n0 + 3 * (cols // 8), dtype=np.uint64)
    full = lambda v: np.full(n.shape, v, dtype=np.uint64)  # noqa: E731
    w = L.philox([n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), full(2), full(4)], [21, 0])
    bits = np.stack([(w[i // 2] >> np.uint64(16 * (i % 2))) & np.uint64(0xFFFF) for i in range(8)], 1).reshape(3, cols)
    assert np.array_equal(tail != 0, bits >= 32768) and set(np.unique(tail)) == {0.0, 2.0}
