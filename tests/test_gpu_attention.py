"""Attention on the GPU, forward and backward, against its definition in 64 bits.

Tolerances (u = 2^-24, n keys).  Products of operands are exact and added in fp32: a score is within e = 64 u scale sum|q||k|
of its value.  exp, the running maximum's factors and the row's sum (n / 2 additions in a lane) leave P within
eps = 3 e + (80 + n / 2) u of it, relatively; P and dS then go through the matrix cores with a relative error rho: 2^-23 for
unrounded results, 2^-15 (two pieces) or 2^-8 (one) for rounded ones.  So

  |o - ref|  <= (eps + rho + (64 + n / 16) u) P |v|
  E = P (|dP - delta| (eps + |lse| u + 8 u) + 64 u |do||v| + (64 u + r) sum |do||o|) + rho |dS|      r: o's own rounding
  |dq - ref| <= scale (E + (64 + n / 16) u |dS|) |k|,  dk, dv alike

A rounded result has to lie between the roundings of the two ends of that interval."""
import ctypes

import numpy as np
import pytest

import layerdef as L

torch = pytest.importorskip("torch")

U = L.U
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def fmt():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2103_15940_amd as lib
    return lib


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def store(fmt, x, f, codes):
    t = dev(x)
    return fmt.fmt_pack16(t, f) if codes else t


def values(fmt, t, f):
    return (fmt.fmt_unpack16(t.contiguous(), f) if t.dtype != torch.float32 else t).cpu().numpy()


def close(got, want, tol, f, result, what):
    lo, hi = want - tol, want + tol
    if result != "f32":
        with np.errstate(over="ignore"):
            lo, hi = (L.rounded(np.nextafter(v.astype(np.float32), np.float32(s * np.inf)), f) for v, s in ((lo, -1), (hi, 1)))
    bad = ~((got >= lo) & (got <= hi))
    assert not bad.any(), (what, int(bad.sum()), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0],
                           float(np.max(np.abs(got - want) / np.maximum(tol, 1e-300))))


def check(fmt, q, k, v, do, f, codes, result, causal=False, window=0, sinks=0, scale=None, lens=None, pos=None, views=lambda t: t):
    """Forward and (with do) backward of numpy inputs against the definition.  views: how the tensors lie in memory."""
    b, nq, h, d = q.shape
    nk, hk = k.shape[1:3]
    scale = d ** -0.5 if scale is None else scale
    rho = {"f32": 2.0 ** -23}.get(result, 2.0 ** -8 if f[1] <= 7 else 2.0 ** -15)
    how = dict(causal=causal, window=window, sinks=sinks, scale=scale, result=result,
               k_lens=None if lens is None else dev(np.asarray(lens, np.int32)), q_pos=None if pos is None else dev(np.asarray(pos, np.int32)))
    tq, tk, tv = (views(store(fmt, t, f, codes)) for t in (q, k, v))
    o, lse = fmt.fmt_attention_fwd(tq, tk, tv, f, **how)
    got = {"o": values(fmt, o, f)}
    only, none = fmt.fmt_attention_fwd(tq, tk, tv, f, keep=False, **how)
    assert none is None and torch.equal(only.view(torch.uint8), o.view(torch.uint8))
    if do is not None:
        tdo = store(fmt, do, f, result == "code16")
        grads = fmt.fmt_attention_bwd(views(tdo), tq, tk, tv, o, lse, f, **how)
        got.update(zip(("dq", "dk", "dv"), (values(fmt, t, f) for t in grads)))
        rdo = L.rounded(do, f).astype(np.float64)
    lse = lse.cpu().numpy()
    vq, vk, vv = (L.rounded(t, f).astype(np.float64) for t in (q, k, v))
    want = {n: np.zeros(t.shape) for n, t in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    tol = {n: np.zeros(t.shape) for n, t in want.items()}
    r = 0.0 if result == "f32" else 2.0 ** -(f[1] + 1)
    for i in range(b):
        n = nk if lens is None else min(max(int(lens[i]), 0), nk)
        seen = L.visible(nq, nk, n, nk - nq if pos is None else int(pos[i]), causal, window, sinks)
        for j in range(h):
            g = j // (h // hk)
            a, x, y = vq[i, :, j], np.where(seen.any(0)[:, None], vk[i, :, g], 0.0), np.where(seen.any(0)[:, None], vv[i, :, g], 0.0)
            ref = L.attention(a, x, y, seen, scale, None if do is None else rdo[i, :, j])
            s = a @ x.T * scale
            with np.errstate(invalid="ignore"):
                p = np.where(seen, np.exp(s - np.where(np.isfinite(ref[1]), ref[1], 0.0)[:, None]), 0.0)
            e = np.where(seen, 64 * U * abs(scale) * (np.abs(a) @ np.abs(x).T), 0.0)
            eps = 3 * e.max(1, keepdims=True, initial=0.0) + (80 + nk / 2) * U
            add = (64 + max(nk, nq * (h // hk)) / 16) * U
            want["o"][i, :, j] = ref[0]
            tol["o"][i, :, j] = (eps + rho + add) * (p @ np.abs(y))
            empty = ~seen.any(1)
            assert np.all(lse[i, j][empty] == -np.inf)
            assert np.all(np.abs(lse[i, j] - ref[1])[~empty] <= (eps[:, 0] + 4 * U * np.abs(ref[1]))[~empty])
            if do is None:
                continue
            w = rdo[i, :, j]
            dp, delta = w @ y.T, (w * ref[0]).sum(1, keepdims=True)
            safe = np.where(np.isfinite(ref[1]), np.abs(ref[1]), 0.0)[:, None]
            ds = p * (dp - delta)
            big = p * (np.abs(dp - delta) * (eps + safe * U + 8 * U) + 64 * U * (np.abs(w) @ np.abs(y).T) +
                       (64 * U + r) * (np.abs(w) * np.abs(ref[0])).sum(1, keepdims=True)) + rho * np.abs(ds)
            want["dq"][i, :, j], tol["dq"][i, :, j] = ref[2], abs(scale) * ((big + add * np.abs(ds)) @ np.abs(x))
            want["dk"][i, :, g] += ref[3]
            tol["dk"][i, :, g] += abs(scale) * ((big + add * np.abs(ds)).T @ np.abs(a))
            want["dv"][i, :, g] += ref[4]
            tol["dv"][i, :, g] += (p * (eps + safe * U + rho + add)).T @ np.abs(w)
    for name in got:
        close(got[name], want[name], tol[name] + 2 * U * np.abs(want[name]), f, result, name)
    return got


def inputs(rng, b, nq, nk, h, hk, d, grad=2.0 ** -6):
    return (1.5 * rng.normal(size=(b, nq, h, d)).astype(np.float32), rng.normal(size=(b, nk, hk, d)).astype(np.float32),
            rng.normal(0.2, 1.0, size=(b, nk, hk, d)).astype(np.float32),
            (rng.normal(size=(b, nq, h, d)) * grad * np.exp2(rng.normal(size=(b, nq, 1, 1)) * 2)).astype(np.float32))


TYPES = [((6, 9, True), False, "f32"), ((6, 9, True), True, "code16"), ((5, 10, True), True, "code16"), ((8, 7, False), True, "code16"),
         ((8, 7, True), False, "f32"), ((6, 9, False), False, "round"), ((4, 3, True), True, "round"), ((5, 10, False), True, "f32"),
         ((7, 15, True), False, "f32")]


@gpu
@pytest.mark.parametrize("f,codes,result", TYPES)
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 37, 5), (False, 20, 3), (True, 1, 0)])
def test_types_and_masks(fmt, f, codes, result, causal, window, sinks):
    rng = np.random.default_rng(f[0] * 100 + window + causal)
    check(fmt, *inputs(rng, 2, 150, 150, 2, 2, 64), f, codes, result, causal, window, sinks)


@gpu
@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 2), (2, 1), (1, 63), (1, 64), (1, 65), (31, 33), (64, 64), (65, 129), (127, 128), (128, 127), (3, 300),
                                   (200, 20), (129, 257)])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(fmt, nq, nk, causal):
    f, codes, result = TYPES[(nq + nk) % 4]
    rng = np.random.default_rng(nq * 1000 + nk)
    check(fmt, *inputs(rng, 2, nq, nk, 3, 3, 40), f, codes, result, causal, 50 if nk > 100 else 0, 2)


@gpu
@pytest.mark.parametrize("d", [1, 2, 3, 7, 8, 16, 17, 31, 32, 33, 40, 64, 65, 72, 80, 96, 100, 127, 128])
def test_head_sizes(fmt, d):
    f, codes, result = TYPES[d % 4]
    rng = np.random.default_rng(d)
    check(fmt, *inputs(rng, 1, 70, 90, 2, 1, d), f, codes, result, True, 33, 2)


@gpu
@pytest.mark.parametrize("h,hk", [(1, 1), (4, 1), (6, 2), (12, 4), (7, 7), (15, 3)])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 30, 4)])
def test_shared_heads(fmt, h, hk, causal, window, sinks):
    f, codes, result = TYPES[h % 4]
    rng = np.random.default_rng(h * 10 + hk)
    check(fmt, *inputs(rng, 2, 61, 61, h, hk, 64), f, codes, result, causal, window, sinks)


@gpu
@pytest.mark.parametrize("f,codes,result", TYPES[:4])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 25, 3), (False, 25, 3)])
def test_sequences_of_several_lengths(fmt, f, codes, result, causal, window, sinks):
    """Lengths from none to more than there are; positions before, inside and past the keys; what lies past a length is NaN."""
    rng = np.random.default_rng(7)
    lens, pos = [0, 1, 64, 65, 200, 999, 130], [0, 0, -20, 30, 190, 10, 500]
    q, k, v, do = inputs(rng, 7, 40, 200, 2, 2, 64)
    for i, n in enumerate(lens):
        if not codes and f[0] == 6:
            k[i, n:], v[i, n:] = np.nan, np.inf
    check(fmt, q, k, v, do, f, codes, result, causal, window, sinks, lens=lens, pos=pos)


@gpu
@pytest.mark.parametrize("f,codes,result", TYPES[:4])
@pytest.mark.parametrize("h,hk,d", [(2, 2, 64), (8, 2, 128), (3, 1, 40), (16, 1, 64), (4, 4, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 4)])
def test_single_tokens(fmt, f, codes, result, h, hk, d, window, sinks):
    """One new token per sequence over a cache."""
    rng = np.random.default_rng(h + d + window)
    lens = [1500, 1, 0, 777, 1024]
    q, k, v, _ = inputs(rng, 5, 1, 1500, h, hk, d)
    for i, n in enumerate(lens):
        if not codes:
            k[i, n:], v[i, n:] = np.inf, np.nan
    check(fmt, q, k, v, None, f, codes, result, True, window, sinks, lens=lens, pos=[n - 1 for n in lens])


@gpu
@pytest.mark.parametrize("nq,h,hk", [(1, 1, 1), (2, 4, 2), (5, 8, 1), (17, 2, 2)])
def test_few_queries_over_many_keys(fmt, nq, h, hk):
    rng = np.random.default_rng(nq)
    for f, codes, result in TYPES[:4]:
        check(fmt, *inputs(rng, 1, nq, 9001, h, hk, 64), f, codes, result, True, 0, 0)


@gpu
def test_extreme_scores(fmt):
    """Scores of some thousand: one key takes all of a row; scores all alike; the scale's sign."""
    f = (6, 9, True)
    rng = np.random.default_rng(4)
    q, k, v, do = inputs(rng, 1, 50, 70, 1, 1, 64)
    check(fmt, q * 64, k * 8, v, do, f, False, "f32", True)
    check(fmt, q, k, v, do, f, False, "f32", True, scale=-0.3)
    check(fmt, q, k, v, do, f, False, "f32", False, scale=0.0)
    check(fmt, q * 0, k, v, do, f, False, "f32", False)


@gpu
@pytest.mark.parametrize("exponent", [-30, -20, -12, 12, 20])
def test_magnitudes(fmt, exponent):
    """Values, keys and gradients far from 1 (scores stay moderate)."""
    f = (6, 9, True)
    rng = np.random.default_rng(exponent + 100)
    q, k, v, do = inputs(rng, 1, 70, 130, 2, 1, 64)
    c = np.float32(2.0 ** exponent)
    check(fmt, q / c if abs(exponent) <= 20 else q, k * c, v, do, f, False, "f32", True)
    check(fmt, q, k, v * c, do, f, False, "f32", True)
    check(fmt, q, k, v, do * c, f, False, "f32", True)
    mixed = v * np.exp2(rng.normal(size=v.shape) * 6).astype(np.float32)
    check(fmt, q, k, mixed, do, f, False, "f32", True)


@gpu
def test_strides(fmt):
    """Parts of one projection, heads before tokens, an expanded input; outputs do not depend on where the inputs lie."""
    f = (6, 9, True)
    rng = np.random.default_rng(5)
    b, n, h, hk, d = 2, 75, 4, 2, 40
    whole = dev(rng.normal(size=(b, n + 3, h + 2 * hk, d)).astype(np.float32))
    q, k, v = whole[:, :n, :h], whole[:, :n, h:h + hk], whole[:, :n, h + hk:]
    o, lse = fmt.fmt_attention_fwd(q, k, v, f, causal=True, result="f32")
    g = torch.randn(b, n, h, d, device="cuda")
    grads = fmt.fmt_attention_bwd(g, q, k, v, o, lse, f, causal=True, result="f32")
    for lay in (lambda t: t.contiguous(), lambda t: t.transpose(1, 2).contiguous().transpose(1, 2), lambda t: t.transpose(0, 2).contiguous().transpose(0, 2)):
        o2, lse2 = fmt.fmt_attention_fwd(lay(q), lay(k), lay(v), f, causal=True, result="f32")
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        for s, t in zip(grads, fmt.fmt_attention_bwd(lay(g), lay(q), lay(k), lay(v), lay(o2), lse2, f, causal=True, result="f32")):
            assert torch.equal(s, t)
    one = k[:1].expand(b, n, hk, d)
    o3, _ = fmt.fmt_attention_fwd(q, one, one, f, causal=True, result="f32")
    o4, _ = fmt.fmt_attention_fwd(q, one.contiguous(), one.contiguous(), f, causal=True, result="f32")
    assert torch.equal(o3, o4)


@gpu
def test_half_and_bfloat16_tensors_are_codes(fmt):
    for dtype, f in ((torch.float16, (5, 10, True)), (torch.bfloat16, (8, 7, False))):
        q, k, v = (torch.randn(2, 50, 2, 64, device="cuda").to(dtype) for _ in range(3))
        o, lse = fmt.fmt_attention_fwd(q, k, v, f, causal=True)
        o2, lse2 = fmt.fmt_attention_fwd(*(t.view(torch.int16) for t in (q, k, v)), f, causal=True)
        assert o.dtype == dtype and o2.dtype == torch.int16 and torch.equal(o.view(torch.int16), o2) and torch.equal(lse, lse2)
        g = torch.randn(2, 50, 2, 64, device="cuda").to(dtype)
        for s in fmt.fmt_attention_bwd(g, q, k, v, o, lse, f, causal=True):
            assert s.dtype == dtype


@gpu
def test_gradients_against_differences(fmt):
    """fp32 values that the format holds exactly, steps of the format: the loss changes by the gradient times the step, up to second order
    (h^2 / 2 |f''| with h = 2^-7 and |f''| a few units of the loss's scale here) and the fp32 error of the two losses (64 u |loss| / h)."""
    f = (6, 9, True)
    g = torch.Generator().manual_seed(3)
    grid = lambda *s: (torch.randint(-64, 65, s, generator=g).float() / 64).cuda()  # noqa: E731
    q, k, v, do = grid(1, 5, 2, 8), grid(1, 6, 1, 8), grid(1, 6, 1, 8), grid(1, 5, 2, 8)
    how = dict(causal=True, window=4, sinks=1, result="f32")
    o, lse = fmt.fmt_attention_fwd(q, k, v, f, **how)
    grads = fmt.fmt_attention_bwd(do, q, k, v, o, lse, f, **how)
    h = 2.0 ** -7
    for n, grad in enumerate(grads):
        for at in ([0, 0, 0, 0], [0, 3, 0, 5], [0, 4, 0, 7]):
            loss = []
            for sign in (1, -1):
                t = [q.clone(), k.clone(), v.clone()]
                t[n][tuple(at)] += sign * h
                loss.append(float((fmt.fmt_attention_fwd(*t, f, **how)[0].double() * do.double()).sum()))
            assert abs((loss[0] - loss[1]) / (2 * h) - float(grad[tuple(at)])) <= h * h + 64 * U * abs(loss[0]) / h


@gpu
def test_same_bits_every_time_streams_and_graphs(fmt):
    f = (8, 7, False)
    q, k, v, g = (torch.randn(2, 300, 4, 64, device="cuda").bfloat16() for _ in range(4))
    o, lse = fmt.fmt_attention_fwd(q, k, v, f, causal=True)
    grads = fmt.fmt_attention_bwd(g, q, k, v, o, lse, f, causal=True)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    o2, lse2 = fmt.fmt_attention_fwd(q, k, v, f, causal=True, stream=side)
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    one, cache = q[:, :1].contiguous(), torch.randn(2, 5000, 4, 64, device="cuda").bfloat16()
    token = fmt.fmt_attention_fwd(one, cache, cache, f)[0]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a = fmt.fmt_attention_fwd(q, k, v, f, causal=True)
        fmt.fmt_attention_bwd(g, q, k, v, *a, f, causal=True)
        fmt.fmt_attention_fwd(one, cache, cache, f)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        a = fmt.fmt_attention_fwd(q, k, v, f, causal=True)
        d = fmt.fmt_attention_bwd(g, q, k, v, *a, f, causal=True)
        tok = fmt.fmt_attention_fwd(one, cache, cache, f)[0]
    for _ in range(3):
        for t in (*a, *d, tok):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a[0], o) and torch.equal(a[1], lse) and torch.equal(tok, token)
        for x, y in zip(d, grads):
            assert torch.equal(x, y)


@gpu
def test_empty(fmt):
    f = (6, 9, True)
    t = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    o, lse = fmt.fmt_attention_fwd(t(2, 3, 4, 8), t(2, 0, 2, 8), t(2, 0, 2, 8), f)
    assert bool((o == 0).all()) and bool((lse == -float("inf")).all())
    dq, dk, dv = fmt.fmt_attention_bwd(t(2, 3, 4, 8), t(2, 3, 4, 8), t(2, 0, 2, 8), t(2, 0, 2, 8), o, lse, f)
    assert bool((dq == 0).all()) and dk.shape == (2, 0, 2, 8)
    k = t(2, 5, 2, 8)
    o, lse = fmt.fmt_attention_fwd(t(2, 0, 4, 8), k, k, f)
    assert o.shape == (2, 0, 4, 8)
    dq, dk, dv = fmt.fmt_attention_bwd(o, t(2, 0, 4, 8), k, k, o, lse, f)
    assert bool((dk == 0).all()) and bool((dv == 0).all())


@gpu
def test_cache_of_more_than_2_to_31_elements(fmt):
    """Keys and values whose offsets pass 32 bits, checked on a window at their end and on sinks at their start."""
    f = (8, 7, False)
    n, hk, d = 1 << 16, 4, 128
    big = torch.zeros(66, n, hk, d, dtype=torch.bfloat16, device="cuda")        # 2.2e9 elements
    rng = np.random.default_rng(6)
    tail = rng.normal(size=(2, 40, hk, d)).astype(np.float32)
    big[65, -20:], big[65, :20] = dev(tail[0, :20]).bfloat16(), dev(tail[0, 20:]).bfloat16()
    q = torch.randn(66, 1, hk, d, device="cuda").bfloat16()
    o, _ = fmt.fmt_attention_fwd(q, big, big, f, causal=True, window=20, sinks=20)
    small = torch.cat((big[65:, :20], big[65:, -20:]), 1).contiguous()
    want, _ = fmt.fmt_attention_fwd(q[65:], small, small, f, causal=True)
    want = want.float()
    assert float((o[65:].float() - want).abs().max()) <= 2.0 ** -6 * float(want.abs().max())


@gpu
def test_binding_refusals(fmt):
    f = (6, 9, True)
    q, k = torch.randn(2, 4, 4, 8, device="cuda"), torch.randn(2, 6, 2, 8, device="cuda")
    for bad in (dict(k=k[:1], v=k[:1]), dict(v=k[:, :5]), dict(q=q.transpose(2, 3)), dict(q=q[0])):
        a = dict(q=q, k=k, v=k) | bad
        with pytest.raises(ValueError):
            fmt.fmt_attention_fwd(a["q"], a["k"], a["v"], f)
    with pytest.raises(TypeError):
        fmt.fmt_attention_fwd(q, k.half(), k.half(), f)
    with pytest.raises(TypeError):
        fmt.fmt_attention_fwd(q, k, k, f, k_lens=torch.tensor([1, 2], device="cuda"))
    with pytest.raises(ValueError):
        fmt.fmt_attention_fwd(q, k, k, f, window=-1)
    for how in (dict(fmt=(8, 23, True)), dict(scale=float("inf"))):
        with pytest.raises(fmt.FmtError):
            fmt.fmt_attention_fwd(q, k, k, **(dict(fmt=f) | how))
    with pytest.raises(fmt.FmtError):
        fmt.fmt_attention_fwd(q[:, :, :3], k, k, f)               # 3 heads over 2
    with pytest.raises(fmt.FmtError):
        wide = torch.randn(1, 2, 1, 129, device="cuda")
        fmt.fmt_attention_fwd(wide, wide, wide, f)
    o, lse = fmt.fmt_attention_fwd(q, k, k, f)
    with pytest.raises(TypeError):
        fmt.fmt_attention_bwd(o, q, k, k, o, lse[:1], f)
    with pytest.raises(TypeError):
        fmt.fmt_attention_bwd(o.half(), q, k, k, o, lse, f)


def test_arguments_are_checked_before_the_gpu():
    import paper_2103_15940_amd as lib
    c = lib.raw_library()
    buf = (ctypes.c_float * (1 << 16))()
    base = ctypes.addressof(buf)
    V = lib._CView
    OK, FORMAT, NULL, SHAPE, ALIGN, RANGE, ALIAS = 0, -1, -2, -3, -4, -5, -6

    def view(at, tokens=4, heads=2, dim=8, **kw):
        return V(*(kw.get(n, x) for n, x in (("data", base + 4 * at), ("sb", tokens * heads * dim), ("st", heads * dim), ("sh", dim))))

    def fwd(q=view(0), k=view(1000), v=view(2000), o=view(3000), lse=None, store=0, result=0, f=(6, 9, 1), **kw):
        a = dict(batch=2, heads=2, kv_heads=2, q_len=4, k_len=4, dim=8, causal=0, window=0, sinks=0, scale=1.0, k_lens=None, q_pos=None) | kw
        return c.fmt_attention_fwd(lib._CAttention(*a.values()), q, k, v, o, lse, store, result, lib._CFormat(*f), None)
    assert fwd(f=(9, 9, 1)) == FORMAT and fwd(f=(8, 16, 1)) == FORMAT and fwd(f=(8, 10, 1), store=1) == FORMAT
    assert fwd(store=7) == RANGE and fwd(result=-1) == RANGE and fwd(causal=2) == RANGE and fwd(window=-1) == RANGE
    assert fwd(sinks=1 << 30) == RANGE and fwd(scale=float("nan")) == RANGE
    assert fwd(dim=0) == SHAPE and fwd(dim=129) == SHAPE and fwd(kv_heads=0) == SHAPE and fwd(heads=3) == SHAPE and fwd(batch=-1) == SHAPE
    assert fwd(batch=70000) == SHAPE and fwd(q=view(0, st=-1)) == SHAPE
    assert fwd(o=view(3000, st=7)) == SHAPE and fwd(o=view(3000, sh=0)) == SHAPE          # outputs that lie over themselves
    assert fwd(q=view(0, data=None)) == NULL and fwd(o=view(0, data=None)) == NULL
    assert fwd(k=view(0, data=base + 1)) == ALIGN and fwd(lse=base + 4 * 5000 + 2) == ALIGN and fwd(k_lens=base + 1) == ALIGN
    assert fwd(o=view(1010)) == ALIAS and fwd(lse=base) == ALIAS and fwd(k_lens=base + 4 * 3001) == ALIAS and fwd(lse=base + 4 * 3010) == ALIAS
    assert fwd(batch=0) == OK and fwd(heads=0) == OK and fwd(q_len=0) == OK

    def bwd(g=view(4000), o=view(3000), lse=base + 4 * 9000, dq=view(5000), dk=view(6000), dv=view(7000), **kw):
        a = dict(batch=2, heads=2, kv_heads=2, q_len=4, k_len=4, dim=8, causal=0, window=0, sinks=0, scale=1.0, k_lens=None, q_pos=None) | kw
        return c.fmt_attention_bwd(lib._CAttention(*a.values()), view(0), view(1000), view(2000), o, g, lse, dq, dk, dv, 0, 0, lib._CFormat(6, 9, 1),
                                   None)
    assert bwd(lse=None) == NULL and bwd(dq=view(0, data=None)) == NULL and bwd(dk=view(5000)) == ALIAS and bwd(dv=view(4001)) == ALIAS
    assert bwd(dk=view(6000, sh=4)) == SHAPE and bwd(dq=view(9000)) == ALIAS
    # slices of one projection's gradient lie side by side, not over one another
    side = dict(sb=4 * 48, st=48, sh=8)
    assert bwd(dq=view(5000, **side), dk=view(5008, **side), dv=view(5032, **side)) == ALIAS
    assert bwd(batch=0, dq=view(5000, **side), dk=view(5016, **side), dv=view(5032, **side)) == OK
