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


def test_slices_of_one_tensor_side_by_side():
    """The gradients of a projection: heads after heads, all three of a head together, heads ahead of tokens."""
    h, d, n = 2, 8, 4
    wide = 3 * h * d
    assert bwd(*(view(5000 + i * h * d, n * wide, wide, d) for i in range(3))) == NULL
    assert bwd(*(view(5000 + i * d, n * wide, wide, 3 * d) for i in range(3))) == NULL
    assert bwd(*(view(5000 + i * d, 3 * h * n * d, 3 * d, 3 * n * d) for i in range(3))) == NULL
    assert bwd(*(view(5000 + i * n * d, 3 * h * n * d, d, 3 * n * d) for i in range(3))) == NULL
    assert bwd(*(view(5000 + i * d, n * wide, wide, 2 * d) for i in range(3))) == ALIAS          # the third of a head is the first of the next
    assert bwd(*(view(5000 + i * (d - 1), n * wide, wide, 3 * d) for i in range(3))) == ALIAS
    assert bwd(view(5000, n * wide, wide, 3 * d), view(5000 + d, n * (wide + 8), wide + 8, 3 * d), view(6000)) == ALIAS
    assert bwd(dk=view(5000 + 4 * 16)) == ALIAS and bwd(dk=view(5000 + 2 * 64)) == NULL          # the second sequence of dq, and past it


def test_no_overlap_is_taken():
    """Random layouts: where two outputs share an element by counting, the call is refused."""
    import numpy as np
    rng = np.random.default_rng(1)
    taken = refused = 0
    for _ in range(4000):
        b, h, n, nk, d = (int(v) for v in (rng.integers(1, 4), rng.integers(1, 4), rng.integers(1, 4), rng.integers(1, 4), rng.integers(1, 5)))
        order = rng.permutation(3)
        strides, inner = [0, 0, 0], d * int(rng.integers(1, 4))
        sizes = (b, max(n, nk), h)
        for i in order:
            strides[i] = inner
            inner = inner * sizes[i] + int(rng.integers(0, 3)) * d
        other = list(strides) if rng.uniform() < 0.8 else [s + int(rng.integers(0, 3)) for s in strides]
        at = 20000 + int(rng.integers(-2 * inner, 2 * inner + 1))
        rc = bwd(lib._CView(BASE + 4 * 20000, *strides), lib._CView(BASE + 4 * at, *other), view(60000, 4000, 400, 40), batch=b, heads=h, kv_heads=h,
                 q_len=n, k_len=nk, dim=d)
        ids = [{first + i * s[0] + t * s[1] + j * s[2] + c for i in range(b) for t in range(m) for j in range(h) for c in range(d)}
               for first, s, m in ((20000, strides, n), (at, other, nk))]
        if rc == SHAPE:
            continue
        assert rc in (NULL, ALIAS)
        if ids[0] & ids[1]:
            assert rc == ALIAS, (b, n, nk, h, d, strides, other, at)
        taken += rc == NULL
        refused += rc == ALIAS
    assert taken > 500 and refused > 500


@pytest.mark.gpu
def test_gradients_into_one_projection():
    """q, k and v of a head next to one another, and their gradients into a tensor of the same layout."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    b, n, h, d = 2, 70, 3, 24
    f = (6, 9, True)
    x, g = torch.randn(b, n, h, 3, d, device="cuda"), torch.randn(b, n, h, d, device="cuda")
    q, k, v = x.unbind(3)
    o, lse = lib.fmt_attention_fwd(q, k, v, f, causal=True, result="f32")
    want = lib.fmt_attention_bwd(g, q, k, v, o, lse, f, causal=True, result="f32")
    out = torch.zeros_like(x)
    at = lambda t: lib._CView(t.data_ptr(), *t.stride()[:3])  # noqa: E731
    a = lib._CAttention(b, h, h, n, n, d, 1, 0, 0, d ** -0.5, None, None)
    rc = lib.raw_library().fmt_attention_bwd(a, at(q), at(k), at(v), at(o), at(g), lse.data_ptr(), *(at(t) for t in out.unbind(3)), 0, 0,
                                             lib._CFormat(*f[:2], 1), torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    for x, y in zip(out.unbind(3), want):
        assert torch.equal(x, y)
