"""Attention's bits where magnitudes lie far apart: every element of an operand counts with all of its bits, and the gradients of a key with the
rows that see it, whatever other rows, channels or tokens of the same tile hold.  Tolerances as in test_gpu_attention.py, element by element."""
import numpy as np
import pytest

from test_gpu_attention import check, fmt, inputs  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SIX, BF16, HALF = (6, 9, True), (8, 7, True), (5, 10, True)
TYPES = [(SIX, False, "f32"), (BF16, True, "f32"), (BF16, True, "code16"), (BF16, False, "f32"), ((7, 8, True), True, "f32")]


@pytest.mark.parametrize("f,codes,result", TYPES)
@pytest.mark.parametrize("exponent", [-20, -30, -36, -45])
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (True, 40, 3)])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_do_far_apart(fmt, f, codes, result, exponent, causal, window, sinks, d):  # noqa: F811
    """The last rows' dO far below the first's: keys that only they see."""
    rng = np.random.default_rng(exponent + 100)
    q, k, v, do = inputs(rng, 1, 330, 330, 2, 2, d, grad=1.0)
    do[:, 250:] *= np.float32(2.0 ** exponent)
    check(fmt, q, k, v, do, f, codes, result, causal, window, sinks)


@pytest.mark.parametrize("f,codes,result", TYPES + [((5, 10, True), True, "f32")])
@pytest.mark.parametrize("n,h,hk", [(150, 2, 2), (700, 2, 1)])
def test_rows_of_do_of_any_size(fmt, f, codes, result, n, h, hk):  # noqa: F811
    """Rows of dO spread over some eighty binades (over thirty where the format has no more), a third of them zero; the rows' order is not theirs."""
    rng = np.random.default_rng(n)
    q, k, v, do = inputs(rng, 1, n, n, h, hk, 40, grad=1.0)
    wide = 40 if f[0] == 8 else 14 if f[0] == 6 else 30 if f[0] == 7 else 6
    do *= np.exp2(rng.uniform(-wide, wide, size=(1, n, h, 1))).astype(np.float32) * (rng.uniform(size=(1, n, h, 1)) > 0.3)
    check(fmt, q, k, v, do, f, codes, result, True)


@pytest.mark.parametrize("f,codes,result", [(SIX, False, "f32"), (BF16, True, "f32")])
@pytest.mark.parametrize("n", [200, 1500])
def test_keys_that_get_little_weight(fmt, f, codes, result, n):  # noqa: F811
    """A few keys take most of every row; the others' dK and dV are small, and have their bits."""
    rng = np.random.default_rng(n)
    q, k, v, do = inputs(rng, 1, n, n, 1, 1, 64, grad=1.0)
    q[..., 0], k[..., 0] = 4.0, 0.0
    k[:, :3, :, 0] = 18.0                        # scores of about 9 more
    check(fmt, q, k, v, do, f, codes, result, True)


@pytest.mark.parametrize("f,codes,result", TYPES[:2] + TYPES[3:])
@pytest.mark.parametrize("exponent", [-25, -28, -30])
@pytest.mark.parametrize("where", ["q", "k", "both"])
def test_small_scores_and_a_large_scale(fmt, f, codes, result, exponent, where):  # noqa: F811
    """Scores are Q K^T times the scale: operands of 2^-28 count where the scale is 2^28."""
    rng = np.random.default_rng(exponent + 50)
    q, k, v, do = inputs(rng, 1, 130, 150, 2, 1, 64)
    c, down = 2.0 ** -exponent / 8, np.float32(2.0 ** exponent)
    if where == "both":
        check(fmt, q * np.float32(2.0 ** (exponent // 2)), k * np.float32(2.0 ** (exponent - exponent // 2)), v, do, f, codes, result, True, scale=c)
    else:
        check(fmt, q * down if where == "q" else q, k * down if where == "k" else k, v, do, f, codes, result, True, scale=c)


@pytest.mark.parametrize("f,codes,result", TYPES + [((6, 4, True), True, "f32"), ((7, 8, False), False, "f32")])
@pytest.mark.parametrize("what", ["channel", "tokens", "element"])
@pytest.mark.parametrize("exponent", [-25, -30, -37, -50, -90])
@pytest.mark.parametrize("nq,nk,h,hk,d,window", [(150, 150, 2, 2, 64, 0), (90, 500, 2, 1, 128, 70), (40, 1700, 1, 1, 40, 0), (9, 130, 1, 1, 100, 0)])
def test_small_v_beside_ordinary(fmt, f, codes, result, what, exponent, nq, nk, h, hk, d, window):  # noqa: F811
    """Output: a channel, the first tokens, or single elements of V far below the others."""
    if exponent < -37 and f[0] == 6:
        pytest.skip("below the format's smallest values")
    rng = np.random.default_rng(nk - exponent)
    q, k, v, _ = inputs(rng, 2, nq, nk, h, hk, d)
    c = np.float32(2.0 ** exponent)
    if what == "channel":
        v[..., 7] *= c
    elif what == "tokens":
        v[:, :70] *= c
    else:
        v[rng.uniform(size=v.shape) < 0.002] *= c
        v[:, :3, :, 5] *= c
    check(fmt, q, k, v, None, f, codes, result, True, window, 0)


@pytest.mark.parametrize("f,codes,result", [(SIX, False, "f32"), (BF16, True, "code16"), (HALF, True, "f32")])
@pytest.mark.parametrize("exponent", [-12, 4, 6])
@pytest.mark.parametrize("n,window,sinks", [(400, 40, 0), (300, 0, 0), (200, 1, 0), (200, 1, 2)])
def test_v_far_from_one_in_blocks(fmt, f, codes, result, exponent, n, window, sinks):  # noqa: F811
    """dS as large and as small as V makes it: blocks of tokens longer than the window; rows that see one key, whose dS is nothing but rounding."""
    rng = np.random.default_rng(n + exponent)
    q, k, v, do = inputs(rng, 1, n, n, 2, 2, 64, grad=1.0)
    v[:, 90:250] *= np.float32(2.0 ** exponent)
    check(fmt, q, k, v, do, f, codes, result, True, window, sinks)


@pytest.mark.parametrize("f,codes,result", TYPES)
@pytest.mark.parametrize("where", ["q", "k", "v", "do"])
@pytest.mark.parametrize("what", ["channel", "tokens", "element"])
@pytest.mark.parametrize("exponent", [-26, -30])
@pytest.mark.parametrize("d", [40, 128])
def test_small_beside_ordinary(fmt, f, codes, result, where, what, exponent, d):  # noqa: F811
    """A channel, the first tokens, or single elements of one operand far below the others."""
    rng = np.random.default_rng(d)
    q, k, v, do = inputs(rng, 1, 150, 150, 2, 2, d, grad=1.0)
    t = {"q": q, "k": k, "v": v, "do": do}[where]
    c = np.float32(2.0 ** exponent)
    if what == "channel":
        t[..., 7] *= c
    elif what == "tokens":
        t[:, :70] *= c
    else:
        t[rng.uniform(size=t.shape) < 0.002] *= c
        t[:, :3, :, 5] *= c
    check(fmt, q, k, v, do, f, codes, result, True)


@pytest.mark.parametrize("f,codes,result", [(SIX, False, "f32"), (SIX, True, "f32"), (BF16, True, "f32"), (HALF, True, "f32")])
@pytest.mark.parametrize("score", [6, 10, 14])
@pytest.mark.parametrize("nq", [5, 60])
def test_a_sink_without_value(fmt, f, codes, result, score, nq):  # noqa: F811
    """The first key takes nearly all of every row and its V is zero: the output is what the others, of little weight, leave."""
    rng = np.random.default_rng(score)
    q, k, v, do = inputs(rng, 1, nq, 700, 1, 1, 64, grad=1.0)
    q[..., 0], k[..., 0] = 4.0, 0.0
    k[:, 0, :, 0] = 2.0 * score                  # a score of `score` more
    v[:, 0] = 0.0
    check(fmt, q, k, v, do if score <= 6 else None, f, codes, result, False)


@pytest.mark.parametrize("f,codes,result", [(SIX, False, "f32"), (BF16, True, "f32"), (BF16, True, "code16"), ((7, 8, True), True, "f32"), (HALF, False, "f32")])
@pytest.mark.parametrize("d,stretch", [(3, 6.0), (40, 4.0), (64, 3.0), (128, 5.0)])
@pytest.mark.parametrize("window", [0, 7])
def test_rows_that_one_key_takes(fmt, f, codes, result, d, stretch, window):  # noqa: F811
    """Scores of some hundred: weights of 1 and of 2^-100 and less, and a dS that is nothing but rounding, or zero, or the smallest number there is."""
    rng = np.random.default_rng(d)
    q, k, v, do = inputs(rng, 3, 90, 90, 3, 1, d, grad=1.0)
    v[:, ::3] *= np.float32(30.0)
    check(fmt, q * np.float32(stretch), k * np.float32(stretch), v, do, f, codes, result, window > 0, window, 130 if window else 0)


@pytest.mark.parametrize("f,codes", [(SIX, False), (BF16, True), ((7, 8, True), True), ((8, 4, True), False), ((8, 10, True), False)])
@pytest.mark.parametrize("d,stretch", [(3, 8.0), (3, 12.0), (16, 10.0), (80, 10.0)])
@pytest.mark.parametrize("channel", [0, 2 ** -8, 2 ** -26])
def test_gradients_stay_numbers(fmt, f, codes, d, stretch, channel):  # noqa: F811
    """The same further on, where most gradients lie below fp32's normal numbers, with channels of K and V that lose bits: none is NaN or infinite, and
    rows that see nothing but keys without weight get what the 64-bit definition gives, to the largest gradient's 2^-17."""
    import layerdef as L
    rng = np.random.default_rng(d)
    q, k, v, do = inputs(rng, 2, 60, 60, 2, 1, d, grad=1.0)
    q, k = q * np.float32(stretch), k * np.float32(stretch)
    k[..., 1] *= np.float32(channel)
    v[..., 2] *= np.float32(channel)
    t = [fmt.fmt_pack16(torch.from_numpy(x).cuda(), f) if codes else torch.from_numpy(x).cuda() for x in (q, k, v)]
    how = dict(causal=True, window=7, sinks=130, result="f32")
    o, lse = fmt.fmt_attention_fwd(*t, f, **how)
    grads = [x.cpu().numpy() for x in fmt.fmt_attention_bwd(torch.from_numpy(do).cuda(), *t, o, lse, f, **how)]
    vq, vk, vv, vdo = (L.rounded(x, f).astype(np.float64) for x in (q, k, v, do))
    want = [np.zeros(x.shape) for x in (q, k, v)]
    seen = L.visible(60, 60, 60, 0, True, 7, 130)
    for i in range(2):
        for j in range(2):
            r = L.attention(vq[i, :, j], vk[i, :, 0], vv[i, :, 0], seen, d ** -0.5, vdo[i, :, j])
            want[0][i, :, j] = r[2]
            want[1][i, :, 0] += r[3]
            want[2][i, :, 0] += r[4]
    # scores of |q||k| / sqrt(d) have 64 u of that, and P and the gradients as much relatively
    score = 64 * 2.0 ** -24 * float((np.abs(vq).max() * np.abs(vk).max() * d) * d ** -0.5)
    for a, x in zip(grads, want):
        assert np.isfinite(a).all()
        assert np.abs(a - x).max() <= (2.0 ** -17 + 3 * score) * np.abs(x).max() * 4


@pytest.mark.parametrize("f,codes", [(BF16, True), ((8, 4, True), False), ((8, 7, False), False), (SIX, False)])
@pytest.mark.parametrize("n,d,window,sinks", [(600, 1, 40, 5), (600, 3, 7, 1), (700, 3, 200, 130), (500, 16, 30, 0)])
@pytest.mark.parametrize("first", [0, 40])
def test_rows_that_see_late_what_others_see_early(fmt, f, codes, n, d, window, sinks, first):  # noqa: F811
    """Rows of one wave whose first keys lie tiles apart, with a dS of next to nothing in between: the factors of those that have seen nothing yet go
    with the others' and stay where products with them are numbers."""
    rng = np.random.default_rng(n + d)
    q, k, v, do = inputs(rng, 2, n, n, 1, 1, d, grad=1.0)
    k = k * np.exp2(rng.normal(size=(1, n, 1, 1)) * 3).astype(np.float32)
    q, k = q * np.float32(4.0), np.clip(k * np.float32(8.0), -100, 100)
    k[:, ::50] *= np.float32(2.0 ** -28)
    t = [fmt.fmt_pack16(torch.from_numpy(x).cuda(), f) if codes else torch.from_numpy(x).cuda() for x in (q, k, v)]
    how = dict(causal=True, window=window, sinks=sinks, result="f32", q_pos=torch.tensor([first, first + 16], dtype=torch.int32, device="cuda"))
    o, lse = fmt.fmt_attention_fwd(*t, f, **how)
    for x in fmt.fmt_attention_bwd(torch.from_numpy(do).cuda(), *t, o, lse, f, **how):
        assert bool(torch.isfinite(x).all())
