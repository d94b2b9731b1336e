"""Attention with a dimension of size zero, over every mask: outputs that exist are zero, and every call returns."""
import itertools

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,nq,nk,h,hk", [(2, 3, 5, 0, 2), (2, 0, 5, 4, 2), (2, 3, 0, 4, 2), (0, 3, 5, 4, 2), (2, 0, 0, 4, 2), (2, 0, 5, 0, 1),
                                          (1, 300, 700, 0, 1), (1, 0, 700, 2, 2)])
@pytest.mark.parametrize("f", [(6, 9, True), (7, 15, True)])
def test_nothing_to_attend(b, nq, nk, h, hk, f):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2103_15940_amd as fmt
    t = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    q, k, v, g = t(b, nq, h, 8), t(b, nk, hk, 8), t(b, nk, hk, 8), t(b, nq, h, 8)
    for causal, window, sinks in itertools.product((False, True), (0, 1, 9), (0, 1, 200)):
        how = dict(causal=causal, window=window, sinks=sinks)
        o, lse = fmt.fmt_attention_fwd(q, k, v, f, **how)
        assert o.shape == q.shape and lse.shape == (b, h, nq) and bool((o == 0).all()) and bool((lse == -float("inf")).all())
        grads = fmt.fmt_attention_bwd(g, q, k, v, o, lse, f, **how)
        for x, like in zip(grads, (q, k, v)):
            assert x.shape == like.shape and bool((x == 0).all())
    torch.cuda.synchronize()
