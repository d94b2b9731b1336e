"""Attention over more workgroups than one launch has threads for (2^32), and more operands than one call's scratch holds: the last sequences are
what a call of their own gives."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F = (8, 7, True)


@pytest.fixture(scope="module")
def fmt():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2103_15940_amd as lib
    yield lib
    lib.fmt_release_scratch()
    torch.cuda.empty_cache()


def tensors(b, n, h, d, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.zeros(b, n, h, d, dtype=torch.bfloat16, device="cuda")
    for at in (slice(0, 3), slice(b // 2 - 2, b // 2 + 2), slice(b - 3, b)):
        t[at] = torch.randn(t[at].shape, generator=g, device="cuda").bfloat16()
    return t


@pytest.mark.parametrize("nq,nk", [(1, 2), (9, 2)])
def test_forward(fmt, nq, nk):
    b, h, d = 65535, 257, 2
    q, k, v = (tensors(b, n, h, d, i) for i, n in enumerate((nq, nk, nk)))
    lens = torch.full((b,), nk, dtype=torch.int32, device="cuda")
    lens[-1] = 1
    o, lse = fmt.fmt_attention_fwd(q, k, v, F, k_lens=lens)
    for at in (slice(0, 3), slice(b // 2 - 2, b // 2 + 2), slice(b - 3, b)):
        want, wl = fmt.fmt_attention_fwd(*(t[at].contiguous() for t in (q, k, v)), F, k_lens=lens[at].contiguous())
        assert torch.equal(o[at], want) and torch.equal(lse[at], wl)


def test_backward(fmt):
    b, h, d = 65535, 33, 4
    q, k, v, g = (tensors(b, 3, h, d, i) for i in range(4))
    pos = torch.zeros(b, dtype=torch.int32, device="cuda")
    pos[-1] = 1
    how = dict(causal=True, q_pos=pos)
    o, lse = fmt.fmt_attention_fwd(q, k, v, F, **how)
    grads = fmt.fmt_attention_bwd(g, q, k, v, o, lse, F, **how)
    for at in (slice(0, 3), slice(b // 2 - 2, b // 2 + 2), slice(b - 3, b)):
        part = [t[at].contiguous() for t in (g, q, k, v, o, lse)]
        for x, y in zip(grads, fmt.fmt_attention_bwd(*part, F, causal=True, q_pos=pos[at].contiguous())):
            assert torch.equal(x[at], y)
