"""Layer norm and dropout over more rows than one launch has threads for (2^32)."""
import numpy as np
import pytest

import layerdef as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F = (8, 7, True)


@pytest.fixture(scope="module")
def fmt():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2103_15940_amd as lib
    yield lib
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,cols", [((1 << 28) + 17, 1), ((1 << 28) + 3, 5), ((1 << 26) + 5, 130)])
def test_norm_forward(fmt, rows, cols):
    """The first rows, those around the launch's end, and the last against a call of their own; the mask is that of their place."""
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    edge = (1 << 28 if cols <= 128 else 1 << 26) - 2
    some = [slice(0, 4), slice(edge, edge + 4), slice(rows - 3, rows)]
    for i, at in enumerate(some):
        x[at] = torch.randn(x[at].shape, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda").bfloat16()
    beta = torch.linspace(1.0, 2.0, cols, device="cuda")
    y, z, mean, rstd = fmt.fmt_layernorm_fwd(x, None, beta, F)
    for at in some:
        want = fmt.fmt_layernorm_fwd(x[at].contiguous(), None, beta, F)
        for a, b in ((y, want[0]), (mean, want[2]), (rstd, want[3])):
            assert torch.equal(a[at], b)
    del y, z, mean, rstd
    y, z, _, _ = fmt.fmt_layernorm_fwd(x, None, beta, F, p=0.5, rng=fmt.new_rng(5), site=1)
    at = rows - 3
    blocks = (cols + 7) // 8
    n = np.arange(at * blocks, rows * blocks, dtype=np.uint64)
    full = lambda v: np.full(n.shape, v, dtype=np.uint64)  # noqa: E731
    w = L.philox([n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), full(0), full(1)], [5, 0])
    kept = np.stack([(w[i // 2] >> np.uint64(16 * (i % 2))) & np.uint64(0xFFFF) for i in range(8)], 1).reshape(3, blocks * 8)[:, :cols] >= 32768
    assert np.array_equal(z[at:].float().cpu().numpy(), np.where(kept, 2.0 * x[at:].float().cpu().numpy(), 0.0))


def test_dropout(fmt):
    """2^34 rows of one column: eights of 2^34, of which a launch takes 2^34 less a few."""
    rows = (1 << 34) + 1500
    x = torch.ones(rows, 1, dtype=torch.bfloat16, device="cuda")
    fmt.fmt_dropout(x, 0.5, fmt.new_rng(9, 4), F, site=2, out=x)
    for at in (0, (1 << 34) - 2000, rows - 1000):
        n = np.arange(at, at + 1000, dtype=np.uint64)
        full = lambda v: np.full(n.shape, v, dtype=np.uint64)  # noqa: E731
        w = L.philox([n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), full(4), full(2)], [9, 0])
        assert np.array_equal(x[at:at + 1000, 0].float().cpu().numpy(), np.where((w[0] & np.uint64(0xFFFF)) >= 32768, 2.0, 0.0))
