"""The engine's products in 8 bits, in either of its types."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def engine(**kw):
    from paper_2408_05235_amd.engine import Engine
    g = np.random.default_rng(0)
    return Engine(g.integers(1, 400, 5), g.integers(0, 60, 5), g.integers(3, 40, 5), 16, 400, n_layers=2, n_heads=8,
                  n_kv_heads=2, head_dim=64, **kw)


@pytest.mark.parametrize("rows", [1, 7, 64])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_products_in_eight_bits(gpu, dtype, rows):
    """The product of what the norm and the weight hold in 8 bits, against 64 bits: sums in
    fp32 (a rounding a term at most, 2^-24 of the terms' sizes, and four for the scales), then
    half a step of the engine's type (finfo.eps / 2 of the value, 2^-25 at least in f16)."""
    from paper_2408_05235_amd import api
    e = engine(quantize=True, vocabulary=3008, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(rows)
    randn = lambda: torch.randn(rows, 512, generator=g, device="cuda").to(dtype)
    for at, weight in ((0, e.qkv[0]), (2, e.head)):
        for residual in (None, randn()):
            x = randn()
            got, _ = e._product(at, x, weight, residual)
            assert got.dtype == dtype and got.shape == (rows, weight.shape[1])
            q, scale = api.tl_norm(x, e.norms[at], residual=residual, group=0)[:2]
            w, columns = e.quantize[at]
            a, b = q.double() * scale.double()[:, None], w.double() * columns.double()
            want, size = a @ b, a.abs() @ b.abs()
            off = (got.double() - want).abs()
            assert bool((off <= want.abs() * torch.finfo(dtype).eps / 2 + size * (512 + 4) * 2.0 ** -24 + 2.0 ** -25).all())
