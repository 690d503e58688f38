"""The engine's options at their ends: one selected page."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def engine(**kw):
    from paper_2408_05235_amd.engine import Engine
    g = np.random.default_rng(0)
    return Engine(g.integers(1, 400, 5), g.integers(0, 60, 5), g.integers(3, 40, 5), 16, 400, n_layers=2, n_heads=8,
                  n_kv_heads=2, head_dim=64, **kw)


@pytest.mark.parametrize("select", [1, 2])
def test_few_selected_pages(gpu, select):
    """One page is the last one, which a new token's own key lies in."""
    e = engine(norm=True, select=select)
    e.prefill()
    for _ in range(3):
        assert bool(torch.isfinite(e.step()).all())
    q = torch.randn(5, 8, 64, device="cuda").bfloat16()
    table = e.cache.select(0, q, 1, first=0, last=1)
    last = ((e.cache.length - 1) // 16).clamp(min=-1)
    here = last >= 0
    assert torch.equal(table[here, :, 0], last[here, None].expand(-1, 2))
