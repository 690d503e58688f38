"""What the engine refuses when it is made (no GPU: before anything is allocated)."""
import pytest
import torch

from paper_2408_05235_amd.engine import Engine


@pytest.mark.parametrize("kw,needle", [
    (dict(select=-1), "select -1"), (dict(select=4097), "select 4097"), (dict(select=4, window=64), "window"),
    (dict(select=4, n_heads=129, n_kv_heads=1), "129 query heads"),
    (dict(quantize=True, vocabulary=3001), "vocabulary of 3001"), (dict(quantize=True, n_heads=3, n_kv_heads=3, head_dim=8), "width of 24"),
    (dict(quantize=True, n_heads=2, n_kv_heads=1, head_dim=24, dtype=torch.float16, vocabulary=8), "vocabulary of 8"),
    (dict(vocabulary=-5), "vocabulary -5"), (dict(vocabulary=(1 << 22) + 1), "vocabulary"),
])
def test_refused(kw, needle):
    with pytest.raises(ValueError, match=needle):
        Engine([5, 9], [0, 0], [3, 3], 16, 40, device="cpu", **kw)
