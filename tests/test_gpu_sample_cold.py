"""The next tokens (tl_sample) at temperatures so low, or logits so large, that a bin of
logits is less than a step of them: what ties at the largest is all that weighs, and top-k
still takes the first of these."""
import numpy as np
import pytest
import torch

from test_gpu_sample import DTYPES, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("temperature", [1e-4, 1e-7, 1e-8, 1e-9, 1e-12, 1e-20, 1e-30, 1e-38])
def test_ties_at_the_largest(gpu, temperature, dtype):
    print(f"sample cold {temperature} {dtype}", flush=True)
    V = 8200
    g = np.random.default_rng(17)
    tops = np.arange(5.0, 61.0, 1.25)
    rows = len(tops)
    x = np.minimum(g.normal(0, 2, (rows, V)), 4).astype(np.float32)
    for b, top in enumerate(tops):
        x[b, g.choice(V, 20, replace=False)] = top
    x[::7] *= -1        # (largest where no tie was put)
    T = np.full(rows, temperature, np.float32)
    k = np.array([1, 5, 19, 20, 21, 100, 0] * rows, np.int32)[:rows]
    for p in (1.0, 0.3, 0.9):
        check(torch.from_numpy(x).to(DTYPES[dtype]), T, k, np.full(rows, p, np.float32), np.zeros(rows, np.float32), g)


@pytest.mark.parametrize("scale", [3e4, 1e10, 1e30, 1e38])
def test_large_logits(gpu, scale):
    """Logits of a size, and temperatures from far below their steps to their size."""
    V = 8200
    g = np.random.default_rng(3)
    rows = 24
    x = (scale * (1 + 0.5 * np.tanh(g.normal(0, 1, (rows, V))))).astype(np.float32)
    x[:, ::3] *= -1
    for b in range(rows):
        x[b, g.choice(V, 9, replace=False)] = 1.75 * scale
    T = (scale * 10.0 ** np.linspace(-12, 0.3, rows)).astype(np.float32)
    k = np.array([0, 3, 8, 9, 10, 500] * 4, np.int32)
    for p in (1.0, 0.6, 0.95):
        check(torch.from_numpy(x), T, k, np.full(rows, p, np.float32), np.zeros(rows, np.float32), g)
