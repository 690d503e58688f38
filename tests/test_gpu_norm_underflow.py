"""The norm (tl_norm) without eps of rows whose squares are below fp32's least number: every
value is its weight's sign times infinity, and so are the scales, whatever lies behind the
row's end."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [1, 5, 64, 100, 520, 1030, 5001, 8200, 40003])
def test_squares_that_underflow(gpu, cols, dtype):
    from paper_2408_05235_amd import api
    x = torch.full((3, cols), 1e-30, device="cuda").to(dtype)
    x[1] = 1
    w = torch.ones(cols, device="cuda", dtype=dtype)
    w[0] = -2
    for residual in (None, torch.zeros_like(x)):
        first = lambda r: r[0] if isinstance(r, tuple) else r
        y = first(api.tl_norm(x, w, 0.0, residual)).float().cpu()
        want = torch.full((3, cols), float("inf"))
        want[1] = 1
        want[:, 0] *= -1
        want[1, 0] = -2
        assert torch.equal(y, want)
        for group in (0, 16, 512):
            q, scale = api.tl_norm(x, w, 0.0, residual, group)[:2]
            scale = scale.cpu().view(3, -1)
            assert bool((scale[[0, 2]] == float("inf")).all()), (group, scale[0])
            assert bool(torch.isfinite(scale[1]).all())
            q = q.float().cpu()
            assert bool(torch.isnan(q[[0, 2]]).all()) and bool(torch.isfinite(q[1]).all())
