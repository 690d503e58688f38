"""The norm's output in 8 bits (tl_norm) is the quotient by the scale, rounded once: bit for
bit, where the norm itself is exact (rows of 1 and -1 without eps, whose root is 1, so that
y is the weight)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# borders between neighbouring values of e4m3, in units of their own: 17 .. 31 (normal, odd:
# half a step of 4 bits) and the odd halves below the least normal one
BORDERS = [b * 2.0 ** e for b in range(17, 32, 2) for e in (-9, -5, 0, 3)] + [b * 2.0 ** -10 for b in range(1, 16, 2)]


def borders(dtype, cols, group, seed):
    """A weight whose quotients lie on borders, of scales m / 64 for odd m (the largest of
    each scale is 448 of them)."""
    g = np.random.default_rng(seed)
    most = {"bf16": 8, "f16": 64, "f32": 1 << 15}[dtype]        # (so that border x m fits the type)
    per = group or cols
    w = np.zeros(cols, np.float32)
    for at in range(0, cols, per):
        n = min(per, cols - at)
        m = 2 * g.integers(1, most // 2) + 1
        unit = np.float32(m / 64)
        w[at: at + n] = g.choice(BORDERS, n) * g.choice([-1, 1], n) * unit
        w[at + g.integers(n)] = 448 * unit
    return w


def expected(w, group):
    per, cols = group or len(w), len(w)
    n = -(-cols // per)
    padded = np.zeros(n * per, np.float32)
    padded[:cols] = w
    s = np.maximum(np.abs(padded.reshape(n, per)).max(1) / np.float32(448), np.float32(2.0 ** -100))
    q = w / np.repeat(s, per)[:cols]
    assert q.dtype == np.float32
    return torch.from_numpy(q).to(torch.float8_e4m3fn).float(), torch.from_numpy(s)


def compare(w, dtype, group):
    from paper_2408_05235_amd import api
    dt = DTYPES[dtype]
    weight = torch.from_numpy(w).to(dt)
    w = weight.float().numpy()
    sign = torch.ones(2, len(w))
    sign[1, ::2] = -1
    for residual in (False, True):
        x = sign.to(dt).cuda()
        kw = dict(residual=torch.zeros_like(x)) if residual else {}
        q, scale = api.tl_norm(x, weight.cuda(), 0.0, group=group, **kw)[:2]
        want, s = expected(w, group)
        assert torch.equal(scale.cpu(), (s if group else s.view(1)).expand(2, -1).reshape(scale.shape))
        assert torch.equal(q.float().cpu() * sign, want.expand(2, -1))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("cols", [64, 1000, 4096, 5000, 8192, 16384, 32768, 40000])
@pytest.mark.parametrize("group", [0, 16, 128])
def test_borders(gpu, cols, dtype, group):
    print(f"norm borders {cols} {dtype} group {group}", flush=True)
    for seed in range(4):
        compare(borders(dtype, cols, group, seed), dtype, group)


@pytest.mark.parametrize("cols", [8000, 1 << 20])
@pytest.mark.parametrize("size", [1.0, 1e-28, 1e-38, 1e36])
def test_any_weight(gpu, cols, size):
    """Normal values, of the least and the largest sizes too (scales at their least,
    values that are no normal numbers)."""
    w = (np.random.default_rng(cols).normal(0, 1, cols) * size).astype(np.float32)
    for group in (0, 32):
        compare(w, "f32", group)


@pytest.mark.parametrize("cols", [64, 40000])
def test_an_infinite_scale(gpu, cols):
    """y beyond fp32: the scale is infinite, a finite y is 0 of it, an infinite one NaN."""
    from paper_2408_05235_amd import api
    x = torch.ones(1, cols, device="cuda")
    x[0, ::2] = 3
    w = torch.ones(cols, device="cuda")
    w[6] = 3e38
    for group in (0, 16):
        q, scale = api.tl_norm(x, w, 0.0, group=group)
        q = q.float().cpu()[0]
        here = slice(0, group or cols)
        assert float(scale.flatten()[0]) == float("inf")
        assert bool(torch.isnan(q[6])) and bool((q[here][torch.arange(q[here].numel()) != 6] == 0).all())
        assert bool(torch.isfinite(q[16:]).all())
