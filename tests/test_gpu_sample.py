"""The next tokens (tl_sample) against whole-number weights made on the host."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
UNIT = 2.0 ** 40


def kept_of(x, T, k, p, q):
    """(kept tokens in index order, their weights, exponents, largest) of one row of float32
    logits, and whether a threshold lies so near a sum that the exponential's last bit
    could move it: it may be off by some units of 2^-53, so a weight by one, a sum by
    as many as it has tokens."""
    x = np.where(np.isnan(x), -np.inf, x).astype(np.float64)
    m = x.max()
    with np.errstate(invalid="ignore"):
        e = np.where(x == m, 0.0, np.where((x == -np.inf) | (m == np.inf), -np.inf, (x - m) / np.float64(T)))
    w = np.rint(np.exp(e) * UNIT).astype(np.int64)
    order = np.lexsort((np.arange(len(x)), -x))
    near = False
    if k > 0:
        order = order[:k]
    if p < 1:
        sums = np.cumsum(w[order])
        need = max(int(np.ceil(np.float64(p) * np.float64(sums[-1]))), 1)
        n = int(np.searchsorted(sums, need)) + 1
        edge = sums[max(n - 2, 0): n]
        near = need > 1 and bool((np.abs(edge - need) <= 2 * len(x)).any())
        order = order[:n]
    if q > 0:
        least = int(np.ceil(min(np.float64(q), 1.0) * UNIT))
        near |= bool((np.abs(w[order] - least) <= 2).any() and q < 1)
        order = order[w[order] >= least]
    order = np.sort(order)
    return order, w[order], e, near


def draw(seed, rows, V, dtype, filters, spread=2.0):
    g = np.random.default_rng(seed)
    x = torch.from_numpy(g.normal(0, spread, (rows, V)).astype(np.float32)).to(DTYPES[dtype])
    T = (0.2 + g.random(rows) * 1.5).astype(np.float32)
    k = np.where(g.random(rows) < 0.4, 0, np.exp(g.random(rows) * np.log(V + 1.0))).astype(np.int32)
    p = np.where(g.random(rows) < 0.3, 1.0, g.random(rows)).astype(np.float32)
    q = np.where(g.random(rows) < 0.5, 0.0, 0.3 * g.random(rows)).astype(np.float32)
    if not filters:
        k[:], p[:], q[:] = 0, 1, 0
    return x, T, k, p, q, g


def expect(x, T, k, p, q, g):
    """Numbers u that lie well inside a token's share, and what they give."""
    u, token, logprob = [], [], []
    for b in range(x.shape[0]):
        order, w, e, near = kept_of(x[b].float().numpy(), T[b], int(k[b]), p[b], q[b])
        while near:                         # (a setting on a border: the next one)
            p[b] = np.nextafter(p[b], np.float32(0)) if p[b] < 1 else p[b]
            q[b] = np.float32(q[b] * 0.99)
            order, w, e, near = kept_of(x[b].float().numpy(), T[b], int(k[b]), p[b], q[b])
        sums = np.cumsum(w)
        for _ in range(1000):
            v = np.float32(g.random())
            r = min(int(np.floor(np.float64(v) * np.float64(sums[-1]))), int(sums[-1]) - 1)
            i = int(np.searchsorted(sums, r, side="right"))
            if r - (sums[i - 1] if i else -10 ** 9) > 4 * len(w) + 64 and sums[i] - r > 4 * len(w) + 64:
                break
        else:
            raise AssertionError("no number lies inside a share")
        u.append(v)
        token.append(order[i])
        logprob.append(e[order[i]] - math.log(sums[-1] / UNIT))
    return np.array(u, np.float32), np.array(token), np.array(logprob)


def run(x, u, T, k, p, q, **kw):
    from paper_2408_05235_amd import api
    c = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return api.tl_sample(x.cuda() if not x.is_cuda else x, c(u), c(T), c(k), c(p), c(q), want_logprob=True, **kw)


def check(x, T, k, p, q, g):
    u, token, logprob = expect(x, T, k, p, q, g)
    t, lp = run(x, u, T, k, p, q)
    assert np.array_equal(t.cpu().numpy(), token)
    # the 64-bit value rounded to 32 (2^-24 of it); sums off by a unit a token (2^-40 of
    # the largest weight, which is at most the sum), and the exponent and logarithm
    off = np.abs(lp.cpu().numpy() - logprob)
    assert bool((off <= np.abs(logprob) * 2.0 ** -24 + x.shape[1] * 2.0 ** -40 + 2.0 ** -40).all()), off.max()


@pytest.mark.parametrize("filters", [False, True])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,V", [(3, 1), (5, 2), (9, 63), (8, 64), (7, 1000), (5, 1025), (4, 8191), (6, 32000),
                                    (3, 50257), (3, 70001), (2, 128000), (2, 262144)])
def test_sizes(gpu, rows, V, dtype, filters):
    print(f"sample {rows} x {V} {dtype} filters {filters}", flush=True)
    check(*draw(rows * V, rows, V, dtype, filters))


@pytest.mark.parametrize("V", [300, 20000, 150000])
def test_ties(gpu, V):
    """Logits of few values: a threshold falls among equal ones, of which the
    lower indices are taken."""
    for seed in range(4):
        x, T, k, p, q, g = draw(seed, 12, V, "bf16", True)
        x = (x.float() * 0.7).round().to(torch.bfloat16)
        if seed == 3:
            x[:] = 1.5          # all equal
        check(x, T, k, p, q, g)


@pytest.mark.parametrize("V", [40, 33000])
def test_edges(gpu, V):
    """Settings at their ends, a row that is mostly or wholly forbidden, and u
    outside [0, 1)."""
    x, T, k, p, q, g = draw(3, 24, V, "f32", False)
    T[0], T[1], T[2], T[3] = 0, -1, math.nan, math.inf
    k[4], k[5], k[6], k[7] = 1, V, V + 5, -3
    p[8], p[9], p[10], p[11] = 0, -1, 1, math.nan
    q[12], q[13], q[14], q[15] = 1, 7, -1, math.nan
    x[16] = -math.inf
    x[16, 7] = -3.0
    x[17, ::2] = math.nan
    x[18] = torch.finfo(torch.float32).min
    x[18, 5:9] = 0
    x[19, 3] = x[19, 11] = math.inf
    x[20, :] = torch.finfo(torch.float32).max
    x[21] *= 1e30
    T[22] = 1e-30
    T[23] = 1e30
    fix = lambda a, d: np.where(np.isnan(a), d, a).astype(np.float32)
    best = ~(T > 0)
    T2, k2 = np.where(best, 1, T).astype(np.float32), np.where(best, 1, k).astype(np.int32)
    u, token, logprob = expect(x, T2, k2, fix(p, 1), fix(q, 0), g)
    t, lp = run(x, u, T, k, p, q)
    assert np.array_equal(t.cpu().numpy(), token)
    assert np.allclose(lp.cpu().numpy(), logprob, rtol=2.0 ** -23, atol=V * 2.0 ** -40 + 2.0 ** -40)
    assert token[0] == int(x[0].argmax()) and lp[0] == 0
    # u at its ends and beyond
    kept = [kept_of(x[b].numpy(), T2[b], int(k2[b]), fix(p, 1)[b], fix(q, 0)[b]) for b in range(24)]
    low = np.array([o[np.flatnonzero(w > 0)[0]] for o, w, _, _ in kept])
    high = np.array([o[np.flatnonzero(w > 0)[-1]] for o, w, _, _ in kept])
    for v, want in ((0.0, low), (-1.0, low), (math.nan, low), (1.0, high), (5.0, high)):
        t, _ = run(x, np.full(24, v, np.float32), T, k, p, q)
        assert np.array_equal(t.cpu().numpy(), want), v
    # nothing to take
    x[2] = -math.inf
    x[9] = math.nan
    t, lp = run(x, u, T, k, p, q)
    for b in (2, 9):
        assert int(t[b]) == -1 and float(lp[b]) == -math.inf
    keep = [b for b in range(24) if b not in (2, 9)]
    assert np.array_equal(t.cpu().numpy()[keep], token[keep])


@pytest.mark.parametrize("spread", [0.02, 0.3, 1.5, 6.0])
def test_thresholds_among_many(gpu, spread):
    """Flat rows and steep ones, with a top-p near 1, and a logit far above the first
    ones of its row: thresholds where many tokens lie, or where the bins end."""
    V = 131072
    x, T, k, p, q, g = draw(21, 12, V, "f32", False, spread)
    p[:] = [0.5, 0.9, 0.99, 0.999, 0.9999, 0.3, 0.97, 0.95, 0.6, 0.99, 0.999, 0.2]
    k[8:10] = 40000, 100000
    q[10] = 1e-4
    T[:] = np.linspace(0.25, 1.6, 12)
    x[5, 100000] = 40.0
    x[6, 70000:70009] = 25.0
    check(x, T, k, p, q, g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_most_columns(gpu, dtype):
    V = 1 << 22
    x, T, k, p, q, g = draw(5, 2, V, dtype, False, 0.5)
    p[0], k[1] = 0.9, 1000000
    T[:] = 0.7
    check(x, T, k, p, q, g)


def test_defaults_strides_and_rows(gpu):
    from paper_2408_05235_amd import api
    x, T, k, p, q, g = draw(8, 700, 501, "bf16", False)
    T[:] = 1
    u, token, _ = expect(x, T, k, p, q, g)
    wide = torch.zeros(1400, 510, dtype=torch.bfloat16)
    wide[::2, 4:505] = x
    for at in (4, 3):           # rows that begin at any element
        wide[::2, at:at + 501] = x
        got = api.tl_sample(wide.cuda()[::2, at:at + 501], torch.from_numpy(u).cuda())
        assert np.array_equal(got.cpu().numpy(), token)
    assert api.tl_sample(x[:0].cuda(), torch.zeros(0, device="cuda")).shape == (0,)
    # one row, many numbers: as often as it weighs
    row = x[:1].expand(4000, -1).cuda()
    u = (np.arange(4000, dtype=np.float32) + 0.5) / 4000
    t = api.tl_sample(row, torch.from_numpy(u).cuda()).cpu().numpy()
    share = torch.softmax(x[0].double(), 0).numpy()
    assert bool((np.diff(t) >= 0).all())        # (the running sum is in index order)
    assert bool((np.abs(np.bincount(t, minlength=501) - 4000 * share) <= 1 + 1e-3).all())


def test_replays_and_streams(gpu):
    x, T, k, p, q, g = draw(11, 16, 32000, "f32", True)
    u, token, _ = expect(x, T, k, p, q, g)
    from paper_2408_05235_amd import api
    c = [torch.from_numpy(a).cuda() for a in (u, T, k, p, q)]
    xg = x.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = api.tl_sample(xg, *c)
    torch.cuda.current_stream().wait_stream(side)
    assert np.array_equal(got.cpu().numpy(), token)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = api.tl_sample(xg, *c)
    for seed in (1, 2, 3):
        x2 = draw(seed, 16, 32000, "f32", True)[0].cuda()
        xg.copy_(x2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, api.tl_sample(xg, *c))
