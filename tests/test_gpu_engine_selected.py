"""The operators as an engine uses them together: norms, 8-bit products,
summaries kept by append, a choice of pages, attention over it, tokens drawn; and the
cache's summaries through forks, refusals and compaction."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def board(n=5, seed=0):
    g = np.random.default_rng(seed)
    return g.integers(1, 400, n), g.integers(0, 60, n), g.integers(3, 40, n)


def engine(pages=400, **kw):
    from paper_2408_05235_amd.engine import Engine
    p, d, r = board()
    return Engine(p, d, r, 16, pages, n_layers=2, n_heads=8, n_kv_heads=2, head_dim=64, **kw)


def test_defaults_are_what_they_were(gpu):
    """Without the new options the same inputs, layers and calls."""
    e, f = engine(), engine()
    x, y = e.prefill(), f.prefill()
    assert torch.equal(x, y) and e.cache.bounds is None and e.embedding is None
    # by hand
    z = e.inputs(5)
    f.inputs(5)
    e.iteration = f.iteration = 1
    for c in (e, f):
        c._extend(torch.ones(5, dtype=torch.int32, device="cuda"))
    want = z
    for layer in range(2):
        qkv = (want @ f.qkv[layer]).view(5, 12, 64)
        f.cache.append(layer, qkv[:, 8:10], qkv[:, 10:])
        want = want + f.cache.attend(layer, qkv[:, :8], max_length=f.max_tokens).view(5, -1) @ f.proj[layer]
    assert torch.equal(e.forward(z), want)


@pytest.mark.parametrize("kw", [dict(norm=True), dict(select=6), dict(vocabulary=3001), dict(quantize=True),
                                dict(norm=True, select=6, vocabulary=3001), dict(quantize=True, select=6, vocabulary=3008)])
def test_iterations(gpu, kw):
    e = engine(**kw)
    if kw.get("vocabulary"):
        f = lambda x: torch.full((5,), x, device="cuda")
        e.sampling = dict(temperature=f(0.8), top_k=torch.full((5,), 50, dtype=torch.int32, device="cuda"), top_p=f(0.9),
                          min_p=f(0.01))
    x = e.prefill()
    seen = []
    for _ in range(20):
        x = e.step()
        assert bool(torch.isfinite(x).all())
        if kw.get("vocabulary"):
            seen.append(e.token.cpu())
            assert bool(((e.token >= 0) & (e.token < kw["vocabulary"])).all())
    if seen:
        assert len(torch.unique(torch.stack(seen))) > 5


def test_choosing_every_page_is_attending_to_all(gpu):
    """As many pages selected as there are: the same hidden states up to the
    order of sums (the outputs of attention differ by a rounding of the 16-bit type, two
    layers' products pass it on)."""
    a, b = engine(norm=True), engine(norm=True, select=64)
    b.qkv, b.proj, b.norms = a.qkv, a.proj, a.norms
    g = torch.Generator(device="cuda").manual_seed(5)
    rows = [torch.randn(n, 512, generator=g, device="cuda").bfloat16() for n in [int(a.tokens.sum())] + [5] * 3]
    at = {}
    for name, e in (("a", a), ("b", b)):
        it = iter(rows)
        e.inputs = lambda n, it=it: next(it)
        at[name] = [e.prefill()] + [e.step() for _ in range(3)]
    assert torch.equal(at["a"][0], at["b"][0])
    for x, y in zip(at["a"][1:], at["b"][1:]):
        assert float((x.double() - y.double()).norm() / x.double().norm()) < 2 * 2.0 ** -8


def test_norms_are_the_formula(gpu):
    """One layer's product by hand, in 64 bits: the norm's output is off by half
    a step of bf16, twice in 8 bits of 2^-4, the product's by half a step of bf16."""
    for quantize in (False, True):
        e = engine(norm=True, quantize=quantize)
        x, r = (torch.randn(7, 512, device="cuda").bfloat16() for _ in range(2))
        got, total = e._product(1, x, e.qkv[1], r)
        h = x.double() + r.double()
        y = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * e.norms[1].double()
        want, size = y @ e.qkv[1].double(), y.abs() @ e.qkv[1].double().abs()
        u = 2 * 2.0 ** -4 + 2.0 ** -8 if quantize else 2.0 ** -8
        # (e4m3 below 2^-6 of its scale's 448: 2^-10 / 448 of the largest value instead)
        extra = 0
        if quantize:
            step = 2.0 ** -10 / 448
            extra = step * (y.abs().amax(1, keepdim=True) * e.qkv[1].double().abs().sum(0)
                            + y.abs().sum(1, keepdim=True) * e.qkv[1].double().abs().amax(0)) * 1.1
        assert bool(((got.double() - want).abs() <= u * size * 1.01 + extra + want.abs() * 2.0 ** -8).all())
        assert bool(((total.double() - h).abs() <= h.abs() * 2.0 ** -8).all())


def cache(**kw):
    from paper_2408_05235_amd import api
    return api.KVCache(2, 64, 3, 16, 64, 6, 200, summaries=True, **kw)


def fill(c, add, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    status = c.extend(torch.tensor(add, dtype=torch.int32, device="cuda"))
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(add)])).cuda()
    T = int(sum(add))
    kv = torch.randn(2, T, 3, 64, generator=g, device="cuda").bfloat16()
    for layer in range(2):
        c.append(layer, kv[0] * (layer + 1), kv[1], off)
    return status


def right(c):
    """Every live page's summary is its keys'."""
    table, length = c.page_table.cpu().numpy(), c.length.cpu().numpy()
    from test_gpu_summaries import summary_of
    for layer in range(2):
        bounds, scale = (x.cpu().numpy() for x in c._summaries(layer))
        keys = c.pages[layer, 0].float().cpu().numpy()
        for b in range(6):
            for j in range(-(-int(length[b]) // 16)):
                p = table[b, j]
                n = min(16, int(length[b]) - 16 * j)
                for h in range(3):
                    want = summary_of(keys[p, h, :n])
                    assert np.array_equal(bounds[p, h], want[0]) and scale[p, h] == want[1], (layer, b, j, h)


def test_summaries_through_a_service(gpu):
    """Appends, forks, frees, a refusal and a compaction."""
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    c = cache()
    fill(c, [40, 0, 100, 17, 0, 0], 1)
    right(c)
    fill(c, [1, 0, 30, 0, 0, 0], 2)
    c.fork(i(2, 0), i(1, 4))
    fill(c, [1, 3, 1, 1, 20, 0], 3)
    right(c)
    c.free(i(0, 2))
    fill(c, [0, 1, 0, 60, 0, 90], 4)
    right(c)
    c.compact()
    right(c)
    status = fill(c, [199, 1, 199, 1, 199, 1], 5)
    assert int((status != 0).sum()) >= 1
    # (a refused slot's pages are left as they are)
    right(c)
    q = torch.randn(6, 6, 64, device="cuda").bfloat16()
    for layer in range(2):
        pages = c.select(layer, q, 4, last=2)
        out = c.attend_pages(layer, q, pages)
        assert bool(torch.isfinite(out).all())
        refused = status.cpu() != 0
        assert bool((pages.cpu()[refused] == -1).all()) and bool((out.cpu()[refused] == 0).all())
    with pytest.raises(ValueError, match="summaries"):
        from paper_2408_05235_amd import api
        api.KVCache(1, 4, 1, 16, 64, 1, 16).select(0, q[:1, :1], 1)


def test_a_step_in_a_graph(gpu):
    """An iteration's calls captured together and replayed, with eager work
    between, each replay equal to the eager result; two graphs of the same state."""
    from paper_2408_05235_amd import api
    c = cache()
    fill(c, [40, 90, 100, 17, 150, 3], 7)
    c.extend(torch.ones(6, dtype=torch.int32, device="cuda"))
    x, r = (torch.randn(6, 192, device="cuda").bfloat16() for _ in range(2))
    w, u = torch.ones(192, device="cuda").bfloat16(), torch.rand(6, device="cuda")
    head = torch.randn(192, 1000, device="cuda").bfloat16()

    def iteration():
        y, h = api.tl_norm(x, w, residual=r)
        kv = y.view(6, 3, 64)
        c.append(0, kv, kv)
        out = c.attend_pages(0, kv, c.select(0, kv, 3))
        q, s, h = api.tl_norm(out.view(6, 192), w, residual=h, group=64)
        return y, out, q, s, h, api.tl_sample(h @ head, u, top_p=u)

    iteration()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = iteration()
        graphs.append((g, res))
    for k in range(4):
        x.normal_(0, 1)
        r.normal_(0, 1)
        u.uniform_(0, 1)
        g, res = graphs[k % 2]
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in res]
        want = iteration()
        for a, b in zip(got, want):
            assert torch.equal(a.view(torch.uint8) if a.dtype == torch.float8_e4m3fn else a,
                               b.view(torch.uint8) if b.dtype == torch.float8_e4m3fn else b)


def test_command(gpu, capsys):
    from paper_2408_05235_amd import engine as module
    module.main(["--iterations", "12", "--layers", "2", "--norm", "--select", "8", "--vocabulary", "2000"])
    assert "iterations/s" in capsys.readouterr().out
    with pytest.raises(ValueError, match="window"):
        engine(select=4, window=64)
