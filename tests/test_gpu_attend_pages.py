"""Attention over selected pages (tl_attend_pages) against 64 bits, with the
bound on its error that tl_attend's tests use (the arithmetic is the same)."""
import math

import numpy as np
import pytest
import torch

import cache_cases

pytestmark = pytest.mark.gpu


def lists(seed, c, K, kind="alike"):
    """[T, G, K] lists of the pages up to each token's; ``alike``: neighbours share
    most; ``any``: none of it, with repetitions, in no order, and entries that are no
    page."""
    g = np.random.default_rng(seed)
    G, N = c["k"].shape[1], c["page"]
    out = []
    for a, n in zip(c["before"].tolist(), c["new"].tolist()):
        base = g.random((G, (a + n) // N + 2))
        for p in range(a, a + n):
            for h in range(G):
                m = p // N + 1
                x = base[h, :m] + 0.4 * g.random(m)
                x[-1] = 9
                s = np.sort(np.argsort(-x)[:K])
                row = np.full(K, -1, np.int64)
                row[:len(s)] = s
                if kind == "any":
                    row = g.integers(-2, m + 2, K)
                    row[g.random(K) < 0.05] = 2 ** 31 - 1
                    row[g.random(K) < 0.05] = -2 ** 31
                out.append(row)
    return torch.from_numpy(np.array(out, np.int32).reshape(-1, G, K))


def exact(c, sel, scale=None):
    """cache_cases.exact for each KV head by itself, tokens seen by its lists."""
    G = c["k"].shape[1]
    per = c["q"].shape[1] // G
    first = np.concatenate([[0], np.cumsum(c["new"])])
    parts = []
    for h in range(G):
        one = dict(c, q=c["q"][:, h * per:(h + 1) * per], dense=[(k[:, h:h + 1], v[:, h:h + 1]) for k, v in c["dense"]])

        def see(b, p, t):
            vis = torch.zeros(p.shape[0], t.shape[1], dtype=torch.bool, device=p.device)
            for i in range(p.shape[0]):
                pages = sel[first[b] + i, h].long()
                pages = pages[(pages >= 0) & (pages < c["table"].shape[1])].to(p.device)
                vis[i] = torch.isin(t[0] // c["page"], pages)
            return vis & (t <= p)

        parts.append(cache_cases.exact(one, scale, see))
    return [torch.cat(x, 1) for x in zip(*parts)]


def run(c, sel, **kw):
    from paper_2408_05235_amd import api
    return api.tl_attend_pages(c["q"], c["k"], c["v"], c["table"], c["length"], sel.cuda(), c["offset"], want_lse=True, **kw)


def check(c, sel, scale=None, **kw):
    got, lse = run(c, sel, scale=scale, **kw)
    out, ref_lse, tol, tol_lse = exact(c, sel, scale)
    assert bool(torch.isfinite(got).all())
    off = (got.double() - out).abs()
    assert bool((off <= tol).all()), f"{float((off / (tol + 1e-300)).max()):.2f} times the bound"
    none = ref_lse == -math.inf
    assert torch.equal(lse == -math.inf, none) and bool((got[none] == 0).all())
    assert bool(((lse.double() - ref_lse).abs()[~none] <= tol_lse[~none]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kv,dim,page,order", [
    (4, 2, 64, 16, "head"), (8, 1, 128, 24, "token"), (5, 5, 80, 7, "head"), (20, 1, 128, 16, "token"),
    (6, 2, 256, 16, "head"), (15, 3, 8, 5, "head"), (32, 2, 128, 1, "token"), (71, 1, 64, 64, "head")])
def test_heads(gpu, heads, kv, dim, page, order, dtype):
    print(f"attend_pages heads {heads} on {kv} of {dim}, pages of {page} {order} {dtype}", flush=True)
    for kind in ("alike", "any"):
        c = cache_cases.make(1, dtype, heads, kv, dim, page, [0, 1, 15, 100, 700], [1] * 5, order=order, offsets=False)
        check(c, lists(1, c, 9, kind))
        c = cache_cases.make(2, dtype, heads, kv, dim, page, [0, 40, 0, 311], [1, 9, 0, 30], order=order)
        check(c, lists(2, c, 6, kind))


@pytest.mark.parametrize("K", [1, 2, 17, 64, 129, 500, 4096])
def test_lengths_of_lists(gpu, K):
    print(f"attend_pages {K} pages", flush=True)
    for kind in ("alike", "any"):
        c = cache_cases.make(3, "bf16", 8, 2, 64, 4, [5000, 3, 1200], [1] * 3, offsets=False)
        check(c, lists(3, c, K, kind))
        c = cache_cases.make(4, "f16", 8, 2, 64, 4, [1500, 0], [17, 25])
        check(c, lists(4, c, K, kind))


def test_workspaces(gpu):
    """In one part and in several: equal up to rounding, each the same again."""
    c = cache_cases.make(5, "bf16", 8, 2, 128, 16, [9000], [1], offsets=False)
    sel = lists(5, c, 256)
    full = run(c, sel)
    for n in (0, 100, 40000, 1 << 22):
        w = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
        check(c, sel, workspace=w)
        a, b = run(c, sel, workspace=w), run(c, sel, workspace=w)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert torch.equal(run(c, sel)[0], full[0])


def test_long_tables_in_windows(gpu):
    """Pages of one token: a table with more of them than the lists' bits hold
    at once (131072 pages)."""
    c = cache_cases.make(6, "bf16", 2, 1, 8, 1, [300000], [1], offsets=False, poison=False)
    sel = lists(6, c, 3000)
    check(c, sel)
    c = cache_cases.make(7, "f16", 2, 1, 8, 1, [70000], [9], poison=False)
    check(c, lists(7, c, 300))


def test_what_no_list_names_is_not_used(gpu):
    """NaN in every page that no list names, and in the first KV head's pages of
    the second's lists."""
    c = cache_cases.make(8, "bf16", 8, 2, 64, 16, [600, 90, 2000], [3, 1, 20])
    sel = lists(8, c, 10)
    used = torch.zeros(c["k"].shape[0], 2, dtype=torch.bool)
    table, first = c["table"].cpu().long(), np.concatenate([[0], np.cumsum(c["new"])])
    for b in range(3):
        for i in range(first[b], first[b + 1]):
            for h in range(2):
                s = sel[i, h].long()
                used[table[b, s[s >= 0]], h] = True
    for x in (c["k"], c["v"]):
        x.masked_fill_(~used.cuda()[:, :, None, None], math.nan)
    check(c, sel)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_infinities_of_another_token(gpu, dtype):
    """Values that are not finite in a page that only some tokens of a chunk
    name reach those and no others."""
    c = cache_cases.make(9, dtype, 8, 2, 128, 16, [400], [12])
    sel = lists(9, c, 6)
    sel[:, :, 0], sel[:, :, 1:5] = 25, torch.arange(1, 5, dtype=torch.int32)     # (the last page)
    sel[:, :, 5] = -1
    sel[3, 0, 5], sel[7, 1, 5] = 7, 9
    table = c["table"].cpu().long()
    want = exact(c, sel)
    kb, vb = c["dense"][0]
    for page, h, x in ((7, 0, math.inf), (9, 1, math.nan)):
        c["v"][table[0, page], h, 5, 2] = x
        vb[page * 16 + 5, h, 2] = x         # (exact takes 0 for it, as nobody else sees it)
    got, lse = run(c, sel)
    out, ref_lse, tol, _ = exact(c, sel)
    assert bool((got[3, :4, 2] == math.inf).all()) and bool(torch.isnan(got[7, 4:, 2]).all())
    rest = torch.ones_like(got, dtype=torch.bool)
    rest[3, :4, 2] = rest[7, 4:, 2] = False
    assert bool(torch.isfinite(got[rest]).all())
    assert bool(((got.double() - out).abs() <= tol)[rest].all())
    assert bool((lse.double() - want[1]).abs().max() < 1e-3)


def test_rows_of_no_sequence_and_refused_ones(gpu):
    from paper_2408_05235_amd import api
    c = cache_cases.make(10, "bf16", 4, 2, 64, 16, [50, 33, 80], [3, 2, 4])
    sel = lists(10, c, 3)
    want, want_lse = run(c, sel)
    pad = lambda x: torch.cat([x[:2] * 0 + 1, x, x[:5] * 0 + 1]).contiguous()
    out = torch.full((16, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    q, s = pad(c["q"].contiguous())[:16], pad(sel)[:16].cuda()
    got = api.tl_attend_pages(q, c["k"], c["v"], c["table"], c["length"], s, c["offset"] + 2, out=out)
    assert torch.equal(got[2:11], want) and bool((got[:2] == 7).all()) and bool((got[11:] == 7).all())
    granted = torch.tensor([3, -1 - 1, 4, 1], dtype=torch.int32, device="cuda")
    got, lse = run(c, sel, granted=granted)
    assert torch.equal(got[:3], want[:3]) and torch.equal(got[5:], want[5:]) and bool((got[3:5] == 0).all())
    assert bool((lse[3:5] == -math.inf).all())
    # nothing in the cache
    none = api.tl_attend_pages(c["q"], c["k"][:0], c["v"][:0], c["table"], c["length"], sel.cuda(), c["offset"])
    assert bool((none == 0).all())


def test_all_pages_are_plain_attention(gpu):
    """Lists of every page give what tl_attend gives."""
    from paper_2408_05235_amd import api
    c = cache_cases.make(11, "f16", 8, 2, 128, 16, [900, 20], [5, 30])
    sel = torch.arange(64, dtype=torch.int32).expand(35, 2, 64).contiguous()
    check(c, sel)
    got, lse = run(c, sel)
    out, tol = exact(c, sel)[0], exact(c, sel)[2]
    both = api.tl_attend(c["q"], c["k"], c["v"], c["table"], c["length"], c["offset"])
    assert bool(((got.double() - both.double()).abs() <= 2 * tol).all())
    del out, lse


def test_streams_and_replays(gpu):
    from paper_2408_05235_amd import api
    c = cache_cases.make(12, "bf16", 8, 1, 128, 16, [9000, 100], [1, 1], offsets=False, poison=False)
    sel = lists(12, c, 100).cuda()
    call = lambda **kw: api.tl_attend_pages(c["q"], c["k"], c["v"], c["table"], c["length"], sel, **kw)
    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for k in range(3):
        for t in ("q", "k", "v"):
            c[t].normal_(0, 1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,kv,dim", [(64, 8, 64), (40, 8, 128), (16, 16, 80)])
def test_two_tiles_of_rows(gpu, heads, kv, dim, dtype):
    """Chunks of many tokens, which go 32 rows a workgroup."""
    print(f"attend_pages two tiles, {heads} on {kv} of {dim} {dtype}", flush=True)
    for kind in ("alike", "any"):
        c = cache_cases.make(13, dtype, heads, kv, dim, 16, [300, 0, 41], [301, 1, 260])
        check(c, lists(13, c, 7, kind))


def test_infinities_in_two_tiles(gpu):
    c = cache_cases.make(14, "bf16", 64, 8, 64, 16, [400], [300], poison=False)
    sel = lists(14, c, 5)
    sel[:, :, 0] = 3
    sel[:, :, 1:] = torch.where(sel[:, :, 1:] == 9, 8, sel[:, :, 1:])
    sel[200, 2, 4] = 9
    table = c["table"].cpu().long()
    c["v"][table[0, 9], 2, 7, 11] = -math.inf
    c["dense"][0][1][9 * 16 + 7, 2, 11] = -math.inf
    got, _ = run(c, sel)
    out, _, tol, _ = exact(c, sel)
    assert bool((got[200, 16:24, 11] == -math.inf).all())
    rest = torch.ones_like(got, dtype=torch.bool)
    rest[200, 16:24, 11] = False
    assert bool(torch.isfinite(got[rest]).all())
    assert bool(((got.double() - out).abs() <= tol)[rest].all())
