"""Attention over the paged cache against its definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import cache_cases as cc

pytestmark = pytest.mark.gpu


def run(c, **kw):
    from paper_2408_05235_amd import api
    print({k: v for k, v in c.items() if k in ("dtype", "page", "window", "sinks")}, tuple(c["q"].shape),
          tuple(c["k"].shape), flush=True)
    out, lse = api.tl_attend(c["q"], c["k"], c["v"], c["table"], c["length"], c["offset"], window=c["window"],
                             sinks=c["sinks"], want_lse=True, **kw)
    torch.cuda.synchronize()
    return out, lse


def lengths(n, most, seed=0):
    """Short and long, the ends of tiles among them."""
    r = np.random.RandomState(seed)
    edge = [x for x in (0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257) if x <= most]
    return [edge[i] if i < len(edge) else int(r.randint(0, most + 1)) for i in range(n)]


DECODE = [
    # dtype, heads, kv_heads, dim, page, window, sinks, order
    ("bf16", 8, 2, 128, 16, 0, 0, "head"),
    ("f16", 8, 8, 64, 16, 0, 0, "token"),
    ("bf16", 5, 5, 128, 24, 0, 0, "head"),
    ("f16", 32, 2, 128, 7, 0, 0, "token"),
    ("bf16", 40, 2, 64, 1, 0, 0, "head"),
    ("bf16", 6, 2, 256, 16, 0, 0, "head"),
    ("f16", 4, 4, 8, 16, 0, 0, "head"),
    ("bf16", 3, 1, 80, 32, 0, 0, "token"),
    ("f16", 12, 4, 200, 24, 0, 0, "head"),
    ("bf16", 71, 1, 64, 64, 0, 0, "head"),
    ("bf16", 8, 2, 128, 16, 1, 0, "head"),
    ("f16", 8, 2, 128, 16, 33, 1, "head"),
    ("bf16", 8, 1, 64, 24, 100, 4, "token"),
    ("f16", 4, 2, 128, 16, 16, 100, "head"),
    ("bf16", 4, 1, 128, 16, 5000, 3, "head"),
]


@pytest.mark.parametrize("dtype,heads,kv,dim,page,window,sinks,order", DECODE)
def test_one_new_token(gpu, dtype, heads, kv, dim, page, window, sinks, order):
    L = np.asarray(lengths(24, 700))
    one = (L > 0).astype(np.int64)
    # an idle slot (length 0) has a row all the same: it gives zeros
    c = cc.make(1, dtype, heads, kv, dim, page, L - one, np.ones_like(L) * one, window, sinks, order, offsets=False)
    rows = torch.zeros((len(L),) + c["q"].shape[1:], dtype=c["q"].dtype, device="cuda")
    live = torch.from_numpy(np.flatnonzero(one)).cuda()
    rows[live] = c["q"]
    full = dict(c, q=rows)
    out, lse = run(full)
    idle = torch.from_numpy(np.flatnonzero(one == 0)).cuda()
    assert bool((out[idle] == 0).all()) and bool((lse[idle] == -math.inf).all())
    cc.check(c, out[live], lse[live])


@pytest.mark.parametrize("dtype,heads,kv,dim,page,window,sinks,order", DECODE)
def test_prompts_and_chunks(gpu, dtype, heads, kv, dim, page, window, sinks, order):
    new = [1, 0, 2, 17, 130, 64, 3, 257, 5]
    before = [0, 9, 100, 0, 0, 333, 20, 0, 640]
    c = cc.make(2, dtype, heads, kv, dim, page, before, new, window, sinks, order)
    cc.check(c, *run(c))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (64, 4), (511, 0), (300, 130)])
def test_long_prompt(gpu, dim, window, sinks):
    c = cc.make(3, "bf16", 4, 2, dim, 16, [0, 700], [1500, 900], window, sinks)
    cc.check(c, *run(c))


@pytest.mark.parametrize("window,sinks", [(0, 0), (1000, 8)])
def test_long_cache_few_rows(gpu, window, sinks):
    c = cc.make(4, "f16", 16, 2, 128, 16, [20000, 17, 9999], [1, 1, 1], window, sinks, offsets=False)
    cc.check(c, *run(c))
    c = cc.make(5, "bf16", 8, 2, 128, 24, [15000, 3], [40, 2], window, sinks)
    cc.check(c, *run(c))


@pytest.mark.parametrize("seed", range(24))
def test_random(gpu, seed):
    r = np.random.RandomState(seed)
    kv = int(r.randint(1, 6))
    heads = kv * int(r.choice([1, 2, 3, 4, 7, 8, 16, 17]))
    B = int(r.randint(1, 9))
    before = r.randint(0, r.choice([3, 70, 900]), B)
    new = r.randint(0, r.choice([2, 5, 40, 300]), B)
    new[r.randint(B)] += 1
    window = int(r.choice([0, 0, 1, 7, 64, 200]))
    c = cc.make(100 + seed, str(r.choice(["bf16", "f16"])), heads, kv, int(r.choice([16, 40, 64, 96, 128, 192, 256])),
                int(r.choice([1, 5, 8, 16, 24, 48, 128])), before, new, window, int(r.choice([0, 2, 33])),
                str(r.choice(["head", "token"])))
    cc.check(c, *run(c))


@pytest.mark.parametrize("dtype,dim,group,page", [("bf16", 128, 2, 16), ("f16", 64, 1, 16), ("bf16", 256, 2, 24),
                                                  ("f16", 80, 3, 7)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 3)])
def test_a_few_long_among_many_single(gpu, dtype, dim, group, page, window, sinks):
    """Offsets where nearly all sequences have one new token: those with more are
    found, whatever comes between; with a table so wide that the call may have much to
    read, and one that has no room for that."""
    r = np.random.RandomState(dim)
    new = np.ones(64, np.int64)
    new[[5, 6, 20, 33, 40, 63]] = 40, 17, 0, 19, 0, 33
    before = r.randint(0, 200, 64)
    before[7], before[40] = 0, 50
    c = cc.make(18, dtype, 8 * group, 8, dim, page, before, new, window, sinks)
    cc.check(c, *run(c))
    wide = torch.full((64, 200 * 16 // page), -1, dtype=torch.int32, device="cuda")
    wide[:, :c["table"].shape[1]] = c["table"]
    c["table"] = wide
    cc.check(c, *run(c))
    cc.check(c, *run(c, max_length=int(c["length"].max())))


def test_peaked_and_low_scores(gpu):
    # wide scores: most weights vanish, the largest comes late or early
    c = cc.make(6, "bf16", 8, 2, 128, 16, [600, 0, 3000], [1, 200, 33], spread=6.0)
    cc.check(c, *run(c))
    c = cc.make(7, "f16", 8, 2, 64, 16, [600, 0, 3000], [1, 200, 33], spread=8.0)
    cc.check(c, *run(c))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 20])
def test_many_small_weights(gpu, dtype, new):
    """One token outweighs each of 32768 others by e^18 (2^26), and its value
    is 0: what is left of the output is the others'.  A weight may be off by 2^-8 of
    itself (bf16; 2^-11 in f16), and in f16 by 2^-31 of the largest, the output by
    2^-8 (2^-11) of itself."""
    L, dim = 32768, 64
    c = cc.make(17, dtype, 2, 1, dim, 16, [L], [new])
    c["q"] = torch.zeros(new, 2, dim, dtype=cc.DTYPES[dtype], device="cuda")
    c["q"][:, :, 3] = 1.0
    c["k"].zero_()
    c["v"].fill_(1.0)
    at = 700
    page = int(c["table"][0, at // 16])
    c["k"][page, 0, at % 16, 3] = 18.0
    c["v"][page, 0, at % 16] = 0.0
    out, lse = run(c, scale=1.0)
    others = torch.arange(L, L + new, device="cuda").double()[:, None, None]
    all = math.exp(18.0) + others
    exact = others / all
    u = 2.0 ** -11 if dtype == "f16" else 2.0 ** -8
    tol = exact * (2.1 * u + 2.0 ** -14) + (2.0 ** -31 * others if dtype == "f16" else 0)
    assert bool(((out.double() - exact).abs() <= tol).all()), (float(out[0, 0, 0]), float(exact[0, 0, 0]))
    assert bool(((lse.double() - torch.log(all)[:, :, 0]).abs() <= 2.0 ** -17).all())


@pytest.mark.parametrize("dtype,q,k", [("f16", 60000.0, 60000.0), ("f16", 30000.0, 2000.0), ("bf16", 1e14, 1e15),
                                       ("bf16", 1e4, 1e4), ("f16", -60000.0, 60000.0), ("bf16", -1e14, 1e15)])
@pytest.mark.parametrize("new", [1, 20])
@pytest.mark.parametrize("rising", [False, True])
def test_large_scores(gpu, dtype, q, k, new, rising):
    """Scores so large that their distances are all that counts: the output is
    the value of the token with the largest one, exactly, and lse that score (2^-20 of
    itself: its product, the scale and the logarithm's factor, each rounded to 24 bits)."""
    L, dim = 3000, 64
    c = cc.make(19, dtype, 2, 1, dim, 16, [L], [new])
    t = torch.arange(L + new, device="cuda")
    steps = (t // 12 if rising else (L + new - 1 - t) // 12).float()       # 12 tokens each have the same score
    top = steps == steps.max() if q > 0 else steps == 0
    keys = (k * (0.5 + steps / 1024)).to(cc.DTYPES[dtype])
    top = keys == (keys.max() if q > 0 else keys.min())
    values = torch.where(top, 3.0, -5.0).to(cc.DTYPES[dtype])
    page = c["table"][0].long()[t // 16]
    c["k"].zero_()
    c["q"] = torch.zeros(new, 2, dim, dtype=cc.DTYPES[dtype], device="cuda")
    c["q"][:, :, 3] = q
    c["k"][page, 0, t % 16, 3] = keys
    c["v"][page, 0, t % 16] = values[:, None]
    out, lse = run(c, scale=1.0)
    q1 = float(c["q"][0, 0, 3])
    for i in range(new):
        seen = keys[: L + i + 1].double() * q1
        best = seen == seen.max()
        assert bool((values[: L + i + 1][best] == values[: L + i + 1][best][0]).all())
        assert bool((out[i] == values[: L + i + 1][best][0]).all()), (i, float(out[i, 0, 0]))
        want = float(seen.max()) + math.log(int(best.sum()))
        assert bool(((lse[i].double() - want).abs() <= 2.0 ** -20 * abs(want) + 2.0 ** -18).all())


def test_scale(gpu):
    c = cc.make(8, "f16", 4, 2, 64, 16, [100, 0], [1, 70])
    cc.check(c, *run(c, scale=0.7), scale=0.7)
    cc.check(c, *run(c, scale=1e-30), scale=1e-30)


def test_one_row_sees_what_another_must_not(gpu):
    """Infinities and NaN in keys and values of a token that only later rows
    see stay out of the earlier rows."""
    for value in (math.inf, -math.inf, math.nan):
        for heads, before, new, at in ((4, 40, 3, 42), (8, 5, 200, 150), (1, 300, 5, 303)):
            c = cc.make(9, "bf16", heads, 1, 128, 16, [before], [new])
            page, row = int(c["table"][0, at // 16]), at % 16
            c["v"][page, 0, row, 3] = value
            c["k"][page, 0, row, 5] = value
            out, lse = run(c)
            early = at - before                  # rows before it
            part = dict(c, q=c["q"][:early], new=np.asarray([early]))
            if early:
                part["dense"] = [tuple(x[:before + early] for x in c["dense"][0])]
                cc.check(part, out[:early], lse[:early])


def test_all_scores_minus_infinity(gpu):
    c = cc.make(10, "bf16", 2, 1, 64, 16, [20], [1], offsets=False)
    c["q"][:] = 1.0
    page = c["table"][0].long()[torch.arange(21, device="cuda") // 16]
    c["k"][page, 0, torch.arange(21, device="cuda") % 16, 0] = -math.inf
    out, lse = run(c)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_missing_pages_are_not_seen(gpu):
    for new in ([1, 1], [30, 100]):
        c = cc.make(11, "f16", 4, 2, 64, 16, [200, 90], new)
        c["table"][0, 2] = -5
        c["table"][0, 3] = c["k"].shape[0]
        c["table"][1, 0] = 2 ** 31 - 1
        gone = [(32, 64), (0, 16)]
        see = lambda b, p, t: (t <= p) & ((t < gone[b][0]) | (t >= gone[b][1]))
        cc.check(c, *run(c), see=see)


def test_lengths_beyond_the_table_and_below_the_rows(gpu):
    c = cc.make(12, "bf16", 2, 2, 64, 16, [10, 40], [4, 8])
    full = run(c)
    # more tokens than the table has room for: those it has
    c["length"][1] = 10 ** 6
    w = c["table"].shape[1]
    c["table"][1, :] = c["table"][1, 0]
    out, _ = run(c)
    assert torch.equal(out[:4], full[0][:4])
    kb = c["dense"][1][0][torch.arange(w * 16) % 16], c["dense"][1][1][torch.arange(w * 16) % 16]
    d = dict(c, dense=[c["dense"][0], kb], before=np.asarray([10, w * 16 - 8]))
    see = lambda b, p, t: (t <= p) if b == 0 else (t >= 0) & (p >= 0)
    cc.check(d, out, None, see=see)
    # fewer than the new rows: the first rows have no position
    c["length"][0] = 2
    out, lse = run(c)
    assert bool((out[:2] == 0).all()) and bool((lse[:2] == -math.inf).all())
    c["length"][0] = -7
    out, lse = run(c)
    assert bool((out[:4] == 0).all()) and bool((lse[:4] == -math.inf).all())


def test_rows_of_no_sequence_are_left_alone(gpu):
    from paper_2408_05235_amd import api
    c = cc.make(13, "bf16", 4, 2, 64, 16, [10, 40], [4, 8])
    q = torch.cat([c["q"], c["q"][:3]])
    out = torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda")
    api.tl_attend(q, c["k"], c["v"], c["table"], c["length"], c["offset"], out=out)
    cc.check(c, out[:12], None)
    assert bool((out[12:] == 5.0).all())


def test_workspace_and_max_length_change_rounding_only(gpu):
    c = cc.make(14, "bf16", 8, 2, 128, 16, [5000, 10, 700], [1, 1, 1], offsets=False)
    for kw in (dict(workspace=torch.empty(0, dtype=torch.uint8, device="cuda")),
               dict(workspace=torch.empty(70000, dtype=torch.uint8, device="cuda")), dict(max_length=5001),
               dict(max_length=100)):
        cc.check(c, *run(c, **kw))


@pytest.mark.parametrize("new,offsets", [([1, 1, 1], False), ([1, 140, 9], True)])
def test_bit_identical_and_on_other_streams(gpu, new, offsets):
    c = cc.make(15, "bf16", 8, 2, 128, 16, [5000, 10, 700], new, offsets=offsets)
    ref = run(c)
    for _ in range(3):
        again = run(c)
        assert torch.equal(again[0], ref[0]) and torch.equal(again[1], ref[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run(c)
    side.synchronize()
    assert torch.equal(again[0], ref[0])


@pytest.mark.parametrize("new,offsets", [([1, 1, 1], False), ([1, 140, 9], True)])
def test_in_a_graph(gpu, new, offsets):
    from paper_2408_05235_amd import api
    c = cc.make(16, "bf16", 8, 2, 128, 16, [5000, 10, 700], new, offsets=offsets)
    args = (c["q"], c["k"], c["v"], c["table"], c["length"], c["offset"])
    ref = api.tl_attend(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    out = torch.empty_like(ref)
    with torch.cuda.stream(side):
        api.tl_attend(*args, out=out)
        side.synchronize()
        with torch.cuda.graph(g, stream=side):
            api.tl_attend(*args, out=out)
    for i in range(4):
        out.fill_(float("nan"))
        eager = api.tl_attend(*args)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(eager, ref), i


def test_offsets_beyond_32_bits(gpu):
    """Pages past 2^32 elements of a large pool."""
    page, dim, kv = 16, 128, 4
    pages = 2 ** 32 // (page * dim * kv) + 600
    k = torch.empty((pages, kv, page, dim), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    c = cc.make(17, "bf16", 8, kv, dim, page, [500, 3], [1, 90])
    n = c["k"].shape[0]
    k[-n:], v[-n:] = c["k"], c["v"]
    table = torch.where(c["table"] >= 0, c["table"] + (pages - n), c["table"])
    c = dict(c, k=k, v=v, table=table)
    cc.check(c, *run(c))


def test_no_tokens_no_sequences(gpu):
    from paper_2408_05235_amd import api
    c = cc.make(18, "bf16", 4, 2, 64, 16, [10, 40], [0, 0], poison=False)
    assert api.tl_attend(c["q"], c["k"], c["v"], c["table"], c["length"], c["offset"]).shape == (0, 4, 64)
    empty = torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    assert api.tl_attend(c["q"], c["k"], c["v"], empty, empty[:, 0].contiguous()).shape == (0, 4, 64)
    # a table without entries: every row is empty
    c = cc.make(19, "bf16", 4, 2, 64, 16, [0], [2], poison=False)
    none = torch.zeros((1, 0), dtype=torch.int32, device="cuda")
    out = api.tl_attend(c["q"], c["k"], c["v"], none, c["length"], c["offset"])
    assert bool((out == 0).all())
