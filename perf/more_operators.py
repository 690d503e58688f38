"""The rest of an engine's iteration, as cases that can be timed and compared.

A case is one pass through an operator of ``paper_2408_05235_amd.api``: the norm
before a product (``norm``: with or without the residual's addition, its output in
the input's type or in e4m3 with scales), the summaries of the pages that new keys
went to (``bounds``), the pages that score best for each new token (``select``), its
attention over them alone (``attend``), and the next tokens drawn from their logits
(``sample``).  Batch sizes, lengths and tokens per page are those of
``paper_2408_05235_amd.configs`` and of the benchmark's other cases (requests in
flight, prompt and generated tokens, 16- and 24-token blocks); widths, head counts
and vocabularies are generic.

Fields of a case: ``kind``; ``B`` sequences, or rows of ``norm`` and ``sample``;
``W`` columns of a row (hidden size, vocabulary); ``dtype``; for ``norm``
``residual`` and ``group`` (-1: no 8 bits, 0: a scale a row, else columns of a scale);
for ``sample`` ``filters`` (whether rows have top-k, top-p and min-p) and ``masked``
(whether some tokens are forbidden); for the others ``lo``/``hi`` tokens that a sequence has in
the cache when the pass begins, ``nlo``/``nhi`` new ones (0 and 0: one each, and the
call gets no offsets), ``Hq``/``Hkv`` heads of ``D`` values, ``N`` tokens per page,
``K`` pages that a token selects, of them the ``first`` and the ``last`` ones always,
``order`` of a page (``head``: [head][token], ``token``: [token][head]) and ``lse``.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6
E4M3_MOST = 448.0
LEAST_SCALE = 2.0 ** -100
UNIT = 2.0 ** 40                # a weight of 1 in ``sample``, whose weights are whole numbers


def _case(name, kind, **kw):
    c = dict(name=name, kind=kind, B=1, W=0, dtype="bf16", residual=False, group=-1, filters=False, masked=False, lo=0,
             hi=0, nlo=0, nhi=0, Hq=32, Hkv=8, D=128, N=16, K=64, first=1, last=2, order="head", lse=False)
    c.update(kw)
    return c


def listed():
    return [
        # Before a product of one iteration of the smallest board's engine (64
        # requests), twice a layer: latency counts.
        _case("norm_step", "norm", B=64, W=4096, residual=True),
        # Before an 8-bit product of a wave of prompts, a scale for 128
        # columns (the largest memory traffic listed for the norm).
        _case("norm_prompts", "norm", B=16384, W=8192, residual=True, group=128),
        # A chunk's rows, a scale a row, a width that fills no wavefront evenly.
        _case("norm_chunk", "norm", B=1999, W=5000, dtype="f16", group=0),
        # One iteration of 256 requests in flight: the page that each one's new key
        # went to.
        _case("bounds_step", "bounds", B=256, lo=16, hi=4352),
        # A wave of prompts entered the cache: all their pages, of 24 tokens.
        _case("bounds_prompts", "bounds", B=32, nlo=16, nhi=4096, N=24, dtype="f16"),
        # One iteration over long contexts: 64 of 36864 tokens or fewer.
        _case("select_step", "select", B=64, lo=16, hi=36864),
        # Two chunks behind their cached contexts, pages for each of their
        # tokens; 24-token pages.
        _case("select_chunk", "select", B=2, lo=9001, hi=16384, nlo=512, nhi=512, N=24, dtype="f16"),
        # One request alone, far into a long context.
        _case("attend_one", "attend", B=1, lo=131071, hi=131071, K=128),
        # One iteration over long contexts, the selection's other half.
        _case("attend_step", "attend", B=64, lo=16, hi=36864, lse=True),
        # Two chunks behind their contexts, token-major pages.
        _case("attend_chunk", "attend", B=2, lo=9001, hi=16384, nlo=256, nhi=256, N=24, K=48, dtype="f16",
              order="token"),
        # One request's next token.
        _case("sample_one", "sample", B=1, W=32000, dtype="bf16", filters=True),
        # The next tokens of 256 requests, each with its own settings (the
        # largest memory traffic listed for the logits).
        _case("sample_board", "sample", B=256, W=128000, dtype="f32", filters=True, masked=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "bounds", "select", "select", "attend", "attend", "attend", "sample", "sample"])
    if kind == "norm":
        W = _log(rng, 1, 32768)
        if rng.random() < 0.6:
            W = max(8, W // 8 * 8)
        c = dict(W=W, B=_log(rng, 1, max(2, min(32768, (1 << 27) // W))), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                 residual=rng.random() < 0.6, group=rng.choice([-1, -1, 0, 32, 64, 128, 256]))
    elif kind == "sample":
        W = _log(rng, 1, 262144)
        c = dict(W=W, B=_log(rng, 1, max(2, min(512, (1 << 25) // W))), dtype=rng.choice(["bf16", "f16", "f32"]),
                 filters=rng.random() < 0.7, masked=rng.random() < 0.5)
    else:
        Hkv = rng.choice([1, 2, 4, 5, 8, 8])
        c = dict(Hkv=Hkv, Hq=Hkv * rng.choice([1, 2, 4, 4, 5, 8, 16, 20]), D=rng.choice([64, 128, 128, 128, 80, 256]),
                 N=rng.choice([16, 16, 24, 32, 7, 64]), dtype=rng.choice(["bf16", "f16"]),
                 order=rng.choice(["head", "token"]))
        if kind == "bounds":
            if rng.random() < 0.5:
                c.update(B=_log(rng, 1, 512), lo=1, hi=_log(rng, 2, 4352))
            else:
                c.update(B=rng.randint(1, 32), lo=0, hi=rng.choice([0, 500]), nlo=1, nhi=_log(rng, 16, 4096))
        else:
            first, last = rng.choice([0, 1, 1, 4]), rng.choice([1, 2, 2, 8])
            c.update(first=first, last=last, K=first + last + _log(rng, 1, 120))
            if rng.random() < 0.6:
                B = _log(rng, 1, 128)
                c.update(B=B, lo=1, hi=_log(rng, 16, min(131072, (1 << 22) // B // Hkv * 4)))
            else:
                B = rng.randint(1, 3)
                n = _log(rng, 2, 512)
                if kind == "attend":        # the plain form gathers every token's pages
                    n = max(1, min(n, (1 << 30) // (B * Hkv * c["K"] * c["N"] * c["D"])))
                c.update(B=B, lo=0, hi=_log(rng, 16, 16384), nlo=max(1, n // 2), nhi=n)
            c.update(lse=kind == "attend" and rng.random() < 0.4)
    return {k: v for k, v in _case("", kind, **c).items() if k != "name"}


# ---------------------------------------------------------------- the case's own numbers

def _lengths(case):
    """(length before the pass, new tokens) per sequence, from the case alone."""
    rng = np.random.RandomState([case["B"], case["lo"], case["hi"], case["nlo"], case["nhi"]])
    old = rng.randint(case["lo"], case["hi"] + 1, case["B"])
    new = np.ones(case["B"], np.int64)
    if case["nhi"]:
        new[:] = rng.randint(case["nlo"], case["nhi"] + 1, case["B"])
        new[0] = case["nhi"]                 # one at the end of the range
    old[0] = case["hi"]
    return old.astype(np.int64), new


def _pages(tokens, N):
    return -(-tokens // N)


def work(case):
    e = torch.finfo(DTYPES[case["dtype"]]).bits // 8
    B, W, N, D, Hkv = case["B"], case["W"], case["N"], case["D"], case["Hkv"]
    if case["kind"] == "norm":
        reads = W * e * (1 + 2 * case["residual"])      # (the sum is written)
        if case["group"] < 0:
            writes = W * e
        else:
            writes = W + 4 * (_pages(W, case["group"]) if case["group"] else 1)
        return {"bytes": B * (reads + writes) + W * e, "flops": 6 * B * W}
    if case["kind"] == "sample":
        return {"bytes": B * W * e + B * (6 * 4 + 8), "flops": 4 * B * W}
    old, new = _lengths(case)
    T, rows = int(new.sum()), int(new.sum()) * case["Hq"]
    if case["kind"] == "bounds":
        first = old // N
        touched = int((_pages(old + new, N) - first).sum())
        keys = int((old + new - first * N).sum())
        return {"bytes": Hkv * (keys * D * e + touched * (2 * D + 4)) + 4 * touched, "flops": 4 * keys * Hkv * D}
    seen = _pages(old + new, N)                         # a sequence's pages
    pairs = np.concatenate([np.arange(a, a + n) // N + 1 for a, n in zip(old, new)])    # of each token
    if case["kind"] == "select":
        return {"bytes": int(seen.sum()) * Hkv * (2 * D + 4) + 4 * int(seen.sum()) + rows * D * e + 4 * T * Hkv * case["K"],
                "flops": int(pairs.sum()) * case["Hq"] * 4 * D}
    taken = np.minimum(pairs, case["K"])
    # pages that some token of the sequence reads, at most
    read = int(np.minimum(seen, np.add.reduceat(taken, np.concatenate([[0], np.cumsum(new)[:-1]]))).sum())
    return {"bytes": read * Hkv * N * D * 2 * e + 2 * rows * D * e + 4 * T * Hkv * case["K"],
            "flops": 4 * int(taken.sum()) * N * case["Hq"] * D}


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    B, W, Hq, Hkv, D, N, K = (case[k] for k in ("B", "W", "Hq", "Hkv", "D", "N", "K"))

    def randn(*shape, std=1.0, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")
    s = dict(case=dict(case))
    if case["kind"] == "norm":
        # a few columns of hidden states are much larger than the others
        x = randn(B, W)
        x[:, :: 97] *= 12
        s.update(x=x, weight=(1 + 0.1 * randn(W, dtype=torch.float32)).to(dt),
                 residual=randn(B, W, std=2.0) if case["residual"] else None)
        return s
    if case["kind"] == "sample":
        # logits of a row: many small ones and some that stand out, more or less
        x = randn(B, W, std=1.5, dtype=torch.float32)
        x.add_((rand(B, W) < 50.0 / max(W, 50)) * 6 * rand(B, 1))
        if case["masked"]:
            x.masked_fill_(rand(B, W) < 0.05, -math.inf)
            x.masked_fill_(rand(B, W) < 0.01, torch.finfo(dt).min)
            x[:, :1] = 0
        s.update(x=x.to(dt), u=rand(B), temperature=0.3 + rand(B))
        s["temperature"][rand(B) < 0.1] = 0          # some ask for the best token
        s.update(top_k=None, top_p=None, min_p=None)
        if case["filters"]:
            # some rows without one or the other
            k = torch.exp(rand(B) * math.log(2000)).to(torch.int32)
            s["top_k"] = torch.where(rand(B) < 0.4, 0, k).to(torch.int32)
            s["top_p"] = torch.where(rand(B) < 0.3, 1.0, 0.5 + 0.5 * rand(B))
            s["min_p"] = torch.where(rand(B) < 0.6, 0.0, 0.1 * rand(B))
        return s
    old, new = _lengths(case)
    dev = lambda a, t=torch.int32: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", t)
    have = _pages(old + new, N)
    pool, width = int(have.sum()) + 3, int(have.max())
    # a table of pages in no order, as after some time of service
    place = torch.randperm(pool, generator=g, device="cuda")[: int(have.sum())]
    at = np.concatenate([np.arange(b * width, b * width + h) for b, h in enumerate(have)])
    table = torch.full((B * width,), -1, dtype=torch.int32, device="cuda")
    table[torch.from_numpy(at).cuda()] = place.to(torch.int32)
    s.update(table=table.view(B, width), length=dev(old + new))
    s["offset"] = dev(np.concatenate([[0], np.cumsum(new)]), torch.int64) if case["nhi"] else None
    T = s["tokens"] = int(new.sum())
    if case["kind"] != "select":
        shape = (pool, Hkv, N, D) if case["order"] == "head" else (pool, N, Hkv, D)
        pages = [randn(*shape) for _ in range(1 + (case["kind"] == "attend"))]
        if case["order"] == "token":
            pages = [x.transpose(1, 2) for x in pages]
        s["k"] = pages[0]
    if case["kind"] == "bounds":
        # what is there from earlier iterations stays where no new key is
        s["bounds"] = torch.randint(-127, 128, (pool, Hkv, 2, D), dtype=torch.int8, generator=g, device="cuda")
        s["scale"] = rand(pool, Hkv)
        return s
    # queries as a layer's one product leaves them
    s["q"] = randn(T, Hq + 2 * Hkv, D, std=1.5)[:, :Hq]
    if case["kind"] == "select":
        # the largest and the least of a page's keys, in 127ths of its largest
        # value: about half of it
        hi = randn(pool, Hkv, D, std=18.0, dtype=torch.float32).add_(64).round_().clamp_(-40, 127)
        lo = randn(pool, Hkv, D, std=18.0, dtype=torch.float32).sub_(64).round_().clamp_(-127, -41)
        s["bounds"] = torch.stack([lo, hi], 2).to(torch.int8)
        s["scale"] = torch.exp(0.2 * randn(pool, Hkv, dtype=torch.float32)) * (3.5 / 127)
        return s
    s["v"] = pages[1]
    # pages that neighbouring tokens select are alike
    selected = torch.full((T, Hkv, K), -1, dtype=torch.int32, device="cuda")
    first = 0
    for a, n, h in zip(old.tolist(), new.tolist(), have.tolist()):
        j = torch.arange(h, device="cuda")
        cur = torch.arange(a, a + n, device="cuda")[:, None] // N
        x = rand(1, Hkv, h) + 0.5 * rand(n, Hkv, h)
        x.masked_fill_(((j < case["first"]) | (j > cur - case["last"]))[:, None], 3.0)
        x.masked_fill_((j > cur)[:, None], -1.0)
        x, at = x.topk(min(K, h), 2)
        at = torch.where(x < 0, h, at).sort(2).values
        selected[first: first + n, :, : at.shape[2]] = torch.where(at == h, -1, at).to(torch.int32)
        first += n
    s["selected"] = selected
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2408_05235_amd import api
    c = s["case"]
    if c["kind"] == "norm":
        r = api.tl_norm(s["x"], s["weight"], EPS, residual=s["residual"], group=None if c["group"] < 0 else c["group"])
        return list(r) if isinstance(r, tuple) else [r]
    if c["kind"] == "sample":
        return list(api.tl_sample(s["x"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], want_logprob=True))
    if c["kind"] == "bounds":
        api.tl_page_bounds(s["k"], s["bounds"], s["scale"], s["table"], s["length"], s["tokens"], s["offset"])
        return [s["bounds"], s["scale"]]
    if c["kind"] == "select":
        return [api.tl_select_pages(s["q"], s["bounds"], s["scale"], s["table"], s["length"], c["N"], c["K"], s["offset"],
                                    first=c["first"], last=c["last"])]
    r = api.tl_attend_pages(s["q"], s["k"], s["v"], s["table"], s["length"], s["selected"], s["offset"], want_lse=c["lse"])
    return list(r) if c["lse"] else [r]


def _run_plain(s):
    return globals()["_%s_plain" % s["case"]["kind"]](s)


def _norm_plain(s):
    c = s["case"]
    x = s["x"].float()
    h = x if s["residual"] is None else x + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"].float()
    after = [] if s["residual"] is None else [h.to(s["x"].dtype)]
    if c["group"] < 0:
        return [y.to(s["x"].dtype)] + after
    B, W = y.shape
    per = c["group"] or W
    n = _pages(W, per)
    z = torch.nn.functional.pad(y, (0, n * per - W)).view(B, n, per)
    scale = (z.abs().amax(2) / E4M3_MOST).clamp(min=LEAST_SCALE)
    q = (z / scale[:, :, None]).clamp(-E4M3_MOST, E4M3_MOST).view(B, n * per)[:, :W]
    return [q.to(torch.float8_e4m3fn), scale[:, 0] if c["group"] == 0 else scale] + after


def _new_tokens(s, T):
    """Sequence and position of every new token."""
    length = s["length"].long()
    if s["offset"] is None:
        return torch.arange(T, device=length.device), length - 1
    token = torch.arange(T, device=length.device)
    seq = torch.searchsorted(s["offset"], token, right=True) - 1
    return seq, length[seq] - (s["offset"][seq + 1] - token)


def _bounds_plain(s):
    c = s["case"]
    N = c["N"]
    k, table, length = s["k"], s["table"], s["length"].long()
    n = torch.ones_like(length) if s["offset"] is None else s["offset"].diff()
    j = torch.arange(table.shape[1], device=table.device)
    touched = (j >= ((length - n) // N)[:, None]) & (j < _pages(length, N)[:, None])
    seq, j = torch.nonzero(touched, as_tuple=True)
    page = table[seq, j].long()
    x = k[page].float()
    there = (j[:, None] * N + torch.arange(N, device=j.device) < length[seq][:, None])[:, None, :, None]
    hi, lo = torch.where(there, x, -math.inf).amax(2), torch.where(there, x, math.inf).amin(2)
    scale = torch.maximum(hi, -lo).amax(2) * (1.0 / 127)
    per = torch.where(scale > 0, scale, 1.0)[:, :, None]
    s["bounds"][page] = torch.stack([(lo / per).floor(), (hi / per).ceil()], 2).clamp(-127, 127).to(torch.int8)
    s["scale"][page] = scale
    return [s["bounds"], s["scale"]]


def _select_plain(s):
    c = s["case"]
    N, D, Hq, Hkv, K = c["N"], c["D"], c["Hq"], c["Hkv"], c["K"]
    B, width = s["table"].shape
    T = s["q"].shape[0]
    seq, pos = _new_tokens(s, T)
    most, row = (1, torch.zeros_like(seq)) if s["offset"] is None else (c["nhi"], torch.arange(T, device=seq.device) - s["offset"][seq])
    # queries in 127ths of their largest value
    q = s["q"].float()
    z = q.abs().amax(2) * (1.0 / 127)
    i = (q / torch.where(z > 0, z, 1.0)[:, :, None]).round()
    both = torch.zeros(B, most, Hq, 2 * D, device=q.device)
    both[seq, row] = torch.cat([i.clamp(max=0), i.clamp(min=0)], 2)      # times the least, times the largest
    both = both.view(B, most, Hkv, Hq // Hkv, 2 * D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, most * (Hq // Hkv), 2 * D)
    at = s["table"].long().clamp(min=0)
    bounds = s["bounds"][at].view(B, width, Hkv, 2 * D).permute(0, 2, 1, 3).float()
    # (whole numbers below 2^24: exact)
    dot = torch.matmul(both, bounds.transpose(2, 3).contiguous()).view(B, Hkv, most, Hq // Hkv, width)
    scales = torch.zeros(B, most, Hq, device=q.device)
    scales[seq, row] = z
    dot = dot.mul_(scales.view(B, most, Hkv, Hq // Hkv).permute(0, 2, 1, 3)[..., None]).amax(3)
    score = dot.mul_(s["scale"][at].permute(0, 2, 1)[:, :, None]).permute(0, 2, 1, 3)[seq, row]     # [T, Hkv, width]
    j = torch.arange(width, device=q.device)
    cur = (pos // N)[:, None]
    score.masked_fill_(((j < c["first"]) | (j > cur - c["last"]))[:, None], math.inf)
    score.masked_fill_((j > cur)[:, None], -math.inf)
    best = torch.sort(score, dim=2, descending=True, stable=True).indices[:, :, :K]
    best = torch.where(best > cur[:, :, None], width, best).sort(2).values
    out = torch.full((T, Hkv, K), -1, dtype=torch.int32, device=q.device)
    out[:, :, : best.shape[2]] = torch.where(best == width, -1, best)
    return [out]


def _attend_plain(s):
    c = s["case"]
    N, D, Hq, Hkv, K = c["N"], c["D"], c["Hq"], c["Hkv"], c["K"]
    T = s["q"].shape[0]
    seq, pos = _new_tokens(s, T)
    sel = s["selected"].long()
    page = s["table"][seq[:, None, None], sel.clamp(min=0)].long()
    head = torch.arange(Hkv, device=sel.device)[:, None]
    k = s["k"][page, head].float().view(T, Hkv, K * N, D)
    t = sel[..., None] * N + torch.arange(N, device=sel.device)
    see = ((sel >= 0)[..., None] & (t <= pos[:, None, None, None])).view(T, Hkv, 1, K * N)
    x = torch.matmul(s["q"].float().reshape(T, Hkv, Hq // Hkv, D), k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D))
    del k
    x.masked_fill_(~see, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m)
    l = p.sum(-1, keepdim=True)
    v = torch.where(see.view(T, Hkv, K * N, 1), s["v"][page, head].float().view(T, Hkv, K * N, D), 0.0)
    out = (torch.matmul(p, v) / l).reshape(T, Hq, D).to(s["q"].dtype)
    return [out, (m + torch.log(l)).reshape(T, Hq)] if c["lse"] else [out]


def _sample_plain(s):
    x = s["x"].float() + 0.0                    # one zero
    x = torch.where(torch.isnan(x), -math.inf, x)
    B, V = x.shape
    xs, at = torch.sort(x, dim=1, descending=True, stable=True)
    m = xs[:, :1]
    # in 64 bits, and weights as whole numbers, whose sums are exact
    temperature = s["temperature"].double()[:, None]
    best = ~(temperature > 0)
    e = torch.where(xs == m, 0.0, (xs.double() - m.double()) / torch.where(best, 1.0, temperature))
    e = torch.where(xs == -math.inf, -math.inf, e)
    w = torch.round(torch.exp(e) * UNIT).long()
    rank = torch.arange(V, device=x.device)[None]
    kept = (rank == 0) | ~best
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        kept &= (k <= 0) | (rank < k)
    w = torch.where(kept, w, 0)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        run_up = torch.cumsum(w, 1)
        need = torch.ceil(p * run_up[:, -1:].double()).long()
        w = torch.where(~(p < 1) | (run_up - w < need) | (rank == 0), w, 0)
    if s["min_p"] is not None:
        least = torch.ceil(s["min_p"].double()[:, None].clamp(0, 1) * UNIT).long()
        w = torch.where(w >= least, w, 0)
    total = w.sum(1)
    there = torch.zeros_like(w).scatter_(1, at, w)
    r = torch.minimum(torch.floor(s["u"].double() * total.double()).long(), total - 1)
    token = (torch.cumsum(there, 1) <= r[:, None]).sum(1)
    e_at = torch.zeros_like(e).scatter_(1, at, e)
    logprob = e_at.gather(1, token[:, None].clamp(max=V - 1))[:, 0] - torch.log(total.double() / UNIT)
    return [token.to(torch.int32), logprob.float()]


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The definitions in float64, a sequence, a token or a row at a time."""
    if case["kind"] == "select":                # whole numbers only
        return None
    s = prepare(case, seed)
    if case["kind"] == "norm":
        h = s["x"].double()
        if case["residual"]:
            h = h + s["residual"].double()
        y = h / torch.sqrt(h.square().sum(1, keepdim=True) / case["W"] + EPS) * s["weight"].double()
        after = [h] if case["residual"] else []
        if case["group"] < 0:
            return [y] + after
        scales = [p.abs().amax(1).div(E4M3_MOST).clamp_min(LEAST_SCALE) for p in y.split(case["group"] or case["W"], 1)]
        q = torch.cat([p / z[:, None] for p, z in zip(y.split(case["group"] or case["W"], 1), scales)], 1)
        return [q, scales[0] if case["group"] == 0 else torch.stack(scales, 1)] + after
    if case["kind"] == "bounds":
        old, new = _lengths(case)
        scale, N = s["scale"].double(), case["N"]
        for b, (a, n) in enumerate(zip(old.tolist(), new.tolist())):
            j = torch.arange(a // N, _pages(a + n, N), device="cuda")
            page = s["table"][b].long()[j]
            most = s["k"][page].double().abs().amax(3)
            most[-1, :, (a + n - 1) % N + 1:] = 0
            scale[page] = most.amax(2) / 127
        return [None, scale]
    if case["kind"] == "attend":
        old, new = _lengths(case)
        T, Hq, Hkv, N, D = int(new.sum()), case["Hq"], case["Hkv"], case["N"], case["D"]
        if T * Hkv > 8192:
            return None
        seq, pos = np.repeat(np.arange(case["B"]), new), np.concatenate([np.arange(a, a + n) for a, n in zip(old, new)])
        out = torch.zeros(T, Hq, D, dtype=torch.float64, device="cuda")
        lse = torch.zeros(T, Hq, dtype=torch.float64, device="cuda")
        line = torch.arange(N, device="cuda")
        for i in range(T):
            for g in range(Hkv):
                j = s["selected"][i, g].long()
                j = j[j >= 0]
                page = s["table"][int(seq[i])].long()[j]
                seen = (j[:, None] * N + line <= int(pos[i])).view(-1)
                k, v = (s[z][page, g].reshape(-1, D)[seen].double() for z in ("k", "v"))
                heads = slice(g * (Hq // Hkv), (g + 1) * (Hq // Hkv))
                x = s["q"][i, heads].double() @ k.T / math.sqrt(D)
                lse[i, heads] = torch.logsumexp(x, 1)
                out[i, heads] = torch.exp(x - lse[i, heads][:, None]) @ v
        return [out, lse] if case["lse"] else [out]
    # a row at a time on the host, the weights whole numbers by definition
    logprob = np.zeros(case["B"])
    x = s["x"].float().cpu().numpy()
    get = lambda name: None if s[name] is None else s[name].cpu().numpy()
    u, T, top_k, top_p, min_p = (get(n) for n in ("u", "temperature", "top_k", "top_p", "min_p"))
    for b in range(case["B"]):
        row = np.where(np.isnan(x[b]), -np.inf, x[b]).astype(np.float64)
        m = row.max()
        if not T[b] > 0:
            continue
        with np.errstate(invalid="ignore"):
            e = (row - m) / np.float64(T[b])
        w = np.rint(np.exp(e) * UNIT).astype(np.int64)
        live = np.flatnonzero(w)
        order = live[np.lexsort((live, -row[live]))]
        if top_k is not None and top_k[b] > 0:
            order = order[: top_k[b]]
        if top_p is not None and top_p[b] < 1:
            sums = np.cumsum(w[order])
            order = order[: 1 + int(np.searchsorted(sums, int(np.ceil(np.float64(top_p[b]) * np.float64(sums[-1])))))]
        if min_p is not None:
            order = order[w[order] >= int(np.ceil(np.float64(min_p[b]) * UNIT))]
        order = np.sort(order)
        sums = np.cumsum(w[order])
        r = min(int(np.floor(np.float64(u[b]) * np.float64(sums[-1]))), int(sums[-1]) - 1)
        i = order[int(np.searchsorted(sums, r, side="right"))]
        logprob[b] = e[i] - math.log(sums[-1] / UNIT)
    return [None, torch.from_numpy(logprob)]
