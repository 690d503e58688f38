"""The paged cache and the attention over it, as cases that can be timed and compared.

A case is one pass through an operator of ``paper_2408_05235_amd.api``: new keys
and values written to their pages (``append``), attention of new tokens over a
paged cache (``attend``: one new token per sequence, prompts, chunks of prompts
behind a cached context, both mixed, with or without a sliding window and first
tokens that stay visible), sequences forked, extended and freed (``fork``), and
a fragmented pool compacted (``compact``).  Batch sizes, lengths and tokens per
page are those of ``paper_2408_05235_amd.configs`` and of the benchmark's other
cases (requests in flight, prompt and generated tokens, 16- and 24-token
blocks); head counts and sizes are generic.

Fields of a case: ``kind``; ``B`` sequences; ``lo``/``hi`` tokens that a
sequence has in the cache when the pass begins; ``nlo``/``nhi`` new tokens per
sequence (0 and 0: one each, and the call gets no offsets); ``decodes`` further
sequences with one new token each; ``Hq``/``Hkv`` heads of ``D`` values; ``N``
tokens per page; ``window`` (0 = none) and ``sinks``; ``dtype`` of cache and
inputs; ``order`` of a page (``head``: [head][token], ``token``: [token][head]);
``lse`` whether the scores' log-sum is asked for; and for pages ``planes``
(layers x 2), ``pool`` pages and ``grow`` tokens that a fork gets.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _case(name, kind, **kw):
    c = dict(name=name, kind=kind, B=1, lo=0, hi=0, nlo=0, nhi=0, decodes=0, Hq=32, Hkv=8, D=128, N=16, window=0,
             sinks=0, dtype="bf16", order="head", lse=False, planes=0, pool=0, grow=0)
    c.update(kw)
    return c


def listed():
    return [
        # One iteration of the smallest board's engine (64 requests): each
        # request's new key and value to its page.  Runs in every layer, so
        # its latency counts.
        _case("append_step", "append", B=64, lo=16, hi=1280),
        # A wave of prompts enters the cache: 24-token pages, odd lengths.
        _case("append_prompts", "append", B=32, nlo=16, nhi=4096, N=24, dtype="f16"),
        # One request alone on the engine, a page or so into its answer.
        _case("decode_one", "attend", B=1, lo=1000, hi=1000),
        # One iteration of the smallest board: 64 requests of 16 to 1280
        # tokens.
        _case("decode_board", "attend", B=64, lo=16, hi=1280, lse=True),
        # 256 requests in flight, prompts up to 4096 and up to 256 generated,
        # every head with its own keys (the largest memory traffic listed).
        _case("decode_256", "attend", B=256, lo=16, hi=4352, Hq=20, Hkv=20, dtype="f16"),
        # Long contexts under a batch cap: few requests, so the cache's
        # length has to be split; token-major 24-token pages.
        _case("decode_long", "attend", B=4, lo=20011, hi=36864, Hq=64, N=24, order="token"),
        # Long contexts with a window and first tokens that stay.
        _case("decode_window", "attend", B=48, lo=1, hi=32768, window=4096, sinks=4, D=64),
        # A wave of ragged prompts.
        _case("prompt_ragged", "attend", B=8, nlo=16, nhi=4096, lse=True, dtype="f16"),
        # One long prompt through a window with sinks, a shard of the heads.
        _case("prompt_window", "attend", B=1, nlo=32768, nhi=32768, Hq=8, Hkv=1, window=4096, sinks=4),
        # Two chunks of long prompts behind their cached contexts together
        # with 62 requests that generate: one iteration under inflight
        # batching.
        _case("mixed_chunks", "attend", B=2, lo=9001, hi=16384, nlo=512, nhi=512, decodes=62, N=24),
        # Sequences forked (shared prompt, several answers): 64 forks with up
        # to 300 new tokens each, over the largest board's pool; then freed.
        _case("pages_fork", "fork", B=16, lo=16, hi=2304, decodes=64, grow=300, planes=8, pool=131072, Hkv=1),
        # A pool after long service, its live pages moved to the front.
        _case("pages_compact", "compact", B=256, lo=16, hi=2304, planes=8, pool=65536, Hkv=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "attend", "attend", "fork", "compact"])
    Hkv = rng.choice([1, 2, 4, 5, 8, 8])
    c = dict(Hkv=Hkv, Hq=Hkv * rng.choice([1, 2, 4, 4, 5, 8]), D=rng.choice([64, 128, 128, 128, 80, 256]),
             N=rng.choice([16, 16, 24, 32, 7, 64]), dtype=rng.choice(["bf16", "f16"]),
             order=rng.choice(["head", "token"]))
    if kind == "append":
        if rng.random() < 0.5:
            c.update(B=_log(rng, 1, 512), lo=1, hi=_log(rng, 2, 4352))
        else:
            c.update(B=rng.randint(1, 32), nlo=1, nhi=_log(rng, 16, 4096))
    elif kind == "attend":
        form = rng.choice(["decode", "decode", "prompt", "chunk", "mixed"])
        c.update(lse=rng.random() < 0.3)
        if rng.random() < 0.4:
            c.update(window=_log(rng, 1, 4096), sinks=rng.choice([0, 1, 4, 100]))
        if form == "decode":
            B = _log(rng, 1, 256)
            c.update(B=B, lo=1, hi=_log(rng, 16, min(36864, (1 << 21) // B // Hkv * 2)))
        elif form == "prompt":
            B = rng.randint(1, 8)
            c.update(B=B, nlo=1, nhi=_log(rng, 16, int(math.sqrt((1 << 28) / B / c["Hq"]) * 2)))
        elif form == "chunk":
            n, B = _log(rng, 2, 1024), rng.randint(1, 4)
            most = int(2e11 / (4 * c["D"] * c["Hq"] * B * n))
            c.update(B=B, lo=0, hi=_log(rng, 16, max(17, min(16384, most))), nlo=max(1, n // 2), nhi=n)
        else:
            n, B, extra = _log(rng, 2, 512), rng.randint(1, 3), rng.randint(1, 48)
            most = int(8e9 / ((B + extra) * n * c["Hq"]))
            c.update(B=B, lo=1, hi=_log(rng, 16, max(17, min(8192, most))), nlo=n, nhi=n, decodes=extra)
    elif kind == "fork":
        c.update(B=_log(rng, 1, 64), lo=1, hi=_log(rng, 16, 2304), decodes=_log(rng, 1, 96), grow=rng.randint(0, 400),
                 planes=rng.choice([2, 4, 8]), Hkv=rng.choice([1, 2]))
        # sometimes fewer free pages than the forks want
        n = int(_pages(_lengths(_case("", kind, **c))[0], c["N"]).sum())
        c.update(pool=n + rng.choice([rng.randint(0, 200), c["decodes"] * (c["grow"] // c["N"] + 2) + rng.randint(0, 4000)]))
    else:
        c.update(B=_log(rng, 1, 256), lo=1, hi=_log(rng, 16, 2304), planes=rng.choice([2, 4, 8]),
                 Hkv=rng.choice([1, 2, 4]), D=rng.choice([64, 128]))
        c.update(pool=int(c["B"] * (c["hi"] // c["N"] + 2) * rng.uniform(1.1, 1.6)) + 3)
    return {k: v for k, v in _case("", kind, **c).items() if k != "name"}


# ---------------------------------------------------------------- the case's own numbers

def _lengths(case):
    """(length before the pass, new tokens) per sequence, from the case alone."""
    rng = np.random.RandomState([case["B"], case["lo"], case["hi"], case["nlo"], case["nhi"], case["decodes"]])
    B, extra = case["B"], case["decodes"] if case["kind"] == "attend" else 0
    old = rng.randint(case["lo"], case["hi"] + 1, B + extra)
    new = np.ones(B + extra, np.int64)
    if case["nhi"]:
        new[:B] = rng.randint(case["nlo"], case["nhi"] + 1, B)
    if case["kind"] in ("fork", "compact"):
        new[:] = 0
    old[:1] = case["hi"]                     # one at each end of the range
    if case["nhi"]:
        new[:1] = case["nhi"]
    return old.astype(np.int64), new


def _pages(tokens, N):
    return -(-tokens // N)


def _visible(case):
    """(query-key pairs seen, keys seen by some query of their sequence)."""
    old, new = _lengths(case)
    W, S = case["window"], case["sinks"]
    pairs = keys = 0
    for a, n in zip(old, new):
        p = np.arange(a, a + n)
        if not W:
            pairs += int((p + 1).sum())
            keys += int(a + n)
        else:
            lo = np.maximum(p - W + 1, 0)
            pairs += int((p + 1 - lo + np.minimum(lo, S)).sum())
            first = max(int(a) - W + 1, 0)
            keys += int(a + n) - first + min(first, S)
    return pairs, keys


def work(case):
    old, new = _lengths(case)
    e, N = 2, case["N"]
    row = case["Hkv"] * case["D"] * e
    if case["kind"] == "append":
        T = int(new.sum())
        return {"bytes": 4 * T * row + 4 * T + 8 * len(new), "flops": 0}
    if case["kind"] == "attend":
        pairs, keys = _visible(case)
        T = int(new.sum())
        return {"bytes": 2 * keys * row + 2 * T * case["Hq"] * case["D"] * e + 4 * keys // N,
                "flops": 4 * pairs * case["Hq"] * case["D"]}
    page = case["planes"] * N * row
    if case["kind"] == "fork":
        parent = _parents(case)
        L = old[parent]
        part = int((L % N != 0).sum())
        entries = int((_pages(L + case["grow"], N)).sum())
        return {"bytes": 2 * part * page + 4 * 4 * entries, "flops": 0}
    n = int(_pages(old, N).sum())
    moved = _moved(case, n)
    return {"bytes": 2 * moved * page + 4 * (2 * case["pool"] + 2 * n), "flops": 0}


def _parents(case):
    return np.random.RandomState([case["B"], case["decodes"]]).randint(0, case["B"], case["decodes"])


def _places(case, n):
    """n distinct pages of the pool: a fragmented pool's own order."""
    rng = np.random.RandomState([case["pool"], n])
    return rng.permutation(case["pool"])[:n]


def _moved(case, n):
    return int((_places(case, n) >= n).sum())


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    old, new = _lengths(case)
    Hq, Hkv, D, N = case["Hq"], case["Hkv"], case["D"], case["N"]
    dev = lambda a, t=torch.int32: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", t)

    def randn(*shape, std=1.0):
        x = torch.empty(shape, dtype=dt, device="cuda")
        return x.normal_(0.0, std, generator=g)

    s = dict(case=dict(case))
    if case["kind"] in ("append", "attend"):
        have = _pages(old + new, N)
        pool = int(have.sum()) + 3
        width = int(have.max())
        # a table of pages in no order, as after some time of service
        place = torch.randperm(pool, generator=g, device="cuda")[: int(have.sum())]
        at = np.concatenate([np.arange(b * width, b * width + h) for b, h in enumerate(have)])
        table = torch.full((len(old) * width,), -1, dtype=torch.int32, device="cuda")
        table[torch.from_numpy(at).cuda()] = place.to(torch.int32)
        s.update(table=table.view(len(old), width), length=dev(old + new))
        s["offset"] = dev(np.concatenate([[0], np.cumsum(new)]), torch.int64) if case["nhi"] else None
        shape = (pool, Hkv, N, D) if case["order"] == "head" else (pool, N, Hkv, D)
        k, v = randn(*shape), randn(*shape)
        if case["order"] == "token":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        # queries, keys and values as one product of a layer leaves them;
        # queries wider than unit, so that some tokens weigh more
        T = int(new.sum())
        qkv = randn(T, Hq + 2 * Hkv, D)
        qkv[:, :Hq] *= 1.5
        s.update(k=k, v=v, q=qkv[:, :Hq], newk=qkv[:, Hq:Hq + Hkv], newv=qkv[:, Hq + Hkv:])
        return s
    pool, planes = case["pool"], case["planes"]
    have = _pages(old, N)
    n = int(have.sum())
    s["pages"] = randn(planes, pool, Hkv, N, D)
    extra = case["decodes"]
    width = int(_pages(np.int64(case["hi"] + case["grow"]), N))
    place = _places(case, n).astype(np.int64)
    if case["kind"] == "compact":            # which sequence has which page goes by the seed
        place = place[torch.randperm(n, generator=g, device="cuda").cpu().numpy()]
    table = np.full((len(old) + extra, width), -1, np.int64)
    table[: len(old)][np.arange(width) < have[:, None]] = place
    ref = np.zeros(pool, np.int64)
    ref[place] = 1
    s.update(ref=dev(ref), table=dev(table), length=dev(np.concatenate([old, np.zeros(extra, np.int64)])))
    if case["kind"] == "fork":
        s.update(parent=dev(_parents(case)), child=dev(np.arange(extra) + case["B"]),
                 add=dev(np.concatenate([np.zeros(len(old)), np.full(extra, case["grow"])])))
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2408_05235_amd import api
    c = s["case"]
    if c["kind"] == "append":
        api.tl_kv_append(s["newk"], s["newv"], s["k"], s["v"], s["table"], s["length"], s["offset"])
        return [s["k"], s["v"]]
    if c["kind"] == "attend":
        r = api.tl_attend(s["q"], s["k"], s["v"], s["table"], s["length"], s["offset"], window=c["window"],
                          sinks=c["sinks"], want_lse=c["lse"])
        return list(r) if c["lse"] else [r]
    if c["kind"] == "fork":
        ref, table, length, N = s["ref"], s["table"], s["length"], c["N"]
        src, dst, status = api.tl_pages_fork(ref, table, length, s["parent"], s["child"], N)
        api.tl_pages_copy(s["pages"], src, dst)
        grown = api.tl_pages_extend(ref, table, length, s["add"], N)
        api.tl_pages_free(ref, table, length, s["child"], N)
        return dict(pages=s["pages"], table=table, ref=ref, length=length, src=src, dst=dst, status=status, grown=grown)
    r = api.tl_pages_compact(s["ref"], s["table"], s["length"], c["N"])
    api.tl_pages_copy(s["pages"], r["copy_src"], r["copy_dst"], r["n_copies"])
    return dict(pages=s["pages"], ref=r["ref"], table=r["page_table"], n=r["n_copies"])


def _new_tokens(s):
    """Sequence and position of every new token."""
    length = s["length"].long()
    if s["offset"] is None:
        return torch.arange(length.numel(), device=length.device), length - 1
    off, T = s["offset"], s["q"].shape[0]
    token = torch.arange(T, device=off.device)
    seq = torch.searchsorted(off, token, right=True) - 1
    return seq, length[seq] - (off[seq + 1] - token)


def _run_plain(s):
    c = s["case"]
    N, D, Hq, Hkv = c["N"], c["D"], c["Hq"], c["Hkv"]
    if c["kind"] == "append":
        seq, pos = _new_tokens(s)
        page = s["table"][seq, pos // N].long()
        s["k"].transpose(1, 2)[page, pos % N] = s["newk"]
        s["v"].transpose(1, 2)[page, pos % N] = s["newv"]
        return [s["k"], s["v"]]
    if c["kind"] == "attend":
        return _attend_plain(s)
    if c["kind"] == "fork":
        return _fork_plain(s)
    ref, table, pool = s["ref"], s["table"], c["pool"]
    live = ref > 0
    before = torch.cumsum(live, 0) - live.long()
    n_live = live.sum()
    at = torch.arange(pool, device=ref.device)
    hole = ~live & (at < n_live)
    mover = live & (at >= n_live)
    # the i-th mover goes to the i-th hole: both in ascending order
    holes = torch.sort((~hole).to(torch.int8), stable=True).indices
    movers = torch.sort((~mover).to(torch.int8), stable=True).indices
    n = mover.sum()
    rank = torch.cumsum(mover, 0) - 1
    to = torch.where(mover, holes[rank.clamp(min=0)], at)
    used = torch.arange(table.shape[1], device=ref.device) < ((s["length"].long() + N - 1) // N)[:, None]
    new_table = torch.where(used, to[table.long().clamp(min=0)].to(torch.int32), table)
    new_ref = torch.zeros_like(ref).scatter_(0, to, torch.where(live, ref, 0), reduce="add")
    k = int(n)
    s["pages"][:, holes[:k]] = s["pages"][:, movers[:k]]
    return dict(pages=s["pages"], ref=new_ref, table=new_table, n=n.to(torch.int32).reshape(1))


def _fork_plain(s):
    c = s["case"]
    N = c["N"]
    ref, table, length = s["ref"], s["table"], s["length"]
    parent, child = s["parent"].long(), s["child"].long()
    # children share the full pages; the partly filled one is copied
    L = length[parent].long()
    part = L % N != 0
    free = torch.sort((ref > 0).to(torch.int8), stable=True).indices
    n_free = (ref == 0).sum()
    before = torch.cumsum(part, 0)
    fits = (before <= n_free) | ~part
    part &= fits
    page = free[(before - 1).clamp(min=0)]
    rows = table[parent].clone()
    full = (torch.arange(table.shape[1], device=L.device) < (L // N)[:, None]) & fits[:, None]
    last = (L // N).clamp(max=table.shape[1] - 1)
    source = rows.gather(1, last[:, None])[:, 0]
    none = torch.full_like(source, -1)
    src, dst = torch.where(part, source, none), torch.where(part, page.to(torch.int32), none)
    kept = table[child].clone()
    kept = torch.where(full, rows, kept)
    kept.scatter_(1, last[:, None], torch.where(part, dst, kept.gather(1, last[:, None])[:, 0])[:, None])
    table[child] = kept
    ref.scatter_add_(0, torch.where(full, rows, 0).long().reshape(-1), full.reshape(-1).to(torch.int32))
    ref.scatter_add_(0, torch.where(part, dst, 0).long(), part.to(torch.int32))
    length[child] = torch.where(fits, L, 0).to(torch.int32)
    status = (~fits).to(torch.int32)
    # (a fork without a copy writes its parent's last page over itself)
    same = rows.gather(1, ((L - 1) // N).clamp(min=0)[:, None])[:, 0]
    s["pages"][:, torch.where(part, dst, same).long()] = s["pages"][:, torch.where(part, src, same).long()]
    # every sequence gets the pages for its further tokens
    old, add = length.long(), s["add"].long()
    have, need = (old + N - 1) // N, (old + add + N - 1) // N
    short = need > table.shape[1]
    want = torch.where(short, 0, need - have)
    free = torch.sort((ref > 0).to(torch.int8), stable=True).indices
    ends = torch.cumsum(want, 0)
    ok = ((ends <= (ref == 0).sum()) | (want == 0)) & ~short
    j = torch.arange(table.shape[1], device=L.device)
    fresh = (j >= have[:, None]) & (j < need[:, None]) & ok[:, None]
    pick = free[((ends - want)[:, None] + j - have[:, None]).clamp(0, ref.numel() - 1)]
    table.copy_(torch.where(fresh, pick.to(torch.int32), table))
    ref.scatter_add_(0, torch.where(fresh, pick, 0).reshape(-1), fresh.reshape(-1).to(torch.int32))
    length.copy_(torch.where(ok, old + add, old).to(torch.int32))
    grown = torch.where(short, 2, (~ok).long()).to(torch.int32)
    # the forks leave again
    used = j < ((length[child].long() + N - 1) // N)[:, None]
    ref.scatter_add_(0, torch.where(used, table[child], 0).long().reshape(-1), -used.reshape(-1).to(torch.int32))
    length[child] = 0
    return dict(pages=s["pages"], table=table, ref=ref, length=length, src=src, dst=dst, status=status, grown=grown)


def _attend_plain(s):
    c = s["case"]
    N, D, Hq, Hkv, W = c["N"], c["D"], c["Hq"], c["Hkv"], c["window"]
    G = Hq // Hkv
    B, width = s["table"].shape
    length = s["length"].long()
    at = s["table"].long().clamp(min=0)
    K = s["k"][at].transpose(1, 2).reshape(B, Hkv, width * N, D).float()
    V = s["v"][at].transpose(1, 2).reshape(B, Hkv, width * N, D).float()
    seq, pos = _new_tokens(s)
    if s["offset"] is None:
        most, row = 1, torch.zeros_like(seq)
    else:
        most, row = max(c["nhi"], 1), torch.arange(seq.numel(), device=seq.device) - s["offset"][seq]
    # queries by (sequence, kv head, token of the sequence, head of the group)
    Q = torch.zeros(B, most, Hq, D, device=K.device)
    Q[seq, row] = s["q"].float()
    Q = Q.view(B, most, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, most * G, D)
    at_pos = torch.full((B, most), -1, dtype=torch.int64, device=K.device)
    at_pos[seq, row] = pos
    t = torch.arange(width * N, device=K.device)
    see = t <= at_pos[:, :, None]
    if W:
        see &= (t > at_pos[:, :, None] - W) | (t < c["sinks"])
    V = torch.where((t < length[:, None])[:, None, :, None], V, 0.0)
    x = torch.matmul(Q, K.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).view(B, Hkv, most, G, width * N)
    x.masked_fill_(~see[:, None, :, None, :], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = x.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, most * G, width * N), V).view(B, Hkv, most, G, D)
    o = o / torch.where(l == 0, 1.0, l)
    out = o.permute(0, 2, 1, 3, 4).reshape(B, most, Hq, D)[seq, row].to(s["q"].dtype)
    if not c["lse"]:
        return [out]
    lse = (m + torch.log(l)).squeeze(-1).permute(0, 2, 1, 3).reshape(B, most, Hq)[seq, row]
    return [out, lse]


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The definition in float64, sequence by sequence and head by head."""
    s = prepare(case, seed)
    if case["kind"] == "append":
        seq, pos = _new_tokens(s)
        k, v = s["k"].clone(), s["v"].clone()
        for h in range(case["Hkv"]):
            page = s["table"].long()[seq, pos // case["N"]]
            k[page, h, pos % case["N"]] = s["newk"][:, h]
            v[page, h, pos % case["N"]] = s["newv"][:, h]
        return [k, v]
    if case["kind"] == "fork":
        # pages hold what they held, those that a fork copies to apart
        old, _ = _lengths(case)
        N, pages = case["N"], s["pages"].clone()
        table = s["table"].cpu().numpy()
        free = np.flatnonzero(s["ref"].cpu().numpy() == 0)
        for i, p in enumerate([p for p in _parents(case) if old[p] % N][: len(free)]):
            pages[:, int(free[i])] = s["pages"][:, int(table[p, old[p] // N])]
        return dict(pages=pages, table=None, ref=None, length=None, src=None, dst=None, status=None, grown=None)
    if case["kind"] == "compact":
        ref, pages = s["ref"].cpu().numpy(), s["pages"].clone()
        n = int((ref > 0).sum())
        holes, movers = np.flatnonzero(ref[:n] == 0), n + np.flatnonzero(ref[n:] > 0)
        pages[:, torch.from_numpy(holes).cuda()] = s["pages"][:, torch.from_numpy(movers).cuda()]
        return dict(pages=pages, ref=None, table=None, n=None)
    N, D, Hq, Hkv, W, S = (case[k] for k in ("N", "D", "Hq", "Hkv", "window", "sinks"))
    if 4.0 * _visible(case)[0] * Hq * D > 2e13:
        return None
    old, new = _lengths(case)
    T = int(new.sum())
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(T, Hq, dtype=torch.float64, device="cuda")
    first = 0
    for b, (a, n) in enumerate(zip(old.tolist(), new.tolist())):
        idx = torch.arange(a + n, device="cuda")
        page, line = s["table"][b].long()[idx // N], idx % N
        for h in range(Hkv):
            kb, vb = s["k"][page, h, line].double(), s["v"][page, h, line].double()
            for r in range(0, n, 2048):
                p = torch.arange(a + r, a + min(n, r + 2048), device="cuda")[:, None]
                hidden = idx[None] > p
                if W:
                    hidden |= (idx[None] <= p - W) & (idx[None] >= S)
                for q in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                    rows = slice(first + r, first + min(n, r + 2048))
                    x = s["q"][rows, q].double() @ kb.T / math.sqrt(D)
                    x[hidden] = -math.inf
                    lse[rows, q] = torch.logsumexp(x, 1)
                    out[rows, q] = torch.exp(x - lse[rows, q][:, None]) @ vb
        first += n
    return [out, lse] if case["lse"] else [out]
