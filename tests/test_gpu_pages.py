"""The paged cache's pool against a plain model of it: rows written, pages given
out, shared, freed, moved and copied; whole numbers and copies, so all equal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

dev = lambda a, t=torch.int32: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", t)
host = lambda x: x.cpu().numpy()
pages_of = lambda tokens, N: -(-int(tokens) // N)


class Model:
    """The pool in plain Python."""

    def __init__(self, ref, table, length, N):
        self.ref, self.table, self.length, self.N = ref.copy(), table.copy(), length.copy(), N

    def free_pages(self):
        return [int(p) for p in np.flatnonzero(self.ref == 0)]

    def extend(self, add):
        W, free, status, given, asked = self.table.shape[1], self.free_pages(), [], [], 0
        for b, a in enumerate(add):
            L = int(self.length[b])
            if L < 0 or a < 0:
                status.append(3)
                continue
            if L + a > W * self.N:
                status.append(2)
                continue
            have, need = pages_of(L, self.N), pages_of(L + a, self.N) - pages_of(L, self.N)
            if need and asked + need > len(free):
                status.append(1)
            else:
                given.append((b, have, free[asked:asked + need], L + a))
                status.append(0)
            asked += need
        for b, have, got, L in given:
            self.table[b, have:have + len(got)] = got
            self.ref[got] = 1
            self.length[b] = L
        return np.asarray(status)

    def fork(self, parent, child):
        S, W = self.table.shape
        free, asked, seen, todo, res = self.free_pages(), 0, set(), [], []
        for p, c in zip(parent, child):
            ok = 0 <= c < S and 0 <= p < S
            first = ok is False or c not in seen
            if 0 <= c < S:
                seen.add(c)
            L = int(self.length[p]) if ok else -1
            if not ok or not first or self.length[c] != 0 or L < 0 or L > W * self.N:
                res.append((-1, -1, 3))
                continue
            full, part = L // self.N, L % self.N != 0
            if part:
                asked += 1
                if asked > len(free):
                    res.append((-1, -1, 1))
                    continue
            todo.append((c, self.table[p, :full].copy(), free[asked - 1] if part else None, L))
            res.append((int(self.table[p, full]), free[asked - 1], 0) if part else (-1, -1, 0))
        for c, rows, page, L in todo:
            self.table[c, :len(rows)] = rows
            np.add.at(self.ref, rows[(rows >= 0) & (rows < len(self.ref))], 1)
            if page is not None:
                self.table[c, len(rows)] = page
                self.ref[page] = 1
            self.length[c] = L
        return np.asarray(res).reshape(-1, 3).T

    def free(self, slots):
        for s in slots:
            if 0 <= s < len(self.length):
                for p in self.table[s, :min(pages_of(max(self.length[s], 0), self.N), self.table.shape[1])]:
                    if 0 <= p < len(self.ref):
                        self.ref[p] -= 1
                self.length[s] = 0

    def compact(self):
        live = np.flatnonzero(self.ref > 0)
        n = len(live)
        movers, holes = live[live >= n], np.flatnonzero(self.ref[:n] <= 0)
        to = {int(p): int(p) for p in live[live < n]}
        to.update({int(a): int(b) for a, b in zip(movers, holes)})
        table = self.table.copy()
        for s, L in enumerate(self.length):
            for i in range(min(pages_of(max(L, 0), self.N), table.shape[1])):
                if 0 <= table[s, i] < len(self.ref):
                    table[s, i] = to.get(int(table[s, i]), -1)
        ref = np.zeros_like(self.ref)
        for a, b in to.items():
            ref[b] = self.ref[a]
        self.ref, self.table = ref, table
        return movers, holes

    def device(self):
        return dev(self.ref), dev(self.table), dev(self.length)

    def same(self, ref, table, length):
        assert np.array_equal(host(ref), self.ref)
        assert np.array_equal(host(table), self.table)
        assert np.array_equal(host(length), self.length)


def random_pool(seed, n_pages, slots, width, N, fill):
    r = np.random.RandomState(seed)
    m = Model(np.zeros(n_pages, np.int64), np.full((slots, width), -1, np.int64), np.zeros(slots, np.int64), N)
    free = list(r.permutation(n_pages))
    for b in range(slots):
        if r.random_sample() < fill:
            L = int(r.randint(0, width * N + 1))
            k = pages_of(L, N)
            if k > len(free):
                continue
            got = [free.pop() for _ in range(k)]
            m.table[b, :k], m.ref[got], m.length[b] = got, 1, L
    return m, r


POOLS = [(0, 1, 1, 4, 16), (1, 50, 7, 9, 16), (2, 4096, 40, 30, 7), (3, 5000, 1030, 6, 24), (4, 20000, 300, 64, 1),
         (5, 140001, 2500, 40, 16), (6, 63, 64, 3, 65536)]


@pytest.mark.parametrize("seed,n_pages,slots,width,N", POOLS)
def test_extend(gpu, seed, n_pages, slots, width, N):
    from paper_2408_05235_amd import api
    for fill in (0.0, 0.5, 1.0):
        m, r = random_pool(seed, n_pages, slots, width, N, fill)
        for most in (1, N, width * N):
            add = r.randint(-1 if most > 1 else 0, most + 1, slots)
            print("extend", n_pages, slots, fill, most, flush=True)
            ref, table, length = m.device()
            st = api.tl_pages_extend(ref, table, length, dev(add), N)
            exp = m.extend(add)
            assert np.array_equal(host(st), exp)
            m.same(ref, table, length)


@pytest.mark.parametrize("seed,n_pages,slots,width,N", POOLS)
def test_fork_and_free(gpu, seed, n_pages, slots, width, N):
    from paper_2408_05235_amd import api
    for fill in (0.2, 0.7):
        m, r = random_pool(seed + 10, n_pages, slots, width, N, fill)
        for _ in range(3):
            F = int(r.randint(1, slots + 1))
            parent, child = r.randint(-1, slots + 1, F), r.randint(-1, slots + 1, F)
            print("fork", n_pages, slots, F, flush=True)
            ref, table, length = m.device()
            got = api.tl_pages_fork(ref, table, length, dev(parent), dev(child), N)
            exp = m.fork(parent, child)
            for g, e in zip(got, exp):
                assert np.array_equal(host(g), e)
            m.same(ref, table, length)
            out = r.randint(-2, slots + 2, int(r.randint(1, slots + 3)))
            api.tl_pages_free(ref, table, length, dev(out), N)
            m.free(out)
            m.same(ref, table, length)


@pytest.mark.parametrize("seed,n_pages,slots,width,N", POOLS)
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(gpu, seed, n_pages, slots, width, N, in_place):
    from paper_2408_05235_amd import api
    for fill in (0.0, 0.3, 0.9):
        m, r = random_pool(seed + 20, n_pages, slots, width, N, fill)
        if slots > 2:
            m.fork(r.randint(0, slots, slots // 3), r.randint(0, slots, slots // 3))
            if m.length[0] > 0:
                m.table[0, 0] = n_pages + 7          # not a page
            freed = np.flatnonzero(m.length == 0)
            if len(freed) and width > 1:
                m.table[freed[0], :] = 0             # stale entries of an empty slot
        print("compact", n_pages, slots, fill, flush=True)
        ref, table, length = m.device()
        before = ref.clone(), table.clone()
        got = api.tl_pages_compact(ref, table, length, N, dict(ref=ref, page_table=table) if in_place else None)
        if not in_place:
            assert torch.equal(ref, before[0]) and torch.equal(table, before[1])
        movers, holes = m.compact()
        n = int(got["n_copies"])
        assert n == len(movers)
        assert np.array_equal(host(got["copy_src"])[:n], movers) and np.array_equal(host(got["copy_dst"])[:n], holes)
        m.same(got["ref"], got["page_table"], length)


@pytest.mark.parametrize("n_pages,planes,shape,dtype", [(9, 1, (1, 1, 8), torch.bfloat16), (40, 6, (3, 7, 24), torch.float16),
                                                        (700, 4, (2, 16, 128), torch.bfloat16),
                                                        (33, 2, (8, 64, 256), torch.float16)])
def test_copy(gpu, n_pages, planes, shape, dtype):
    from paper_2408_05235_amd import api
    r = np.random.RandomState(n_pages)
    x = torch.randint(-30000, 30000, (planes, n_pages, *shape), dtype=torch.int16, device="cuda").view(dtype)
    perm = r.permutation(n_pages)
    k = n_pages // 2
    src, dst = perm[:k].copy(), perm[k:2 * k].copy()
    src[0], dst[-1] = -1, n_pages                     # no pages: skipped
    for count in (None, 0, k // 2, k + 9):
        y, e = x.clone(), x.clone().view(torch.int16)
        use = k if count is None else min(count, k)
        for s, d in zip(src[:use], dst[:use]):
            if 0 <= s < n_pages and 0 <= d < n_pages:
                e[:, int(d)] = x.view(torch.int16)[:, int(s)]
        api.tl_pages_copy(y, dev(src), dev(dst), None if count is None else dev([count]))
        assert torch.equal(y.view(torch.int16), e)


@pytest.mark.parametrize("B,most,heads,dim,N,order,dtype", [(1, 1, 1, 8, 1, "head", "f16"), (70, 1, 8, 128, 16, "head", "bf16"),
                                                            (9, 300, 3, 80, 24, "token", "bf16"),
                                                            (40, 400, 2, 256, 7, "head", "f16")])
def test_append(gpu, B, most, heads, dim, N, order, dtype):
    from paper_2408_05235_amd import api
    from cache_cases import DTYPES
    r = np.random.RandomState(B)
    new = np.ones(B, np.int64) if most == 1 else r.randint(0, most, B)
    length = new + r.randint(0, 500, B)
    have = np.array([pages_of(x, N) for x in length])
    pool, width = int(have.sum()) + 2, int(have.max()) + 1
    table = np.full((B, width), -1)
    place = r.permutation(pool)
    for b, at in zip(range(B), np.concatenate([[0], np.cumsum(have)[:-1]])):
        table[b, :have[b]] = place[at:at + have[b]]
    if most > 1:
        table[2, 0] = pool                            # no such page: its tokens go nowhere
        length[3] = max(new[3] - 5, 0)                # the first rows have no position
        length[4] = width * N + 3                     # the last ones no room
    T = int(new.sum()) + (3 if most > 1 else 0)       # rows of no sequence
    qkv = torch.randn(T, 5 * heads, dim, device="cuda").to(DTYPES[dtype])
    key, value = qkv[:, heads:2 * heads], torch.randn(T, heads, dim, device="cuda").to(DTYPES[dtype])
    shape = (pool, heads, N, dim) if order == "head" else (pool, N, heads, dim)
    k = torch.zeros(shape, dtype=DTYPES[dtype], device="cuda")
    v = torch.zeros_like(k)
    if order == "token":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    ek, ev = k.cpu().clone(), v.cpu().clone()
    off = np.concatenate([[0], np.cumsum(new)])
    hk, hv = key.cpu(), value.cpu()
    for b in range(B):
        for i in range(new[b]):
            p = length[b] - new[b] + i
            if 0 <= p < width * N and 0 <= table[b, p // N] < pool:
                ek[table[b, p // N], :, p % N], ev[table[b, p // N], :, p % N] = hk[off[b] + i], hv[off[b] + i]
    api.tl_kv_append(key, value, k, v, dev(table), dev(length), None if most == 1 else dev(off, torch.int64))
    assert torch.equal(k.cpu(), ek) and torch.equal(v.cpu(), ev)


def test_cache_object_round(gpu):
    """Sequences through KVCache: prompts, forks that diverge, a compaction in
    between; every step's attention against 64 bits."""
    import cache_cases as cc
    from paper_2408_05235_amd import api
    g = torch.Generator().manual_seed(5)
    N, kv, heads, dim, slots = 16, 2, 8, 64, 6
    cache = api.KVCache(2, 60, kv, N, dim, slots, 200)
    cache.pages.fill_(float("nan"))
    m = Model(host(cache.ref).astype(np.int64), host(cache.page_table).astype(np.int64),
              host(cache.length).astype(np.int64), N)
    dense = [[(torch.zeros(0, kv, dim, dtype=torch.bfloat16),) * 2 for _ in range(slots)] for _ in range(2)]

    def step(add):
        add = np.asarray(add)
        assert np.array_equal(host(cache.extend(dev(add))), m.extend(add))
        off = np.concatenate([[0], np.cumsum(add)])
        T = int(add.sum())
        for layer in range(2):
            q, k, v = (torch.randn(T, h, dim, generator=g).bfloat16() for h in (heads, kv, kv))
            cache.append(layer, k.cuda(), v.cuda(), dev(off, torch.int64))
            out = cache.attend(layer, q.cuda(), dev(off, torch.int64))
            for b in range(slots):
                new = slice(off[b], off[b + 1])
                dense[layer][b] = tuple(torch.cat([x, y[new]]) for x, y in zip(dense[layer][b], (k, v)))
            c = dict(q=q.cuda(), dense=dense[layer], before=m.length - add, new=add, window=0, sinks=0, dtype="bf16")
            cc.check(c, out, None)
        m.same(cache.ref, cache.page_table, cache.length)

    step([40, 17, 0, 0, 0, 0])
    step([1, 1, 0, 0, 0, 0])
    parent, child = np.array([0, 0, 1]), np.array([2, 4, 5])
    assert np.array_equal(host(cache.fork(dev(parent), dev(child))), m.fork(parent, child)[2])
    for layer in range(2):
        for p, c in zip(parent, child):
            dense[layer][c] = dense[layer][p]
    step([1, 1, 1, 0, 30, 1])
    cache.free(dev([0, 1]))
    m.free([0, 1])
    for layer in range(2):
        dense[layer][0] = dense[layer][1] = (torch.zeros(0, kv, dim, dtype=torch.bfloat16),) * 2
    moved = cache.compact()
    movers, _ = m.compact()
    assert int(moved) == len(movers) > 0
    m.same(cache.ref, cache.page_table, cache.length)
    assert int(cache.pages_used()) == int((m.ref > 0).sum())
    step([20, 0, 1, 5, 1, 1])
