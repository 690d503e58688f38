"""Random service on a small pool: slots extended, forked, freed and refused,
the pool compacted; what every slot holds and sees is followed token by token."""
import numpy as np
import pytest
import torch

from test_gpu_pages import Model, dev, host
from test_gpu_pool_full import LAYERS, N, OK, Served

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(6))
def test_random_service(gpu, seed):
    r = np.random.RandomState(seed)
    slots, pages = 7, int(r.choice([9, 16, 25]))
    s = Served(pages, slots, 120, seed)
    m = Model(host(s.cache.ref), host(s.cache.page_table), host(s.cache.length), N)
    refused = forks = 0

    def same():
        m.same(s.cache.ref, s.cache.page_table, s.cache.length)
        for layer in range(LAYERS):
            for b in range(slots):
                assert s.dense[layer][b][0].shape[0] == m.length[b]

    for _ in range(25):
        what = r.choice(["step", "step", "step", "grow", "fork", "free", "compact"])
        if what in ("step", "grow"):
            add = (m.length > 0).astype(np.int64) if what == "step" else r.choice([0, 0, 1, 5, 30, 60], slots)
            offsets = what == "grow" or r.rand() < 0.5
            status = s.extend(add)
            assert np.array_equal(status, m.extend(add))
            s.rows(add, np.where(status == OK, add, 0), offsets)
            refused += int((status != OK).sum())
        elif what == "fork":
            parent, child = r.randint(0, slots, 2), r.randint(0, slots, 2)
            status = host(s.cache.fork(dev(parent), dev(child)))
            before = [list(d) for d in s.dense]
            assert np.array_equal(status, m.fork(parent, child)[2])
            for layer in range(LAYERS):
                for p, c, st in zip(parent, child, status):
                    if st == OK:
                        s.dense[layer][c] = before[layer][p]
            forks += int((status == OK).sum())
        elif what == "free":
            gone = r.randint(0, slots, 2)
            s.cache.free(dev(gone))
            m.free(gone)
            for layer in range(LAYERS):
                for b in gone:
                    s.dense[layer][b] = tuple(x[:0] for x in s.dense[layer][b])
        else:
            moved = int(s.cache.compact())
            assert moved == len(m.compact()[0])
        same()
    # what is left reads as it was written
    for layer in range(LAYERS):
        table = host(s.cache.page_table)
        for b in range(slots):
            t = torch.arange(int(m.length[b]))
            page = torch.from_numpy(table[b].astype(np.int64))[t // N]
            for plane in range(2):
                got = s.cache.pages[layer, plane].cpu()[page, :, t % N]
                assert torch.equal(got, s.dense[layer][b][plane].view_as(got)), (layer, b)
    assert refused or forks
