"""The engine on a pool that is too small: requests without room stop, with the
tokens that they have; the others do not notice."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

PROMPT, DONE = np.array([40, 30, 17, 64, 5]), np.array([0, 3, 15, 0, 1])
LEFT, N = np.array([60, 9, 60, 60, 60]), 16


def in_order(capacity, iterations):
    """Pages taken in the requests' order, a request that does not fit stopping:
    its tokens after each iteration, and which ones have stopped."""
    tokens, stopped, log = np.zeros(5, np.int64), np.zeros(5, bool), []
    pages = lambda t: -(-t // N)
    for j in range(iterations + 1):
        if j:
            tokens[LEFT == j] = 0
        add = PROMPT + DONE if j == 0 else (LEFT > j) & ~stopped
        free, asked = capacity - pages(tokens).sum(), 0
        for b in np.flatnonzero(add):
            need = pages(tokens[b] + add[b]) - pages(tokens[b])
            asked += need
            if need and asked > free:
                stopped[b] = True
            else:
                tokens[b] += add[b]
        log.append((tokens.copy(), stopped.copy()))
    return log


@pytest.mark.parametrize("capacity", [40, 14, 13, 11, 3])
def test_requests_without_room_stop(gpu, capacity):
    from paper_2408_05235_amd.engine import Engine
    e, ample = Engine(PROMPT, DONE, LEFT, N, capacity), Engine(PROMPT, DONE, LEFT, N, 40)
    log = in_order(capacity, 50)
    assert bool(log[-1][1].any()) == (capacity < 30)
    for j, (tokens, stopped) in enumerate(log):
        kept = {}
        if j:
            for b in np.flatnonzero(log[j - 1][1] & (tokens > 0)):
                kept[b] = [e.cache.pages[:, :, int(p)].clone() for p in e.cache.page_table[int(b), :-(-tokens[b] // N)]]
        x, y = (z.step() if j else z.prefill() for z in (e, ample))
        assert e.cache.length.tolist() == tokens.tolist(), j
        assert e.stopped.tolist() == stopped.tolist(), j
        assert int(e.cache.pages_used()) == int((-(-tokens // N)).sum()) <= capacity
        rows = np.repeat(~stopped, PROMPT + DONE) if j == 0 else ~stopped & (tokens > 0)
        rows = torch.from_numpy(np.flatnonzero(rows)).cuda()
        assert torch.equal(x[rows], y[rows]), j
        for b, pages in kept.items():
            for i, page in enumerate(pages):
                now = e.cache.pages[:, :, int(e.cache.page_table[int(b), i])]
                n = min(tokens[b] - i * N, N)
                assert torch.equal(now[..., :n, :], page[..., :n, :]), (j, b)
