"""What a row does not see changes no bit of it."""
import math

import pytest
import torch

import cache_cases as cc

pytestmark = pytest.mark.gpu


def run(c, **kw):
    from paper_2408_05235_amd import api
    return api.tl_attend(c["q"], c["k"], c["v"], c["table"], c["length"], c["offset"], window=c["window"],
                         sinks=c["sinks"], want_lse=True, **kw)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64), ("bf16", 80), ("f16", 256)])
@pytest.mark.parametrize("new", [2, 5, 8, 40])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_what_no_row_sees_changes_no_bit(gpu, dtype, dim, new, window, sinks):
    """Finite or not: free pages (the first one among them), the rest of the
    last page, tokens before every row's window."""
    c = cc.make(21, dtype, 4, 2, dim, 16, [70, 3, 31], [new] * 3, window, sinks, poison=False)
    table, k, v = c["table"], c["k"], c["v"]
    spare = [p for p in range(k.shape[0]) if not bool((table == p).any())]
    if 0 not in spare:                          # page 0 is nobody's
        k[spare[0]], v[spare[0]] = k[0], v[0]
        table[table == 0] = spare[0]
        spare[0] = 0
    table[0, 1] = -1                            # tokens without a page
    ref = run(c)
    assert bool(torch.isfinite(ref[0]).all())
    hidden = [(p, slice(0, 16)) for p in spare]
    for b, (before, n) in enumerate(zip(c["before"], c["new"])):
        end = int(before + n)
        if end % 16:
            hidden.append((int(table[b, end // 16]), slice(end % 16, 16)))
        for t in range(sinks, max(int(before) - window + 1, 0) if window else 0):
            if int(table[b, t // 16]) >= 0:
                hidden.append((int(table[b, t // 16]), slice(t % 16, t % 16 + 1)))
    for value in (math.nan, math.inf):
        for page, rows in hidden:
            k[page, :, rows], v[page, :, rows] = value, value
        out, lse = run(c)
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1]), value
