"""Rows of a packed batch that lie before the first sequence's: whole tiles of
them are nobody's.  (The search for a tile's sequence took the largest 32-bit number
where no sequence begins at or before the tile: an unsigned 0 - 1 through a maximum
in floating point.)"""
import pytest
import torch

import cache_cases as cc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shift", [1, 127, 128, 1000])
def test_rows_before_the_first_sequence(gpu, shift):
    from paper_2408_05235_amd import api
    c = cc.make(21, "bf16", 4, 2, 64, 16, [10, 40, 5], [40, 8, 300])
    q = torch.cat([torch.ones(shift, 4, 64, dtype=c["q"].dtype, device="cuda"), c["q"]])
    out = torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda")
    api.tl_attend(q, c["k"], c["v"], c["table"], c["length"], c["offset"] + shift, out=out)
    assert bool((out[:shift] == 5.0).all())
    cc.check(c, out[shift:], None)
